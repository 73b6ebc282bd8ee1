"""Measured cases of the operators that a state space language model adds to this library: the short causal convolution of a
sequence, the selective scan over a state per channel, each with its gradient and its step for single tokens, and the
log-probabilities of given tokens straight from the head's operands, in pieces of the vocabulary, with their gradient.

A case is a dict of plain values.  `prepare` makes what a program holds before the call, `run` makes one call (a training step of
an operator: the forward call and its gradient): the plain form (elementary torch operations in 32 bits, rounded once) or, where
`own` is true, the library's entry points.  `exact` gives the same results from the definitions in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda:0"

# the work of a drawn case stays within that of the largest listed case of its kind
MOST = {"conv": 8192 * 2 * 4096, "conv_train": 2048 * 8 * 2048, "scan": 2048 * 8 * 2048 * 16, "scan_train": 2048 * 8 * 2048 * 16,
        "head": 8192 * 1024 * 32768, "head_train": 4096 * 2048 * 131072}
PIECE = 1 << 28                                     # elements of a piece of the scores in the plain form


def listed():
    return [
        # one token of 64 running sequences, channels twice the width of the library's LSTM workload: what a server does per token
        dict(name="conv step", kind="conv", T=1, B=64, D=2048, K=4, dtype="bf16", silu=True, bias=True, ragged=False),
        # the prompts of two long documents
        dict(name="conv long", kind="conv", T=8192, B=2, D=4096, K=4, dtype="bf16", silu=True, bias=True, ragged=False),
        # the gradient of a training batch
        dict(name="conv train", kind="conv_train", T=2048, B=8, D=2048, K=4, dtype="bf16", silu=True, bias=True, ragged=False),
        # one token of 64 running sequences
        dict(name="scan step", kind="scan", T=1, B=64, D=2048, N=16, dtype="bf16", gated=True, softplus=True, packed=True, ragged=False),
        # the prompt of one long document: few channels, many steps
        dict(name="scan long", kind="scan", T=16384, B=1, D=2048, N=16, dtype="bf16", gated=True, softplus=True, packed=True, ragged=False),
        # the forward pass of a batch, for scoring
        dict(name="scan batch", kind="scan", T=2048, B=8, D=2048, N=16, dtype="bf16", gated=True, softplus=True, packed=True, ragged=False),
        # a training step of that batch: the forward call, which leaves behind what the gradient needs, and the gradient
        dict(name="scan train", kind="scan_train", T=2048, B=8, D=2048, N=16, dtype="bf16", gated=True, softplus=True, packed=True, ragged=False),
        # a training step on a padded batch of odd sizes, in fp32, with steps that the model made itself
        dict(name="scan train ragged", kind="scan_train", T=1001, B=5, D=333, N=10, dtype="f32", gated=False, softplus=False, packed=False, ragged=True),
        # scoring a few hundred tokens over an odd vocabulary with padded positions
        dict(name="head score odd", kind="head", N=509, K=1024, V=50021, dtype="bf16", tied=False, temperature=0.7, padded=True),
        # scoring the tokens of a batch
        dict(name="head score", kind="head", N=8192, K=1024, V=32768, dtype="bf16", tied=False, temperature=1.0, padded=False),
        # a training step of that head
        dict(name="head train", kind="head_train", N=8192, K=1024, V=32768, dtype="bf16", tied=False, temperature=1.0, padded=True),
        # a training step over a large vocabulary whose head is the embedding table itself
        dict(name="head train tied", kind="head_train", N=4096, K=2048, V=131072, dtype="bf16", tied=True, temperature=1.0, padded=True),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi) + 0.49)))))))


def draw(rng):
    kind = rng.choice(["conv", "conv_train", "scan", "scan", "scan_train", "scan_train", "head", "head_train"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind.startswith("head"):
        most = MOST[kind] if dtype == "bf16" else MOST[kind] // 16
        K = _log(rng, 64, 4096)
        V = _log(rng, 1000, min(262144, most // (K * 16)))
        if rng.random() < 0.6:
            K = K // 8 * 8
        if rng.random() < 0.5:
            V = V // 64 * 64
        N = _log(rng, 1, max(1, min(16384, most // (K * V))))
        return dict(kind=kind, N=N, K=K, V=V, dtype=dtype, tied=rng.random() < 0.5, temperature=rng.choice([1.0, 1.0, 0.7, 1.3]),
                    padded=rng.random() < 0.5)
    states = rng.choice([16, 16, 16, 8, 32, rng.randint(1, 64)]) if kind.startswith("scan") else 1
    most = MOST[kind] // states
    T = 1 if not kind.endswith("train") and rng.random() < 0.2 else _log(rng, 1, 16384)
    D = _log(rng, 16, min(8192, most // T))
    if rng.random() < 0.6:
        D = max(8, D // 8 * 8)
    B = _log(rng, 1, max(1, min(256, most // (T * D))))
    case = dict(kind=kind, T=T, B=B, D=D, dtype=dtype, ragged=rng.random() < 0.3)
    if kind.startswith("conv"):
        return dict(case, K=rng.choice([2, 3, 4, 4, 4, 5, 8]), silu=rng.random() < 0.7, bias=rng.random() < 0.7)
    return dict(case, N=states, gated=rng.random() < 0.6, softplus=rng.random() < 0.6, packed=rng.random() < 0.5)


# ---- inputs -------------------------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    kind, t = case["kind"], _dtype(case)

    def randn(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    def rand(*shape):
        return torch.rand(shape, generator=g, device=DEV)

    s = dict(case)
    if kind.startswith("head"):
        N, K, V = case["N"], case["K"], case["V"]
        w = (1.5 / math.sqrt(K)) * randn(V, K)
        tokens = torch.randint(0, V, (N,), generator=g, device=DEV)
        x = randn(N, K) + torch.where(rand(N, 1) < 0.5, 3.0, 0.0) * w[tokens]      # half of the tokens are expected ones
        s["w"] = (w if case["tied"] else w.T.contiguous()).to(t)
        s["x"] = x.to(t)
        tokens = tokens.to(torch.int32)
        if case["padded"]:
            tokens.masked_fill_(rand(N) < 0.1, -1)
        s["tokens"] = tokens
        s["logp"], s["lse"] = torch.empty(N, device=DEV), torch.empty(N, device=DEV)
        if kind == "head_train":
            s["dlogp"] = -(0.5 + rand(N)) / N                                      # of a weighted mean of the losses
            s["dx"], s["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
        return s
    T, B, D = case["T"], case["B"], case["D"]
    s["lengths"] = None
    if case["ragged"]:
        n = torch.randint(0, T + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
        n[0] = T
        s["lengths"] = n
    if kind.startswith("conv"):
        K = case["K"]
        s["x"] = randn(T, B, D).to(t)
        s["w"] = (randn(K, D) / math.sqrt(K)).to(t)
        s["b"] = 0.2 * randn(D) if case["bias"] else None
        s["before"] = randn(K - 1, B, D).to(t)                                     # the inputs ahead of the first step
        if kind == "conv":
            s["y"], s["after"] = torch.empty_like(s["x"]), torch.empty_like(s["before"])
        else:
            s["dy"] = randn(T, B, D).to(t)
            s["dx"], s["dbefore"] = torch.empty_like(s["x"]), torch.empty_like(s["before"])
            s["dw"], s["db"] = torch.empty(K, D, device=DEV), torch.empty(D, device=DEV) if case["bias"] else None
        return s
    N = case["N"]
    x = randn(T, B, D)
    s["u"] = (x * torch.sigmoid(x)).to(t)                                            # what the convolution before it gives
    steps = torch.exp(math.log(1e-3) + rand(D) * math.log(100.0))                  # each channel's own step, 0.001 to 0.1
    if case["softplus"]:
        s["delta"], s["delta_bias"] = (0.5 * randn(T, B, D)).to(t), torch.log(torch.expm1(steps))
    else:
        s["delta"], s["delta_bias"] = (steps * torch.exp(0.5 * randn(T, B, D))).to(t), None
    s["a"] = -torch.arange(1, N + 1, device=DEV) * torch.exp(0.1 * randn(D, N))
    bc = randn(T, B, 2 * N).to(t)
    s["b"], s["c"] = (bc, None) if case["packed"] else (bc[..., :N].contiguous(), bc[..., N:].contiguous())
    s["d"] = 1.0 + 0.1 * randn(D)
    s["z"] = randn(T, B, D).to(t) if case["gated"] else None
    s["h0"] = randn(B, D, N)
    s["y"], s["h_final"] = torch.empty_like(s["u"]), torch.empty(B, D, N, device=DEV)
    if kind == "scan_train":
        s["dy"], s["dh_final"] = randn(T, B, D).to(t), 0.1 * randn(B, D, N)
        for k in ("u", "delta", "b", "c", "z", "a", "d", "delta_bias", "h0"):
            s["d" + k] = None if s[k] is None else torch.empty_like(s[k])
    return s


# ---- the plain forms ----------------------------------------------------------------------------------
def _inside(s):
    if s["lengths"] is None:
        return None
    return (torch.arange(s["T"], device=DEV)[:, None] < s["lengths"][None, :])[:, :, None]


def _silu_slope(x):
    p = torch.sigmoid(x)
    return p * (1.0 + x * (1.0 - p))


def _taps(s):
    """All inputs in fp32, those ahead of the first step in front; what lies behind a sequence's end is not used."""
    x, inside = s["x"].float(), _inside(s)
    if inside is not None:
        x = torch.where(inside, x, 0.0)
    return torch.cat([s["before"].float(), x]), inside


def _conv_sum(s, x):
    T, K, w = s["T"], s["K"], s["w"].float()
    y = torch.zeros_like(x[:T]) if s["b"] is None else s["b"].expand(T, s["B"], s["D"]).clone()
    for k in range(K):
        y += w[k] * x[k:k + T]
    return y


def _conv(s):
    x, inside = _taps(s)
    y = _conv_sum(s, x)
    if s["silu"]:
        y = y * torch.sigmoid(y)
    if inside is not None:
        y = torch.where(inside, y, 0.0)
        at = s["lengths"].long()[None, :] + torch.arange(s["K"] - 1, device=DEV)[:, None]
        after = torch.gather(x, 0, at[:, :, None].expand(-1, -1, s["D"]))
    else:
        after = x[s["T"]:]
    return y.to(s["x"].dtype), after.to(s["x"].dtype)


def _conv_grad(s):
    T, K, t = s["T"], s["K"], s["x"].dtype
    x, inside = _taps(s)
    g = s["dy"].float()
    if inside is not None:
        g = torch.where(inside, g, 0.0)
    if s["silu"]:
        g = g * _silu_slope(_conv_sum(s, x))
    w, dx = s["w"].float(), torch.zeros_like(x)
    dw = torch.empty(K, s["D"], device=DEV)
    for k in range(K):
        dx[k:k + T] += w[k] * g
        dw[k] = torch.sum(g * x[k:k + T], dim=(0, 1))
    db = None if s["b"] is None else torch.sum(g, dim=(0, 1))
    return dx[K - 1:].to(t), dw, db, dx[:K - 1].to(t)


def _scan(a, b):
    """h[t] = a[t] h[t-1] + b[t] with h[-1] = 0, by doubling the span that each step has summed up; overwrites a and b."""
    k = 1
    while k < a.shape[0]:
        b[k:] += a[k:] * b[:-k]
        a[k:] = a[k:] * a[:-k]
        k *= 2
    return b


def _scan_parts(s):
    """Everything in fp32: inputs, steps, decays (T,B,D,N); steps behind a sequence's end change nothing."""
    N = s["N"]
    u, raw = s["u"].float(), s["delta"].float()
    b, c = (s["b"][..., :N], s["b"][..., N:]) if s["c"] is None else (s["b"], s["c"])
    b, c = b.float(), c.float()
    if s["delta_bias"] is not None:
        raw = raw + s["delta_bias"]
    step = torch.clamp(raw, min=0.0) + torch.log1p(torch.exp(-torch.abs(raw))) if s["softplus"] else raw
    inside = _inside(s)
    if inside is not None:
        u, step, b, c = (torch.where(inside, v, 0.0) for v in (u, step, b, c))
    decay = torch.exp(step[..., None] * s["a"])
    return u, raw, step, b, c, decay, inside


def _scan_forward(s, parts):
    u, raw, step, b, c, decay, inside = parts
    add = (step * u)[..., None] * b[:, :, None, :]
    add[0] += decay[0] * s["h0"]
    h = _scan(decay.clone(), add)
    y = torch.sum(h * c[:, :, None, :], dim=3) + s["d"] * u
    return h, y


def _selective_scan(s):
    parts = _scan_parts(s)
    h, y = _scan_forward(s, parts)
    if s["z"] is not None:
        z = s["z"].float()
        y = y * (z * torch.sigmoid(z))
    if parts[-1] is not None:
        y = torch.where(parts[-1], y, 0.0)
    return y.to(s["u"].dtype), h[-1].clone()


def _selective_scan_train(s):
    t = s["u"].dtype
    parts = _scan_parts(s)
    u, raw, step, b, c, decay, inside = parts
    h, plain = _scan_forward(s, parts)
    dy, out, y = s["dy"].float(), {}, plain
    if inside is not None:
        dy = torch.where(inside, dy, 0.0)
    if s["z"] is not None:
        z = s["z"].float()
        y = plain * (z * torch.sigmoid(z))
        dz = dy * plain * _silu_slope(z)
        out["dz"] = (torch.where(inside, dz, 0.0) if inside is not None else dz).to(t)
        dy = dy * (z * torch.sigmoid(z))
        if inside is not None:
            dy = torch.where(inside, dy, 0.0)
    if inside is not None:
        y = torch.where(inside, y, 0.0)
    out["y"], out["h_final"] = y.to(t), h[-1].clone()
    dc = torch.sum(dy[..., None] * h, dim=2)
    # g[t] = dy[t] c[t] + a[t+1] g[t+1], run backwards; the partial of the final state enters as the last step's
    g = dy[..., None] * c[:, :, None, :]
    g[-1] += s["dh_final"]
    after = torch.cat([decay[1:], torch.ones_like(decay[:1])])
    g = torch.flip(_scan(torch.flip(after, [0]), torch.flip(g, [0])), [0])
    del after
    out["dh0"] = decay[0] * g[0]
    out["dd"] = torch.sum(dy * u, dim=(0, 1))
    db = torch.sum(g * (step * u)[..., None], dim=2)
    along = torch.sum(g * b[:, :, None, :], dim=3)
    out["du"] = (dy * s["d"] + along * step).to(t)
    decay *= torch.cat([s["h0"][None], h[:-1]])                # what is left of the state before
    decay *= g
    out["da"] = torch.sum(decay * step[..., None], dim=(0, 1))
    dstep = torch.sum(decay * s["a"], dim=3) + along * u
    if s["softplus"]:
        dstep = dstep * torch.sigmoid(raw)
    if inside is not None:
        dstep = torch.where(inside, dstep, 0.0)
    out["ddelta"] = dstep.to(t)
    if s["delta_bias"] is not None:
        out["ddelta_bias"] = torch.sum(dstep, dim=(0, 1))
    if s["c"] is None:
        out["db"] = torch.cat([db, dc], dim=2).to(t)
    else:
        out["db"], out["dc"] = db.to(t), dc.to(t)
    return out


def _columns(s):
    step = max(1, min(s["V"], PIECE // s["N"]))
    return [slice(i, min(i + step, s["V"])) for i in range(0, s["V"], step)]


def _scores(s, x, r):
    """A piece of the scores in fp32, and the piece of the head (K,v) that made it."""
    w = (s["w"][r].float().T if s["tied"] else s["w"][:, r].float())
    return (x @ w) / s["temperature"], w


def _head(s):
    x, N = s["x"].float(), s["N"]
    top = torch.full((N,), -math.inf, device=DEV)
    total, at = torch.zeros(N, device=DEV), torch.zeros(N, device=DEV)
    token = s["tokens"].long()
    for r in _columns(s):
        z, _ = _scores(s, x, r)
        new = torch.maximum(top, torch.amax(z, dim=1))
        total = total * torch.exp(top - new) + torch.sum(torch.exp(z - new[:, None]), dim=1)
        top = new
        here = (token >= r.start) & (token < r.stop)
        at = torch.where(here, torch.gather(z, 1, torch.clamp(token - r.start, 0, z.shape[1] - 1)[:, None])[:, 0], at)
    lse = top + torch.log(total)
    valid = (token >= 0) & (token < s["V"])
    return dict(logp=torch.where(valid, at - lse, 0.0), lse=lse)


def _head_train(s):
    out = _head(s)
    x, t = s["x"].float(), s["x"].dtype
    token = s["tokens"].long()
    scale = torch.where((token >= 0) & (token < s["V"]), s["dlogp"], 0.0) / s["temperature"]
    dx, dw = torch.zeros_like(x), torch.empty_like(s["w"])
    for r in _columns(s):
        z, w = _scores(s, x, r)
        dz = -scale[:, None] * torch.exp(z - out["lse"][:, None])
        here = (token >= r.start) & (token < r.stop)
        dz.scatter_add_(1, torch.clamp(token - r.start, 0, z.shape[1] - 1)[:, None], torch.where(here, scale, 0.0)[:, None])
        dx += dz @ w.T
        if s["tied"]:
            dw[r] = (dz.T @ x).to(t)
        else:
            dw[:, r] = (x.T @ dz).to(t)
    return dict(out, dx=dx.to(t), dw=dw)


# ---- the library's calls ------------------------------------------------------------------------------
def _workspace(s, nbytes):
    """Scratch that a program keeps from call to call."""
    if "ws" not in s:
        s["ws"] = torch.empty(max(16, nbytes), dtype=torch.uint8, device=DEV)
    return s["ws"]


def _run_own(s):
    from paper_1810_00952_b200 import binding as B
    kind = s["kind"]
    if kind.startswith("conv"):
        act = B.ACT_SILU if s["silu"] else B.ACT_NONE
        if kind == "conv":
            B.relay_causal_conv(s["x"], s["w"], s["b"], s["before"], s["lengths"], act, s["y"], s["after"])
            return s["y"], s["after"]
        ws = s.get("ws")
        if ws is None:
            ws = _workspace(s, B.relay_workspace_bytes_causal_conv_grad(s["x"], s["w"]))
        B.relay_causal_conv_grad(s["x"], s["w"], s["b"], s["before"], s["lengths"], act, s["dy"], None, s["dx"], s["dw"], s["db"],
                                 s["dbefore"], ws)
        return s["dx"], s["dw"], s["db"], s["dbefore"]
    if kind.startswith("scan"):
        inputs = [s[k] for k in ("u", "delta", "a", "b", "c", "d", "z", "delta_bias")]
        if kind == "scan":
            B.relay_selective_scan(*inputs, s["h0"], s["lengths"], s["softplus"], s["y"], s["h_final"], None)
            return s["y"], s["h_final"]
        if "states" not in s:
            spans = -(-s["T"] // B.SCAN_SPAN)
            s["states"] = torch.empty(spans, s["B"], s["D"], s["N"], device=DEV)
            _workspace(s, B.relay_workspace_bytes_selective_scan_grad(s["u"], s["a"]))
        B.relay_selective_scan(*inputs, s["h0"], s["lengths"], s["softplus"], s["y"], s["h_final"], s["states"])
        B.relay_selective_scan_grad(*inputs, s["lengths"], s["softplus"], s["states"], s["dy"], s["dh_final"],
                                    *[s["d" + k] for k in ("u", "delta", "a", "b", "c", "d", "z", "delta_bias", "h0")], s["ws"])
        names = ("dz", "y", "h_final", "dh0", "dd", "du", "da", "ddelta", "ddelta_bias", "db", "dc")
        return {k: s[k] for k in names if s[k] is not None}
    ws = s.get("ws")
    if ws is None:
        need = B.relay_workspace_bytes_linear_logprob(s["x"], s["w"], s["tied"])
        if kind == "head_train":
            need = max(need, B.relay_workspace_bytes_linear_logprob_grad(s["x"], s["w"], s["tied"]))
        ws = _workspace(s, need)
    B.relay_linear_logprob(s["x"], s["w"], s["tied"], s["tokens"], s["temperature"], s["logp"], s["lse"], ws)
    out = dict(logp=s["logp"], lse=s["lse"])
    if kind == "head":
        return out
    B.relay_linear_logprob_grad(s["x"], s["w"], s["tied"], s["tokens"], s["temperature"], s["lse"], s["dlogp"], s["dx"], s["dw"], ws)
    return dict(out, dx=s["dx"], dw=s["dw"])


def run(state):
    if own:
        return _run_own(state)
    return {"conv": _conv, "conv_train": _conv_grad, "scan": _selective_scan, "scan_train": _selective_scan_train, "head": _head,
            "head_train": _head_train}[state["kind"]](state)


# ---- what a pass cannot do without --------------------------------------------------------------------
def work(case):
    kind, e = case["kind"], 2 if case["dtype"] == "bf16" else 4
    if kind.startswith("head"):
        n, k, v = case["N"], case["K"], case["V"]
        if kind == "head":
            return {"bytes": (n + v) * k * e + 12 * n, "flops": 2 * n * k * v}
        return {"bytes": 2 * (n + v) * k * e + 16 * n, "flops": 6 * n * k * v}          # scores, dx and dw: one product each
    n, rows, D = case["T"] * case["B"] * case["D"], case["T"] * case["B"], case["D"]
    if kind.startswith("conv"):
        state = (case["K"] - 1) * case["B"] * D * e
        if kind == "conv":
            return {"bytes": 2 * n * e + 2 * state, "flops": 2 * case["K"] * n}
        return {"bytes": 3 * n * e + 2 * state, "flops": 6 * case["K"] * n}
    N, z = case["N"], 1 if case["gated"] else 0
    if kind == "scan":                                  # u, delta, z, y; b and c; the state before and after
        return {"bytes": (3 + z) * n * e + 2 * rows * N * e + 8 * case["B"] * D * N, "flops": 7 * n * N}
    # and again with dy, the partials of u, delta, z, b, c and of both states
    return {"bytes": (6 + 2 * z) * n * e + 4 * rows * N * e + 16 * case["B"] * D * N, "flops": 25 * n * N}


# ---- the definitions in 64 bits -----------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"conv": _exact_conv, "conv_train": _exact_conv_grad, "scan": _exact_scan, "scan_train": _exact_scan_train, "head": _exact_head,
            "head_train": _exact_head}[case["kind"]](s)


def _ends(s):
    if s["lengths"] is None:
        return torch.full((s["B"],), s["T"], device=DEV)
    return s["lengths"].long()


def _exact_line(s):
    """x[t] for t from -(K-1) on, at index t + K - 1, and the sums before the activation."""
    T, K = s["T"], s["K"]
    line = torch.cat([s["before"], s["x"]]).double()
    w = s["w"].double()
    total = sum(w[K - 1 - j] * line[K - 1 - j:K - 1 - j + T] for j in range(K))          # j steps back
    if s["b"] is not None:
        total = total + s["b"].double()
    return line, total


def _exact_conv(s):
    line, total = _exact_line(s)
    y = total / (1 + torch.exp(-total)) if s["silu"] else total
    after = torch.empty_like(s["before"], dtype=torch.float64)
    for i, end in enumerate(_ends(s).tolist()):
        y[end:, i] = 0
        after[:, i] = line[end:end + s["K"] - 1, i]
    return y, after


def _exact_conv_grad(s):
    T, K = s["T"], s["K"]
    line, total = _exact_line(s)
    g = s["dy"].double()
    if s["silu"]:
        e = torch.exp(-total)
        g = g * (1 / (1 + e) + total * e / (1 + e) ** 2)
    dline, w = torch.zeros_like(line), s["w"].double()
    dw = torch.zeros(K, s["D"], dtype=torch.float64, device=DEV)
    db = torch.zeros(s["D"], dtype=torch.float64, device=DEV)
    for i, end in enumerate(_ends(s).tolist()):
        for k in range(K):
            dline[k:k + end, i] += w[k] * g[:end, i]
            dw[k] += (g[:end, i] * line[k:k + end, i]).sum(0)
        db += g[:end, i].sum(0)
    return dline[K - 1:], dw, None if s["b"] is None else db, dline[:K - 1]


def _exact_inputs(s):
    N = s["N"]
    b, c = (s["b"][..., :N], s["b"][..., N:]) if s["packed"] else (s["b"], s["c"])
    raw = s["delta"].double()
    if s["delta_bias"] is not None:
        raw = raw + s["delta_bias"].double()
    step = torch.logaddexp(raw, torch.zeros_like(raw)) if s["softplus"] else raw
    return s["u"].double(), raw, step, s["a"].double(), b.double(), c.double(), s["d"].double()


def _exact_states(s, u, step, a, b):
    """The state after each step, (T,B,D,N) in 64 bits."""
    h, ends = s["h0"].double(), _ends(s)[:, None, None]
    states = torch.empty(s["T"], *h.shape, dtype=torch.float64, device=DEV)
    for t in range(s["T"]):
        new = torch.exp(step[t][:, :, None] * a) * h + (step[t] * u[t])[:, :, None] * b[t][:, None, :]
        h = torch.where(t < ends, new, h)
        states[t] = h
    return states


def _gate(z):
    """silu and its slope."""
    e = torch.exp(-z)
    return z / (1 + e), 1 / (1 + e) + z * e / (1 + e) ** 2


def _exact_scan(s):
    u, raw, step, a, b, c, d = _exact_inputs(s)
    h, ends = s["h0"].double(), _ends(s)[:, None, None]
    y = torch.zeros_like(u)
    for t in range(s["T"]):
        new = torch.exp(step[t][:, :, None] * a) * h + (step[t] * u[t])[:, :, None] * b[t][:, None, :]
        h = torch.where(t < ends, new, h)
        y[t] = torch.einsum("bdn,bn->bd", h, c[t]) + d * u[t]
    if s["z"] is not None:
        y = y * _gate(s["z"].double())[0]
    for i, end in enumerate(_ends(s).tolist()):
        y[end:, i] = 0
    return y, h


def _exact_scan_train(s):
    u, raw, step, a, b, c, d = _exact_inputs(s)
    states, ends = _exact_states(s, u, step, a, b), _ends(s)[:, None]
    y, out = torch.einsum("tbdn,tbn->tbd", states, c) + d * u, {}
    on = torch.arange(s["T"], device=DEV)[:, None, None] < ends[None]
    zero = torch.zeros((), dtype=torch.float64, device=DEV)
    dy = torch.where(on, s["dy"].double(), zero)
    out["h_final"] = states[-1].clone()
    if s["z"] is not None:
        gate, slope = _gate(s["z"].double())
        out["dz"] = torch.where(on, dy * y * slope, zero)
        y, dy = y * gate, dy * gate
    out["y"] = torch.where(on, y, zero)
    carry = s["dh_final"].double()
    du, dstep = torch.zeros_like(u), torch.zeros_like(u)
    db, dc = torch.zeros_like(b), torch.zeros_like(c)
    da = torch.zeros_like(a)
    for t in reversed(range(s["T"])):
        live = (t < ends)[:, :, None]
        before = states[t - 1] if t else s["h0"].double()
        g = carry + dy[t][:, :, None] * c[t][:, None, :]
        decay = torch.exp(step[t][:, :, None] * a)
        dc[t] = torch.where(live[:, :, 0], torch.einsum("bdn,bd->bn", states[t], dy[t]), zero)
        db[t] = torch.where(live[:, :, 0], torch.einsum("bdn,bd->bn", g, step[t] * u[t]), zero)
        along = torch.einsum("bdn,bn->bd", g, b[t])
        kept = torch.where(live, g * decay * before, zero)
        da += torch.einsum("bdn,bd->dn", kept, step[t])
        dstep[t] = torch.where(live[:, :, 0], torch.einsum("bdn,dn->bd", kept, a) + along * u[t], zero)
        du[t] = torch.where(live[:, :, 0], dy[t] * d + along * step[t], zero)
        carry = torch.where(live, g * decay, carry)
    if s["softplus"]:
        dstep = dstep / (1 + torch.exp(-raw))
    out.update(dh0=carry, dd=(dy * u).sum((0, 1)), du=du, da=da, ddelta=dstep)
    if s["delta_bias"] is not None:
        out["ddelta_bias"] = dstep.sum((0, 1))
    if s["packed"]:
        out["db"] = torch.cat([db, dc], dim=2)
    else:
        out["db"], out["dc"] = db, dc
    return out


def _exact_head(s):
    w = s["w"].double() if not s["tied"] else s["w"].T.double()
    dw = torch.zeros_like(w) if s["kind"] == "head_train" else None
    step, parts = max(1, (1 << 28) // s["V"]), []
    for i in range(0, s["N"], step):
        r = slice(i, min(i + step, s["N"]))
        x, token = s["x"][r].double(), s["tokens"][r].long()
        z = (x @ w) / s["temperature"]
        lse = torch.logsumexp(z, dim=1)
        valid = (token >= 0) & (token < s["V"])
        rows, at = torch.arange(len(x), device=DEV), token.clamp(0, s["V"] - 1)
        part = dict(logp=torch.where(valid, z[rows, at] - lse, 0.0), lse=lse)
        if dw is not None:
            slope = torch.where(valid, s["dlogp"][r].double(), 0.0) / s["temperature"]
            z -= lse[:, None]
            dz = torch.exp(z, out=z).mul_(-slope[:, None])
            dz[rows, at] += slope
            part["dx"] = dz @ w.T
            dw += x.T @ dz
        parts.append(part)
    out = {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
    if dw is not None:
        out["dw"] = dw.T if s["tied"] else dw
    return out
