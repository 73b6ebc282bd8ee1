"""Measured cases of the operators that a recurrent language model adds to this library: the gated linear recurrence over a
sequence with its gradient, the log-probabilities of given tokens with entropy and top alternatives and their gradient, and the
orthogonalisation of an update by Newton-Schulz products.

A case is a dict of plain values.  `prepare` makes what a program holds before the call, `run` makes one call: the plain form
(elementary torch operations in 32 bits, rounded once) or, where `own` is true, the library's entry point.  `exact` gives the
same results from the definitions in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda:0"
NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315)     # the usual quintic: steep at zero, then near one
STEPS = 5
EPS = 1e-7

# the work of a drawn case stays within that of the largest listed case of its kind
MOST = {"recurrence": 16384 * 4096, "recurrence_grad": 4096 * 8 * 1024, "logprob": 4096 * 32768, "logprob_grad": 4096 * 32768}
MOST_PRODUCTS = 4 * 4096 ** 3


def listed():
    return [
        # one token of 64 running sequences at the width of the library's LSTM workload: what a server does per token
        dict(name="recurrence step", kind="recurrence", T=1, B=64, D=1024, dtype="bf16", gate="mix", packed=True, ragged=False),
        # the LSTM workload's own sequence shape, gates and values as the two column blocks of one dense result
        dict(name="recurrence batch", kind="recurrence", T=128, B=64, D=1024, dtype="bf16", gate="mix", packed=True, ragged=False),
        # one long document read at once: few channels, many steps
        dict(name="recurrence long", kind="recurrence", T=16384, B=1, D=4096, dtype="bf16", gate="sigmoid", packed=False, ragged=False),
        # the gradient of a training batch of long sequences
        dict(name="recurrence grad", kind="recurrence_grad", T=4096, B=8, D=1024, dtype="bf16", gate="mix", packed=True, ragged=False),
        # the gradient of a padded batch of odd sizes, in fp32, with coefficients that the model made itself
        dict(name="recurrence grad ragged", kind="recurrence_grad", T=1001, B=13, D=333, dtype="f32", gate="given", packed=False, ragged=True),
        # the next token of a few sequences, with the alternatives a server returns
        dict(name="logprob decode", kind="logprob", N=8, V=131072, dtype="bf16", top=20, temperature=0.8, masked=True),
        # scoring a batch of given tokens
        dict(name="logprob score", kind="logprob", N=4096, V=32768, dtype="bf16", top=8, temperature=1.0, masked=False),
        # the gradient of that batch, with an entropy term
        dict(name="logprob grad", kind="logprob_grad", N=4096, V=32768, dtype="bf16", temperature=1.0, masked=False, entropy=True),
        # fp32 scores of an odd vocabulary with forbidden words and padded positions
        dict(name="logprob grad masked", kind="logprob_grad", N=509, V=50021, dtype="f32", temperature=0.7, masked=True, entropy=True),
        # the update of one square layer of the library's MLP workload
        dict(name="orthogonalize square", kind="orthogonalize", L=1, M=4096, N=4096, dtype="bf16"),
        # the wide layers of a stack, all at once
        dict(name="orthogonalize layers", kind="orthogonalize", L=8, M=1024, N=4096, dtype="f32"),
        # a few small tall matrices of odd sizes, where latency counts
        dict(name="orthogonalize odd", kind="orthogonalize", L=3, M=500, N=333, dtype="f32"),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi) + 0.49)))))))


def draw(rng):
    kind = rng.choice(["recurrence", "recurrence_grad", "logprob", "logprob_grad", "orthogonalize"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind.startswith("recurrence"):
        most = MOST[kind]
        T = 1 if kind == "recurrence" and rng.random() < 0.2 else _log(rng, 1, 16384)
        D = _log(rng, 16, min(4096, most // T))
        if rng.random() < 0.6:
            D = max(8, D // 8 * 8)
        B = _log(rng, 1, max(1, min(256, most // (T * D))))
        return dict(kind=kind, T=T, B=B, D=D, dtype=dtype, gate=rng.choice(["mix", "sigmoid", "given"]), packed=rng.random() < 0.5,
                    ragged=rng.random() < 0.3)
    if kind.startswith("logprob"):
        V = _log(rng, 4000, 262144)
        if rng.random() < 0.5:
            V = V // 64 * 64
        N = _log(rng, 1, max(1, min(8192, MOST[kind] // V)))
        case = dict(kind=kind, N=N, V=V, dtype=dtype, temperature=rng.choice([1.0, 1.0, 0.7, 1.3]), masked=rng.random() < 0.3)
        if kind == "logprob":
            return dict(case, top=rng.choice([0, 1, 5, 20]))
        return dict(case, entropy=rng.random() < 0.5)
    while True:
        L, M, N = _log(rng, 1, 16), _log(rng, 32, 4096), _log(rng, 32, 4096)
        if L * min(M, N) ** 2 * (min(M, N) + 3 * max(M, N)) <= MOST_PRODUCTS:
            return dict(kind=kind, L=L, M=M, N=N, dtype=dtype)


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
    if kind.startswith("recurrence"):
        T, B, D = case["T"], case["B"], case["D"]
        if case["gate"] == "given":
            f = 1.0 - torch.exp(-5.0 * rand(D) - 0.5 - rand(T, B, D))          # decays of one to a few hundred steps
        else:
            f = 4.0 * rand(D) + randn(T, B, D)                                # gates mostly open, each channel its own span
        u = randn(T, B, D)
        s["h0"] = randn(B, D)
        s["lengths"] = None
        if case["ragged"]:
            n = torch.randint(0, T + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
            n[0] = T
            s["lengths"] = n
        if case["packed"]:
            s["f"], s["u"] = torch.cat([f, u], dim=2).to(t), None
        else:
            s["f"], s["u"] = f.to(t), u.to(t)
        if kind == "recurrence":
            s["h_all"] = torch.empty(T, B, D, dtype=t, device=DEV)
            s["h_final"] = torch.empty(B, D, device=DEV)
        else:
            s["h_all"] = _recurrence(s)[0]                                     # what the forward call left behind
            s["dh_all"], s["dh_final"] = randn(T, B, D).to(t), randn(B, D)
            s["df"] = torch.empty_like(s["f"])
            s["du"] = None if case["packed"] else torch.empty_like(s["u"])
            s["dh0"] = torch.empty(B, D, device=DEV)
        return s
    if kind.startswith("logprob"):
        N, V = case["N"], case["V"]
        z = 2.5 * randn(N, V)
        if case["masked"]:
            z.masked_fill_(rand(1, V) < 0.1, -math.inf)                        # forbidden words
            if N > 2:
                z[N // 2] = -math.inf                                          # a row whose mask leaves nothing
        s["scores"] = z.to(t)
        guess = torch.argmax(z, dim=1)
        other = torch.randint(0, V, (N,), generator=g, device=DEV)
        tokens = torch.where(rand(N) < 0.4, guess, other).to(torch.int32)
        if case["masked"]:
            tokens.masked_fill_(rand(N) < 0.2, -1)                             # padded positions
        s["tokens"] = tokens
        del z

        def vector():
            return torch.empty(N, device=DEV)

        if kind == "logprob":
            s["logp"], s["entropy"], s["lse"] = vector(), vector(), vector()
            k = case["top"]
            s["top_logp"] = torch.empty(N, k, device=DEV) if k else None
            s["top_ids"] = torch.empty(N, k, dtype=torch.int32, device=DEV) if k else None
        else:
            r = _logprob(dict(s, top=0))
            s["lse"], s["h"] = r["lse"], r["entropy"] if case["entropy"] else None
            s["dlogp"], s["dentropy"] = randn(N) / N, 0.01 * randn(N) / N if case["entropy"] else None
            s["dscores"] = torch.empty(N, V, dtype=t, device=DEV)
        return s
    # gradients of weights: every row and column at a scale of its own, and a few directions that many samples share
    L, M, N = case["L"], case["M"], case["N"]
    x = randn(L, M, N) * torch.exp(0.5 * randn(L, M, 1)) * torch.exp(0.5 * randn(L, 1, N))
    x += torch.bmm(randn(L, M, 8), randn(L, 8, N)) / math.sqrt(8.0)
    s["x"] = (1e-3 * x).to(t)
    s["y"] = torch.empty(L, M, N, dtype=torch.bfloat16, device=DEV)
    return s


# ---- the plain forms ----------------------------------------------------------------------------------
def _split(s):
    """Gates and values in fp32, and the steps that are inside their sequences (None: all)."""
    f, u = (s["f"], s["u"]) if s["u"] is not None else torch.chunk(s["f"], 2, dim=2)
    inside = None
    if s["lengths"] is not None:
        steps = torch.arange(s["T"], device=DEV, dtype=torch.int32)
        inside = (steps[:, None] < s["lengths"][None, :])[:, :, None]
    return f.float(), u.float(), inside


def _scan(a, b):
    """h[t] = a[t] h[t-1] + b[t] with h[-1] = 0, by doubling the span that each step has summed up; overwrites a and b."""
    k = 1
    while k < a.shape[0]:
        b[k:] += a[k:] * b[:-k]
        a[k:] = a[k:] * a[:-k]
        k *= 2
    return b


def _recurrence(s):
    f, u, inside = _split(s)
    if s["gate"] == "given":
        a, b = f.clone(), u.clone()
    else:
        a = torch.sigmoid(f)
        b = torch.sigmoid(-f) * u if s["gate"] == "mix" else u.clone()
    if inside is not None:
        a, b = torch.where(inside, a, 1.0), torch.where(inside, b, 0.0)
    b[0] += a[0] * s["h0"]
    h = _scan(a, b)
    h_final = h[-1].clone()
    if inside is not None:
        h = torch.where(inside, h, 0.0)
    return h.to(s["f"].dtype), h_final


def _recurrence_grad(s):
    f, u, inside = _split(s)
    a = f if s["gate"] == "given" else torch.sigmoid(f)
    h_before = torch.cat([s["h0"][None], s["h_all"][:-1].float()])
    dh = s["dh_all"].float()
    if inside is not None:
        a, dh = torch.where(inside, a, 1.0), torch.where(inside, dh, 0.0)
    # g[t] = dh[t] + a[t+1] g[t+1], run backwards; the partial of the final state enters as the last step's
    dh = dh.clone()
    dh[-1] += s["dh_final"]
    after = torch.cat([a[1:], torch.ones_like(a[:1])])
    g = torch.flip(_scan(torch.flip(after, [0]), torch.flip(dh, [0])), [0])
    dh0 = a[0] * g[0]
    if s["gate"] == "given":
        df, du = g * h_before, g
    elif s["gate"] == "sigmoid":
        df, du = g * h_before * a * torch.sigmoid(-f), g
    else:
        one_less = torch.sigmoid(-f)
        df, du = g * (h_before - u) * a * one_less, g * one_less
    if inside is not None:
        df, du = torch.where(inside, df, 0.0), torch.where(inside, du, 0.0)
    t = s["f"].dtype
    if s["u"] is None:
        return torch.cat([df, du], dim=2).to(t), None, dh0
    return df.to(t), du.to(t), dh0


def _logprob(s):
    z = s["scores"].float() / s["temperature"]
    m = torch.amax(z, dim=1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    lse = m + torch.log(torch.sum(torch.exp(z - m), dim=1, keepdim=True))
    nothing = lse == -math.inf                                                # the mask leaves nothing
    lp = torch.where(nothing, -math.inf, z - lse)
    p = torch.exp(lp)
    entropy = -torch.sum(torch.where(p > 0, p * lp, 0.0), dim=1)
    token = s["tokens"].long()
    valid = (token >= 0) & (token < s["V"])
    logp = torch.gather(lp, 1, torch.clamp(token, 0, s["V"] - 1)[:, None])[:, 0]
    out = dict(logp=torch.where(valid, logp, 0.0), entropy=entropy, lse=lse[:, 0])
    if s["top"]:
        # largest first, equal scores by the lower index: the order of (score, -index) as one whole number
        bits = (s["scores"].float() + 0.0).view(torch.int32).long()
        order = torch.where(bits >= 0, bits, bits ^ 0x7FFFFFFF)
        key = order * 2 ** 32 + (2 ** 32 - 1 - torch.arange(s["V"], device=DEV))
        best = torch.topk(key, s["top"], dim=1).values
        ids = 2 ** 32 - 1 - (best & 0xFFFFFFFF)
        out["top_ids"], out["top_logp"] = ids.int(), torch.gather(lp, 1, ids)
    return out


def _logprob_grad(s):
    z = s["scores"].float() / s["temperature"]
    lse = s["lse"][:, None]
    lp = z - lse
    p = torch.exp(lp)
    token = s["tokens"].long()
    valid = (token >= 0) & (token < s["V"])
    dlogp = torch.where(valid, s["dlogp"], 0.0)[:, None]
    d = -dlogp * p
    if s["dentropy"] is not None:
        d -= s["dentropy"][:, None] * torch.where(p > 0, p * (lp + s["h"][:, None]), 0.0)
    d.scatter_add_(1, torch.clamp(token, 0, s["V"] - 1)[:, None], dlogp)
    d = torch.where(lse == -math.inf, 0.0, d / s["temperature"])
    return d.to(s["scores"].dtype)


def _orthogonalize(s):
    a, b, c = NEWTON_SCHULZ
    x = s["x"].float()
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2)
    x = x / (torch.sqrt(torch.sum(x * x, dim=(1, 2), keepdim=True)) + EPS)
    for _ in range(STEPS):
        gram = torch.bmm(x, x.transpose(1, 2))
        x = a * x + torch.bmm(b * gram + c * torch.bmm(gram, gram), x)
    return (x.transpose(1, 2) if tall else x).to(torch.bfloat16).contiguous()


# ---- the library's calls ------------------------------------------------------------------------------
def _workspace(s, nbytes):
    """Scratch that a program keeps from call to call."""
    if "ws" not in s:
        s["ws"] = torch.empty(max(16, nbytes), dtype=torch.uint8, device=DEV)
    return s["ws"]


def _run_own(s):
    from paper_1810_00952_b200 import binding as B
    kind = s["kind"]
    if kind.startswith("recurrence"):
        gate = {"given": B.GATE_GIVEN, "sigmoid": B.GATE_SIGMOID, "mix": B.GATE_MIX}[s["gate"]]
        if kind == "recurrence":
            B.relay_gated_recurrence(s["f"], s["u"], s["h0"], s["lengths"], gate, s["h_all"], s["h_final"])
            return s["h_all"], s["h_final"]
        B.relay_gated_recurrence_grad(s["f"], s["u"], s["h0"], s["lengths"], gate, s["h_all"], s["dh_all"], s["dh_final"],
                                      s["df"], s["du"], s["dh0"])
        return s["df"], s["du"], s["dh0"]
    if kind == "logprob":
        B.relay_token_logprob(s["scores"], s["tokens"], s["temperature"], s["logp"], s["entropy"], s["lse"], s["top_logp"], s["top_ids"])
        return {k: s[k] for k in (("logp", "entropy", "lse", "top_logp", "top_ids") if s["top"] else ("logp", "entropy", "lse"))}
    if kind == "logprob_grad":
        B.relay_token_logprob_grad(s["scores"], s["tokens"], s["temperature"], s["lse"], s["h"], s["dlogp"], s["dentropy"], s["dscores"])
        return s["dscores"]
    ws = s.get("ws")
    if ws is None:
        ws = _workspace(s, B.relay_workspace_bytes_orthogonalize(s["x"]))
    B.relay_orthogonalize(s["x"], STEPS, NEWTON_SCHULZ, EPS, 1.0, s["y"], ws)
    return s["y"]


def run(state):
    if own:
        return _run_own(state)
    return {"recurrence": _recurrence, "recurrence_grad": _recurrence_grad, "logprob": _logprob, "logprob_grad": _logprob_grad,
            "orthogonalize": _orthogonalize}[state["kind"]](state)


# ---- what a pass cannot do without --------------------------------------------------------------------
def work(case):
    kind, e = case["kind"], 2 if case["dtype"] == "bf16" else 4
    if kind.startswith("recurrence"):
        n, c = case["T"] * case["B"] * case["D"], case["B"] * case["D"]
        if kind == "recurrence":                    # gates, values and states once; h0 and the final state
            return {"bytes": 3 * n * e + 8 * c, "flops": 8 * n}
        return {"bytes": 6 * n * e + 12 * c, "flops": 16 * n}
    if kind == "logprob":
        n = case["N"] * case["V"]
        return {"bytes": n * e + case["N"] * (16 + 8 * case["top"]), "flops": 6 * n}
    if kind == "logprob_grad":
        n = case["N"] * case["V"]
        return {"bytes": 2 * n * e + case["N"] * 20, "flops": 8 * n}
    m, n = min(case["M"], case["N"]), max(case["M"], case["N"])
    # per step: the Gram matrix and its square are symmetric (one triangle each), the product with x is full
    return {"bytes": case["L"] * m * n * (e + 2), "flops": case["L"] * STEPS * (m * m * n + m * m * m + 2 * m * m * n)}


# ---- the definitions in 64 bits -----------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind.startswith("recurrence"):
        return _exact_recurrence(s) if kind == "recurrence" else _exact_recurrence_grad(s)
    if kind == "logprob":
        return _exact_logprob(s)
    if kind == "logprob_grad":
        return _exact_logprob_grad(s)
    a, b, c = NEWTON_SCHULZ
    out = []
    for x in s["x"].double():                       # q(X X^T) X with q(A) = a I + b A + c A A, whichever side is the shorter
        x = x / (torch.linalg.norm(x) + EPS)
        eye = torch.eye(min(x.shape), dtype=torch.float64, device=DEV)
        for _ in range(STEPS):
            if x.shape[0] <= x.shape[1]:
                w = x @ x.T
                x = (a * eye + b * w + c * w @ w) @ x
            else:
                w = x.T @ x
                x = x @ (a * eye + b * w + c * w @ w)
        out.append(x)
    return torch.stack(out)


def _coefficients64(s):
    D = s["D"]
    f, u = (s["f"][..., :D].double(), s["f"][..., D:].double()) if s["packed"] else (s["f"].double(), s["u"].double())
    if s["gate"] == "given":
        return f, torch.ones_like(f), u
    e = torch.exp(-f)
    return 1 / (1 + e), (e / (1 + e) if s["gate"] == "mix" else torch.ones_like(f)), u


def _ends(s):
    if s["lengths"] is None:
        return torch.full((s["B"],), s["T"], device=DEV)
    return s["lengths"].long()


def _exact_recurrence(s):
    a, i, u = _coefficients64(s)
    h, ends = s["h0"].double(), _ends(s)[:, None]
    h_all = torch.zeros_like(a)
    for t in range(s["T"]):
        on = t < ends
        h = torch.where(on, a[t] * h + i[t] * u[t], h)
        h_all[t] = torch.where(on, h, 0.0)
    return h_all, h


def _exact_recurrence_grad(s):
    a, i, u = _coefficients64(s)
    g, ends = s["dh_final"].double(), _ends(s)[:, None]
    df, du = torch.zeros_like(a), torch.zeros_like(a)
    for t in reversed(range(s["T"])):
        on = t < ends
        before = (s["h_all"][t - 1] if t else s["h0"]).double()
        here = g + s["dh_all"][t].double()
        if s["gate"] == "given":
            da = here * before
        elif s["gate"] == "sigmoid":
            da = here * before * a[t] * (1 - a[t])
        else:
            da = here * (before - u[t]) * a[t] * i[t]
        df[t], du[t] = torch.where(on, da, 0.0), torch.where(on, here * i[t], 0.0)
        g = torch.where(on, a[t] * here, g)
    if s["packed"]:
        return torch.cat([df, du], dim=2), None, g
    return df, du, g


def _rows(s):
    """Slices of a few rows, so that 64-bit copies stay small."""
    step = max(1, (1 << 25) // s["V"])
    return [slice(i, min(i + step, s["N"])) for i in range(0, s["N"], step)]


def _exact_logprob(s):
    parts = []
    for r in _rows(s):
        z = s["scores"][r].double() / s["temperature"]
        lse = torch.logsumexp(z, dim=1)
        lp = torch.where(lse[:, None] == -math.inf, -math.inf, z - lse[:, None])
        token = s["tokens"][r].long()
        valid = (token >= 0) & (token < s["V"])
        part = dict(logp=torch.where(valid, lp[torch.arange(len(lp), device=DEV), token.clamp(0, s["V"] - 1)], 0.0),
                    entropy=torch.special.entr(torch.exp(lp)).sum(1), lse=lse)
        if s["top"]:
            ids = torch.sort(s["scores"][r].float(), dim=1, descending=True, stable=True).indices[:, :s["top"]]
            part["top_ids"], part["top_logp"] = ids.int(), torch.gather(lp, 1, ids)
        parts.append(part)
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}


def _exact_logprob_grad(s):
    out = []
    for r in _rows(s):
        z = s["scores"][r].double() / s["temperature"]
        lse = torch.logsumexp(z, dim=1, keepdim=True)
        p = torch.where(lse == -math.inf, 0.0, torch.exp(z - lse))
        token = s["tokens"][r].long()
        hot = torch.arange(s["V"], device=DEV)[None, :] == token[:, None]
        d = s["dlogp"][r].double()[:, None] * torch.where((token >= 0)[:, None], hot.double() - p, 0.0)
        if s["dentropy"] is not None:
            entropy = torch.special.entr(p).sum(1, keepdim=True)
            d += s["dentropy"][r].double()[:, None] * (torch.special.entr(p) - p * entropy)
        out.append(torch.where(lse == -math.inf, 0.0, d / s["temperature"]))
    return torch.cat(out)
