"""GPU parity: orthogonalised updates against the fp64 definition, through the C ABI.

Tolerances.  The products' operands carry fp16 rounding (2^-12 of an element at most): three operands a step and five steps, each
error kept or damped by the later steps for matrices without singular values far below the largest; rounding the operands of the
fp64 iteration that way on the CPU gives errors of 1.1e-3 to 1.9e-3 of the result's norm over the shapes here.  With the bf16 rounding
of the result (2^-9 / sqrt(3) of an element, 1.7e-3 of the norm at most) the sum stays below 3e-3; the bound is 4e-3 of the norm, and
2e-2 of the RMS (ten standard deviations) plus half a unit in the last place for every element."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import language as L
from paper_1810_00952_b200 import binding as B

from parity import Guarded, bf16_ulp, rms, to_np

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
QUINTIC = (3.4445, -4.7750, 2.0315)


def matrices(shape, dt, seed, scale=1.0):
    """Rows and columns of scales of their own, and a few shared directions."""
    r = np.random.default_rng(seed)
    M, N = shape[-2:]
    x = r.normal(size=shape) * np.exp(0.4 * r.normal(size=(*shape[:-1], 1))) * np.exp(0.4 * r.normal(size=(*shape[:-2], 1, N)))
    x += r.normal(size=(*shape[:-1], 4)) @ r.normal(size=(*shape[:-2], 4, N)) / 2
    return torch.from_numpy(scale * x).to(dt)


def run(x, steps=5, coef=QUINTIC, eps=1e-7, scale=1.0):
    y = Guarded(tuple(x.shape), BF16, DEV)
    xd = x.to(DEV)
    n = B.relay_workspace_bytes_orthogonalize(xd)
    ws = torch.full((max(n, 16) + 512,), 255, dtype=torch.uint8, device=DEV)     # bytes that read as NaN
    B.relay_orthogonalize(xd, steps, coef, eps, scale, y.t, ws[:n] if n else None)
    torch.cuda.synchronize()
    B.relay_poll_status()
    assert bool((ws[n:] == 255).all()), "write behind the workspace"
    return y.check()


def close(y, want):
    g = to_np(y)
    assert np.all(np.isfinite(g))
    for k in np.ndindex(*want.shape[:-2]):
        d, w = g[k] - want[k], want[k]
        assert rms(d) <= 4e-3 * rms(w) + 1e-30, (k, rms(d) / rms(w))
        assert np.all(np.abs(d) <= 2e-2 * rms(w) + 0.5 * bf16_ulp(w)), (k, np.abs(d).max() / rms(w))


# one tile and its edges, several tiles, wide and tall, rows whose 16-byte pieces do not come out even, long contractions
SHAPES = [(1, 1), (1, 7), (9, 1), (2, 3), (5, 64), (64, 64), (65, 63), (100, 128), (128, 128), (129, 127), (127, 257), (200, 333), (333, 200),
          (130, 1030), (1030, 130), (256, 256), (257, 511), (512, 520), (520, 264), (40, 3001), (3001, 24)]


@pytest.mark.gpu
@pytest.mark.parametrize("M,N", SHAPES)
@pytest.mark.parametrize("dt", [F32, BF16])
def test_shapes(M, N, dt):
    x = matrices((M, N), dt, M * 5 + N)
    close(run(x), L.orthogonalize(to_np(x), 5, QUINTIC, 1e-7, 1.0))


# either side of the sizes at which another kernel takes over: 512 elements, 128 rows, 256 columns for each of 1, 2, 4, 8 blocks
@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(16, 32), (19, 27), (1, 512), (1, 513), (32, 32), (1, 1025), (33, 33), (2, 600), (16, 65), (40, 40), (97, 97), (128, 256), (256, 128), (128, 257), (257, 128),
                                   (31, 513), (128, 1000), (1000, 128), (128, 1024), (1025, 97), (120, 2048), (2048, 120), (3, 2047), (2047, 3), (128, 2049),
                                   (129, 129), (9, 40, 300), (20, 300, 40), (30, 128, 2048)])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_sizes_at_which_the_kernel_changes(shape, dt):
    x = matrices(shape, dt, sum(shape))
    close(run(x), L.orthogonalize(to_np(x), 5, QUINTIC, 1e-7, 1.0))


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(3, 70, 90), (2, 3, 90, 70), (5, 130, 130), (40, 16, 16), (2, 2, 2, 2, 33, 65), (1, 600, 600), (200, 8, 40)])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_batches(shape, dt):
    x = matrices(shape, dt, sum(shape))
    y = run(x)
    close(y, L.orthogonalize(to_np(x), 5, QUINTIC, 1e-7, 1.0))
    last = tuple(n - 1 for n in shape[:-2])
    assert torch.equal(run(x[last].clone()), y[last])                    # a matrix does not depend on its neighbours


@pytest.mark.gpu
@pytest.mark.parametrize("steps", [1, 2, 3, 6])
@pytest.mark.parametrize("coef", [QUINTIC, (1.5, -0.5, 0.0), (2.0, -1.5, 0.5)])
def test_steps_coefficients_and_scale(steps, coef):
    for shape in [(90, 150), (150, 90)]:
        x = matrices(shape, F32, steps)
        c = tuple(float(np.float32(v)) for v in coef)
        close(run(x, steps, coef, 0.0, 0.5), L.orthogonalize(to_np(x), steps, c, 0.0, 0.5))


@pytest.mark.gpu
@pytest.mark.parametrize("coef,steps", [((10, 0, 0), 6), ((10, 0, 0), 16), ((0.1, 0, 0), 6), ((0.1, 0, 0), 16), ((-3, 0, 0), 9), ((1e4, 0, 0), 3), ((1e-4, 0, 0), 3),
                                        ((2, 0.5, 0), 4), ((3, 1, 0), 3), ((4, -1, 0), 3)])
@pytest.mark.parametrize("shape", [(16, 20), (90, 150), (150, 90), (40, 600), (300, 200), (200, 300), (600, 900)])
def test_coefficients_that_let_the_matrix_grow_or_shrink(coef, steps, shape):
    """From 1e-19 to 1e14 of the norm, far outside the 16-bit operands' own range.  Rounding the operands of the fp64 iteration on the
    CPU, kept in range by powers of two, gives errors of 1.4e-4 to 8.6e-4 of the result's norm over these cases: the bounds above hold."""
    x = matrices(shape, F32, steps)
    c = tuple(float(np.float32(v)) for v in coef)
    close(run(x, steps, coef, 0.0, 1.0), L.orthogonalize(to_np(x), steps, c, 0.0, 1.0))


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e12, 1e30])
def test_only_the_direction_counts(scale):
    x = matrices((140, 200), F32, 3)
    want = L.orthogonalize(to_np(x), 5, QUINTIC, 0.0, 1.0)
    close(run((x.double() * scale).float(), eps=0.0), want)


@pytest.mark.gpu
def test_eps_counts_beside_a_small_norm():
    x = matrices((30, 50), F32, 4)
    x = (x / torch.linalg.norm(x) * 1e-3).float()
    want = L.orthogonalize(to_np(x), 1, QUINTIC, float(np.float32(1e-3)), 1.0)
    close(run(x, steps=1, eps=1e-3), want)


@pytest.mark.gpu
def test_zero_matrices_stay_zero_beside_others():
    x = matrices((3, 60, 140), BF16, 5)
    x[1] = 0
    y = run(x)
    assert not bool(y[1].any())
    want = L.orthogonalize(to_np(x), 5, QUINTIC, 1e-7, 1.0)
    close(y[[0, 2]], want[[0, 2]])
    x[2, :, 7:] = 0; x[0, 5:] = 0                                        # rows and columns of zeros: rank-deficient
    y = run(x)
    assert not bool(y[2, :, 7:].any()) and not bool(y[0, 5:].any())
    close(y[[0, 2]], L.orthogonalize(to_np(x), 5, QUINTIC, 1e-7, 1.0)[[0, 2]])


@pytest.mark.gpu
def test_singular_values_come_out_near_one():
    x = matrices((700, 500), F32, 6)
    s = np.linalg.svd(to_np(run(x)), compute_uv=False)
    # the quintic takes [0.003, 1] into [0.68, 1.2] in five steps (a scan of the scalar map); 500 values of a matrix whose smallest is
    # about 1e-3 of its norm start in [0.0004, 0.6]
    assert s.max() < 1.22 and np.median(s) > 0.65


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(1024, 1024), (512, 4096), (4096, 640), (3, 900, 1100)])
def test_large_against_an_fp64_iteration(shape):
    x = matrices(shape, BF16, 7)
    y = run(x)
    m = x.to(DEV).double()
    m = m / (torch.linalg.matrix_norm(m, keepdim=True) + 1e-7)
    for _ in range(5):
        g = m @ m.mT if m.shape[-2] <= m.shape[-1] else m.mT @ m
        q = QUINTIC[1] * g + QUINTIC[2] * g @ g
        m = QUINTIC[0] * m + (q @ m if m.shape[-2] <= m.shape[-1] else m @ q)
    close(y, to_np(m))


@pytest.mark.gpu
def test_same_bits_every_time_and_on_another_stream():
    x = matrices((2, 300, 700), F32, 8)
    y = run(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(3):
            assert torch.equal(run(x), y)


@pytest.mark.gpu
def test_empty_tensors():
    for shape in [(0, 4), (4, 0), (0, 3, 4)]:
        x = torch.zeros(shape, device=DEV)
        assert B.relay_workspace_bytes_orthogonalize(x) == 0
        B.relay_orthogonalize(x, 5, QUINTIC, 1e-7, 1.0, torch.zeros(shape, dtype=BF16, device=DEV), None)


def test_refusals_leave_the_output_untouched(monkeypatch):
    """Everything here is refused on the host, before a launch; the tensors are host memory."""
    monkeypatch.setattr(B, "_stream", lambda: ctypes.c_void_p(None))
    x, y = torch.zeros(80, 96), torch.full((80, 96), 5, dtype=BF16)
    ws = torch.zeros(B.relay_workspace_bytes_orthogonalize(x), dtype=torch.uint8)
    f = lambda x=x, steps=5, coef=QUINTIC, eps=1e-7, scale=1.0, y=y, ws=ws: B.relay_orthogonalize(x, steps, coef, eps, scale, y, ws)
    nan, inf = float("nan"), float("inf")
    cases = [(dict(x=None), "ERR_NULL"), (dict(y=None), "ERR_NULL"),
             (dict(x=torch.zeros(8)), "ERR_RANK"), (dict(y=y.view(1, 80, 96)), "ERR_RANK"),
             (dict(x=x.int()), "ERR_DTYPE"), (dict(y=torch.zeros(80, 96)), "ERR_DTYPE"),
             (dict(y=torch.zeros(96, 80, dtype=BF16)), "ERR_SHAPE"), (dict(x=torch.zeros(1, 65537), y=torch.zeros(1, 65537, dtype=BF16)), "ERR_SHAPE"),
             (dict(steps=0), "ERR_ATTR"), (dict(steps=17), "ERR_ATTR"), (dict(coef=(nan, 0, 0)), "ERR_ATTR"), (dict(scale=inf), "ERR_ATTR"),
             (dict(eps=-1.0), "ERR_ATTR"), (dict(eps=inf), "ERR_ATTR"), (dict(eps=nan), "ERR_ATTR"),
             (dict(x=torch.zeros(80 * 96 + 1)[1:].view(80, 96)), "ERR_ALIGN"), (dict(ws=None), "ERR_WORKSPACE"), (dict(ws=ws[:-1]), "ERR_WORKSPACE"),
             (dict(ws=ws[8:]), "ERR_WORKSPACE")]
    n0 = B.relay_launch_count()
    for i, (kw, status) in enumerate(cases):
        with pytest.raises(B.RelayError) as e:
            f(**kw)
        assert e.value.status_name == status, (i, e.value)
    same = torch.zeros(80, 96, dtype=BF16)
    with pytest.raises(B.RelayError) as e:
        f(x=same, y=same, ws=torch.zeros(1 << 18, dtype=torch.uint8))
    assert e.value.status_name == "ERR_ATTR"
    assert B.relay_launch_count() == n0 and bool((y == 5).all())


@pytest.mark.parametrize("shape", [(200, 333), (333, 200), (2, 3, 200, 333)])
def test_products_refuse_a_workspace_that_is_too_small_or_misaligned(monkeypatch, shape):
    """Sizes whose workspace the kernels write; refused on the host, before a launch (host memory)."""
    monkeypatch.setattr(B, "_stream", lambda: ctypes.c_void_p(None))
    x, y = torch.zeros(shape), torch.full(shape, 5, dtype=BF16)
    n = B.relay_workspace_bytes_orthogonalize(x)
    m, k = min(shape[-2:]), max(shape[-2:])
    batch = int(np.prod(shape[:-2], initial=1))
    assert n >= batch * 2 * (2 * m * k + 2 * m * m)                       # X twice, G and P in 16 bits
    less = B.relay_workspace_bytes_orthogonalize(torch.zeros(*shape[:-2], 190, 333))
    assert less < n
    ws = torch.zeros(n + 64, dtype=torch.uint8)
    ws = ws[(-ws.data_ptr()) % 16:]
    n0 = B.relay_launch_count()
    for bad in (None, ws[:0], ws[:16], ws[:n - 1], ws[:less], ws[8:8 + n], ws[1:1 + n]):
        with pytest.raises(B.RelayError) as e:
            B.relay_orthogonalize(x, 5, QUINTIC, 1e-7, 1.0, y, bad)
        assert e.value.status_name == "ERR_WORKSPACE"
    assert B.relay_launch_count() == n0 and bool((y == 5).all())


# Singular values that fall off, as those of gradients do.  Rounding the operands of the fp64 iteration on the CPU gives, over the
# sizes here, at most these errors over the result's norm; the results' own rounding adds 1.7e-3, and a fifth is left for the order of sums.
DECAY = {"1/i": 0.0033, "1/i^2": 0.0204, "rank 8 and noise of 1 %": 0.0230, "rank 16": 0.0478}


@pytest.mark.gpu
@pytest.mark.parametrize("spectrum", list(DECAY))
@pytest.mark.parametrize("shape", [(96, 160), (128, 1000), (333, 500), (512, 768), (768, 512)])
def test_singular_values_that_fall_off(spectrum, shape):
    x = falling(shape, spectrum)
    w = L.orthogonalize(to_np(x), 5, tuple(float(np.float32(v)) for v in QUINTIC), 1e-7, 1.0)
    g = to_np(run(x))
    assert rms(g - w) <= (1.2 * DECAY[spectrum] + 1.7e-3) * rms(w), rms(g - w) / rms(w)


def falling(shape, spectrum):
    r = np.random.default_rng(shape[0] + shape[1])
    n = min(shape)
    u, v = np.linalg.qr(r.normal(size=(shape[0], n)))[0], np.linalg.qr(r.normal(size=(shape[1], n)))[0]
    i = np.arange(1, n + 1)
    s = {"1/i": 1.0 / i, "1/i^2": 1.0 / i ** 2, "rank 8 and noise of 1 %": np.where(i <= 8, 1.0, 0.0), "rank 16": np.where(i <= 16, 1.0, 0.0)}[spectrum]
    x = (u * s) @ v.T
    if spectrum.startswith("rank 8"):
        x = x + 0.01 * np.linalg.norm(x) / np.sqrt(x.size) * r.normal(size=shape)
    return torch.from_numpy(x).to(F32)
