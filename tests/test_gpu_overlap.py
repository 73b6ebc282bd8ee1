"""Calls that overlap: on two streams, or from two host threads, each with buffers of its own.  Results have the bits of the same call
alone."""
import ctypes
import threading

import pytest
import torch

from paper_1810_00952_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
QUINTIC = (3.4445, -4.7750, 2.0315)


def randn(*shape, dt=BF16, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dt).to(DEV)


class Orthogonalize:
    def __init__(self, shape, seed, dt=BF16):
        self.x, self.y = randn(*shape, dt=dt, seed=seed), torch.empty(shape, dtype=BF16, device=DEV)
        self.ws = torch.empty(max(16, B.relay_workspace_bytes_orthogonalize(self.x)), dtype=torch.uint8, device=DEV)
        self.outs = [self.y]

    def __call__(self):
        B.relay_orthogonalize(self.x, 5, QUINTIC, 1e-7, 1.0, self.y, self.ws)


class Recurrence:
    """The forward call and its gradient group, one after the other."""

    def __init__(self, T, Bn, D, seed, dt=BF16):
        self.f, self.u, self.dh = (randn(T, Bn, D, dt=dt, seed=seed + k) for k in range(3))
        self.h0 = randn(Bn, D, dt=F32, seed=seed + 3)
        self.h, self.df, self.du = (torch.empty_like(self.f) for _ in range(3))
        self.last, self.dh0 = torch.empty_like(self.h0), torch.empty_like(self.h0)
        self.outs = [self.h, self.last, self.df, self.du, self.dh0]

    def __call__(self):
        B.relay_gated_recurrence(self.f, self.u, self.h0, None, B.GATE_MIX, self.h, self.last)
        B.relay_gated_recurrence_grad(self.f, self.u, self.h0, None, B.GATE_MIX, self.h, self.dh, self.h0, self.df, self.du, self.dh0)


class TokenLogprob:
    def __init__(self, N, V, top, seed, dt=BF16):
        self.z = randn(N, V, dt=dt, seed=seed)
        self.tok = torch.arange(N, device=DEV, dtype=torch.int32) % V
        self.d = randn(N, dt=F32, seed=seed + 1)
        self.logp, self.entropy, self.lse = (torch.empty(N, device=DEV) for _ in range(3))
        self.top, self.ids = torch.empty(N, top, device=DEV), torch.empty(N, top, device=DEV, dtype=torch.int32)
        self.dz = torch.empty_like(self.z)
        self.outs = [self.logp, self.entropy, self.lse, self.top, self.ids, self.dz]

    def __call__(self):
        B.relay_token_logprob(self.z, self.tok, 0.8, self.logp, self.entropy, self.lse, self.top, self.ids)
        B.relay_token_logprob_grad(self.z, self.tok, 0.8, self.lse, self.entropy, self.d, self.d, self.dz)


def alone(call):
    call()
    torch.cuda.synchronize()
    B.relay_poll_status()
    return [t.clone() for t in call.outs]


def check_overlap(first, second, rounds=20):
    """The second stream has the higher priority, so that its blocks are placed while the first one's wait for room."""
    want = [alone(first), alone(second)]
    low, high = torch.cuda.Stream(priority=0), torch.cuda.Stream(priority=-1)
    for _ in range(3):
        for t in first.outs + second.outs:
            t.fill_(7)
        for s in (low, high):
            s.wait_stream(torch.cuda.current_stream())
        for _ in range(rounds):
            for s, call in ((low, first), (high, second)):
                with torch.cuda.stream(s):
                    call()
        torch.cuda.synchronize()
        B.relay_poll_status()
        for w, call in zip(want, (first, second)):
            assert all(torch.equal(a, b) for a, b in zip(w, call.outs))


def capture(call):
    g = torch.cuda.CUDAGraph(keep_graph=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        call()
    return g


def kernel_nodes(graph):
    """The kernel nodes of a captured graph that need not have been run, and the driver library."""
    cu = ctypes.CDLL("libcuda.so.1")
    n = ctypes.c_size_t(0)
    g = ctypes.c_void_p(graph.raw_cuda_graph())
    assert cu.cuGraphGetNodes(g, None, ctypes.byref(n)) == 0
    nodes = (ctypes.c_void_p * n.value)()
    assert cu.cuGraphGetNodes(g, nodes, ctypes.byref(n)) == 0
    out = []
    for node in nodes:
        kind = ctypes.c_int(-1)
        assert cu.cuGraphNodeGetType(ctypes.c_void_p(node), ctypes.byref(kind)) == 0
        if kind.value == 0:                                   # CU_GRAPH_NODE_TYPE_KERNEL
            out.append(ctypes.c_void_p(node))
    return out, cu


class KernelNodeParams(ctypes.Structure):                     # CUDA_KERNEL_NODE_PARAMS_v2
    _fields_ = [("func", ctypes.c_void_p), ("dims", ctypes.c_uint * 6), ("shared_bytes", ctypes.c_uint), ("params", ctypes.c_void_p),
                ("extra", ctypes.c_void_p), ("kern", ctypes.c_void_p), ("ctx", ctypes.c_void_p)]


class LaunchAttribute(ctypes.Structure):                      # CUlaunchAttribute
    _fields_ = [("id", ctypes.c_int), ("pad", ctypes.c_int), ("value", ctypes.c_uint * 16)]


class LaunchConfig(ctypes.Structure):                         # CUlaunchConfig
    _fields_ = [("dims", ctypes.c_uint * 6), ("shared_bytes", ctypes.c_uint), ("stream", ctypes.c_void_p),
                ("attributes", ctypes.POINTER(LaunchAttribute)), ("n", ctypes.c_uint)]


@pytest.mark.parametrize("shape", [(300, 500), (2048, 2048)])
def test_products_whose_blocks_wait_for_one_another_are_launched_cooperatively(shape):
    """The last kernel of the call (norm, copy, products) must be placed whole or not at all: seen on a captured graph before it is
    run; then replayed."""
    call = Orthogonalize(shape, 1)
    want = alone(call)                                        # also loads the module and sets the kernel's attributes
    g = capture(call)
    nodes, cu = kernel_nodes(g)
    cooperative = []
    for node in nodes:
        value = (ctypes.c_int * 16)()                         # CUlaunchAttributeValue: 64 bytes
        assert cu.cuGraphKernelNodeGetAttribute(node, 2, value) == 0          # CU_LAUNCH_ATTRIBUTE_COOPERATIVE
        cooperative.append(value[0])
    assert len(cooperative) == 3 and cooperative.count(1) == 1, cooperative
    call.y.fill_(7)
    g.instantiate()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    B.relay_poll_status()
    assert torch.equal(call.y, want[0])


@pytest.mark.parametrize("first,second", [((300, 500), (500, 300)), ((2048, 2048), (1024, 2048)), ((8, 512, 1024), (300, 300))])
def test_orthogonalised_updates_on_two_streams(first, second):
    check_overlap(Orthogonalize(first, 1), Orthogonalize(second, 2, F32))


def test_a_small_matrix_on_the_chip_leaves_room_for_a_large_one():
    """The limit of dynamic shared memory is the kernel's, whichever thread set it last."""
    small, large = Orthogonalize((40, 40), 1), Orthogonalize((128, 2048), 2)
    alone(large)
    g = capture(large)
    nodes, cu = kernel_nodes(g)
    p = KernelNodeParams()
    assert len(nodes) == 1 and cu.cuGraphKernelNodeGetParams_v2(nodes[0], ctypes.byref(p)) == 0
    func = ctypes.c_void_p(p.func)
    if not p.func:
        assert cu.cuKernelGetFunction(ctypes.byref(func), ctypes.c_void_p(p.kern)) == 0
    limit = ctypes.c_int(0)
    for call in (large, small):
        alone(call)
        assert cu.cuFuncGetAttribute(ctypes.byref(limit), 8, func) == 0       # CU_FUNC_ATTRIBUTE_MAX_DYNAMIC_SHARED_SIZE_BYTES
        assert limit.value >= p.shared_bytes > 150 * 1024, (limit.value, p.shared_bytes)


def test_matrices_on_the_chip_from_two_host_threads():
    """They share a kernel and differ in the shared memory that they ask for."""
    calls = [Orthogonalize((40, 40), 1), Orthogonalize((128, 2048), 2)]
    want = [alone(c) for c in calls]
    for t in (calls[0].y, calls[1].y):
        t.fill_(7)
    torch.cuda.synchronize()
    errors = []

    def work(call):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(3000):
                    call()
                torch.cuda.current_stream().synchronize()
        except Exception as e:                                # shown by the assertion below
            errors.append(e)

    threads = [threading.Thread(target=work, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    B.relay_poll_status()
    for w, c in zip(want, calls):
        assert torch.equal(w[0], c.y)


@pytest.mark.parametrize("dt,out_dt", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("tiles", [8, 35, 72, 128, 160, 512])
def test_persistent_clusters_of_the_recurrence_are_planned_for_the_room_they_find(dt, out_dt, grad, tiles):
    """A cluster walks over tiles, so a grid that does not fit at once makes the last clusters wait for a whole share.  What fits is
    CUDA's occupancy query for this kernel, its cluster size and its shared memory."""
    T, D = 512, 64 * tiles
    f, u, h, dh = (torch.zeros(T, 1, D, dtype=t, device=DEV) for t in (dt, dt, out_dt, out_dt))
    df, du = torch.empty_like(f), torch.empty_like(u)

    def call():
        if grad:
            B.relay_gated_recurrence_grad(f, u, None, None, B.GATE_MIX, h, dh, None, df, du, None)
        else:
            B.relay_gated_recurrence(f, u, None, None, B.GATE_MIX, h, None)

    call()
    g = capture(call)
    nodes, cu = kernel_nodes(g)
    p = KernelNodeParams()
    assert len(nodes) == 1 and cu.cuGraphKernelNodeGetParams_v2(nodes[0], ctypes.byref(p)) == 0
    func = ctypes.c_void_p(p.func)
    if not p.func:
        assert cu.cuKernelGetFunction(ctypes.byref(func), ctypes.c_void_p(p.kern)) == 0
    size = (ctypes.c_uint * 16)()
    assert cu.cuGraphKernelNodeGetAttribute(nodes[0], 4, size) == 0           # CU_LAUNCH_ATTRIBUTE_CLUSTER_DIMENSION
    attribute = LaunchAttribute(id=4)
    attribute.value[:3] = size[:3]
    config = LaunchConfig(dims=p.dims, shared_bytes=p.shared_bytes, attributes=ctypes.pointer(attribute), n=1)
    clusters = ctypes.c_int(0)
    assert cu.cuOccupancyMaxActiveClusters(ctypes.byref(clusters), func, ctypes.byref(config)) == 0
    assert p.dims[0] // size[0] <= clusters.value, (p.dims[0], size[0], clusters.value)


@pytest.mark.parametrize("first,second", [
    (lambda: Recurrence(3000, 1, 512, 1), lambda: Recurrence(700, 4, 1024, 11, F32)),
    (lambda: Recurrence(900, 3, 333, 1), lambda: Recurrence(8, 64, 1024, 11)),
    (lambda: TokenLogprob(8, 131072, 20, 1), lambda: TokenLogprob(600, 5003, 5, 11, F32)),
    (lambda: Recurrence(3000, 1, 512, 1), lambda: TokenLogprob(8, 131072, 20, 11)),
    (lambda: Orthogonalize((300, 500), 1), lambda: Recurrence(3000, 1, 512, 11, F32)),
    (lambda: Orthogonalize((128, 2048), 1), lambda: TokenLogprob(600, 5003, 64, 11))],
    ids=["tiles", "spans and steps", "log-probabilities", "recurrence and log-probabilities", "products and recurrence", "on the chip and log-probabilities"])
def test_operators_of_a_language_model_on_two_streams(first, second):
    check_overlap(first(), second())
