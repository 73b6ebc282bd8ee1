"""Calls that overlap: on two streams, or from two host threads, each with buffers of its own.  Results have the bits of the same call
alone."""
import ctypes

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


def kernel_attributes(graph, attribute):
    """Of every kernel node of a captured graph that was not run."""
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
            value = (ctypes.c_int * 16)()                     # CUlaunchAttributeValue: 64 bytes
            assert cu.cuGraphKernelNodeGetAttribute(ctypes.c_void_p(node), attribute, value) == 0
            out.append(value[0])
    return out


@pytest.mark.parametrize("shape", [(300, 500), (2048, 2048)])
def test_products_whose_blocks_wait_for_one_another_are_launched_cooperatively(shape):
    """The last kernel of the call (norm, copy, products) must be placed whole or not at all: seen on a captured graph before it is
    run; then replayed."""
    call = Orthogonalize(shape, 1)
    want = alone(call)                                        # also loads the module and sets the kernel's attributes
    g = torch.cuda.CUDAGraph(keep_graph=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        call()
    cooperative = kernel_attributes(g, 2)                     # CU_LAUNCH_ATTRIBUTE_COOPERATIVE
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
