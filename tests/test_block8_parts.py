"""Products in 8 bits made in parts through a workspace, with a second launch that adds them: on another stream and in a captured graph."""
import pytest
import torch

import paper_2601_07396_amd as svdc
from test_block8 import bytes_of, make_product

pytestmark = pytest.mark.gpu

PRODUCTS = [(1160, 320, 11072, torch.float32, "none"), (1160, 320, 11072, torch.bfloat16, "gelu"), (1160, 320, 11072, torch.float8_e4m3fn, "swiglu"),
            (300, 500, 12000, torch.bfloat16, "swiglu"), (468, 285, 5218, torch.float32, "swiglu"), (150, 260, 8000, torch.float8_e4m3fn, "gelu")]


def outputs(M, N, dtype):
    if dtype == torch.float8_e4m3fn:
        return svdc.alloc_q8(M, N, "cuda")
    return torch.empty(M, N, device="cuda", dtype=dtype), None


def same(a, b):
    return all((x is None and y is None) or (bytes_of(x) == bytes_of(y)).all() for x, y in zip(a, b))


def in_parts(M, N, K, dtype, act):
    p = svdc.make_matmul8(M, N, K, dtype, act)
    ws = svdc.alloc_matmul8_workspace(p, "cuda")
    assert ws is not None, "made without a workspace: not what this test is for"
    return p, ws


@pytest.mark.parametrize("M,N,K,dtype,act", PRODUCTS)
def test_parts_on_other_streams(M, N, K, dtype, act):
    """Two streams at once, a workspace each, give the bits of the current one; what was in the workspace does not matter."""
    p, ws = in_parts(M, N, K, dtype, act)
    (A, As, _), (W, Ws, _) = make_product(M, 2 * N if act == "swiglu" else N, K, 7)
    want = outputs(M, N, dtype)
    svdc.svdcache_matmul8(p, A, As, W, Ws, None, *want, ws.fill_(0xFF))
    torch.cuda.synchronize()
    sides = [(torch.cuda.Stream(), svdc.alloc_matmul8_workspace(p, "cuda").fill_(i), outputs(M, N, dtype)) for i in (0, 0x7F)]
    for _ in range(3):
        for stream, mine, out in sides:
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                for _ in range(4):
                    svdc.svdcache_matmul8(p, A, As, W, Ws, None, *out, mine)
        for stream, _, out in sides:
            stream.synchronize()
            assert same(out, want)
            out[0].view(torch.uint8).zero_()
        torch.cuda.synchronize()


@pytest.mark.parametrize("M,N,K,dtype,act", PRODUCTS)
def test_parts_in_a_graph(M, N, K, dtype, act):
    """Captured once with the quantisation before it, replayed on new inputs with eager work in between."""
    p, ws = in_parts(M, N, K, dtype, act)
    _, (W, Ws, _) = make_product(1, 2 * N if act == "swiglu" else N, K, 3)
    X = torch.randn(M, K, device="cuda")
    (Q, s), out, pq = svdc.alloc_q8(M, K, "cuda"), outputs(M, N, dtype), svdc.make_quant8(X)

    def step():
        svdc.svdcache_quantize8(pq, X, Q, s)
        svdc.svdcache_matmul8(p, Q, s, W, Ws, None, *out, ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        X.normal_(generator=torch.Generator("cuda").manual_seed(i))
        step()
        want = [None if t is None else t.clone() for t in out]
        out[0].view(torch.uint8).zero_()
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert same(out, want)
