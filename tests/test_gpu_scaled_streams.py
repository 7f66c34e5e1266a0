"""An explicit stream of the 8-bit calls is the one that runs: a graph is captured on it while another stream is the current one, so that a launch elsewhere is not in
the graph."""
import pytest
import torch

from paper_2605_19269_amd import coda
from tests import q8_ref as R

pytestmark = pytest.mark.gpu


def calls():
    """name -> (call of a stream, its outputs)"""
    g = torch.Generator().manual_seed(3)
    dev = lambda t: t.cuda()
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")
    X = dev(torch.randn(40, 256, generator=g).to(torch.bfloat16))
    q, s, st = u8(40, 256), u8(2, 48), u8(1, 256)
    codes, scales = dev(R.random_codes(g, (40, 256))), dev(R.random_scales(g, 2, 40))
    back = torch.zeros(40, 256, dtype=torch.bfloat16, device="cuda")
    out = {"quantize": (lambda at: coda.coda_quantize(X, q, s, stream=at), (q, s)),
           "square": (lambda at: coda.coda_quantize(X, q, s, scales_t=st, square=True, stream=at), (q, s, st)),
           "dequantize": (lambda at: coda.coda_dequantize(codes, scales, back, stream=at), (back,))}
    for name, M, N, K, ws in (("few rows", 8, 256, 512, False), ("tiles", 40, 256, 512, False), ("partials", 70, 544, 2064, True)):
        a, sa = dev(R.random_codes(g, (M, K))), dev(R.random_scales(g, R.blocks(K), M))
        b, sb = dev(R.random_codes(g, (N, K))), dev(R.random_scales(g, R.blocks(K), N))
        D = torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")
        w = u8(coda.coda_gemm_scaled_workspace_bytes(M, N, K)) if ws else None
        out[name] = (lambda at, a=a, sa=sa, b=b, sb=sb, D=D, w=w: coda.coda_gemm_scaled(a, sa, b, sb, [coda.store(D)], transB=True, workspace=w, stream=at), (D,))
    for name, ws in (("gradient", False), ("gradient in ranges", True)):
        a, sa = dev(R.random_codes(g, (1000, 272))), dev(R.random_scales(g, 3, 1000))
        b, sb = dev(R.random_codes(g, (1000, 144))), dev(R.random_scales(g, 2, 1000))
        D = torch.zeros(272, 144, device="cuda")
        w = u8(coda.coda_grad_scaled_workspace_bytes(272, 144, 1000)) if ws else None
        out[name] = (lambda at, a=a, sa=sa, b=b, sb=sb, D=D, w=w: coda.coda_grad_scaled(a, sa, b, sb, D, workspace=w, stream=at), (D,))
    return out


@pytest.mark.parametrize("name", ["quantize", "square", "dequantize", "few rows", "tiles", "partials", "gradient", "gradient in ranges"])
def test_an_explicit_stream_is_the_one_that_runs(name):
    call, outputs = calls()[name]
    call(None)
    torch.cuda.synchronize()
    once = [t.clone() for t in outputs]
    assert all(bool(t.any()) for t in once)
    side, other, graph = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        with torch.cuda.stream(other):
            call(side)
    for _ in range(3):
        for t in outputs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, want) for t, want in zip(outputs, once))
