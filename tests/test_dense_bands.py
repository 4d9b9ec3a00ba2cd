"""Dense layers of many rows: tiles in several bands of rows, the last of them of fewer, across many columns of tiles; and graphs replayed on inputs that
have changed."""
import math

import pytest
import torch

import dense_reference as ref
from paper_2008_08272_b200 import binding

pytestmark = pytest.mark.gpu


def normal(g, *size):
    return torch.randn(*size, generator=g, device="cuda")


# (tokens, width, channels): a band is at most 32 row tiles (of 128 rows, or 256 of a pair), and what takes 40 MB of A's rows: 16500 rows of 64 are 129
# row tiles in bands of 26 and 25, or 65 in 22 and 21; 4900 of 8200 are 39 in bands of 20 and 19 (8 bits) or 13, or 20 in bands of 10 or of 7 and 6
@pytest.mark.parametrize("size", [(16500, 64, 1300), (4900, 8200, 600)], ids=str)
@pytest.mark.parametrize("tile", ["", "1x64", "1x256", "2x64", "2x256"])
def test_bands_of_rows(tile, size, monkeypatch):
    if tile:
        monkeypatch.setenv("ONNXB_DENSE_TILE", tile)
    M, K, F = size
    g = torch.Generator(device="cuda").manual_seed(91)
    A, B, Bu = (torch.randint(-128, 128, (n, K + 16 + -K % 16), generator=g, device="cuda", dtype=torch.int8)[:, :K] for n in (M, F, F))
    sa, sb, su = (torch.rand(n, generator=g, device="cuda") / 99 / math.sqrt(K) for n in (M, F, F))
    for y_type in (torch.float32, torch.bfloat16):
        assert ref.worst(binding.onnx_gemm_int8(A, sa, B, sb, sb, dtype=y_type), ref.gemm_int8(A, sa, B, sb, sb, False, y_type)) <= 1
        assert ref.worst(binding.onnx_gated_int8(A, sa, B, sb, Bu, su, dtype=y_type), ref.gated_int8(A, sa, B, sb, Bu, su, "silu", y_type)) <= 1
    t = torch.bfloat16
    X, Wg, Wu = normal(g, M, K).to(t), (normal(g, F, K) / math.sqrt(K)).to(t), (normal(g, F, K) / math.sqrt(K)).to(t)
    got = binding.onnx_gated(X, Wg, Wu, save=True)
    for y, pair in zip(got, ref.gated(X, Wg, Wu, "silu")):
        assert ref.worst(y, pair) <= 1
    assert torch.equal(binding.onnx_gated(X, Wg, Wu), got[0])
    assert binding.last_device_status() == 0


@pytest.mark.parametrize("M", [1, 12, 30, 300])
def test_a_graph_reads_its_inputs_anew(M):
    """Every operator captured once and replayed after all its inputs have been written over, in place: what a fresh call gives."""
    K, F, t = 200, 144, torch.bfloat16

    def inputs(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        halves = [normal(g, M, K).to(t), (normal(g, F, K) / 14).to(t), (normal(g, F, K) / 14).to(t), *(normal(g, M, F).to(t) for _ in range(3))]
        codes = [torch.randint(-128, 128, (n, K), generator=g, device="cuda", dtype=torch.int8) for n in (M, F, F)]
        scales = [torch.rand(n, generator=g, device="cuda") / 99 for n in (M, F, F)]
        return halves + codes + scales

    def calls(X, Wg, Wu, dH, G, U, A, B, Bu, sa, sb, su):
        odd = (X[:, 1:], Wg[:, 1:], Wu[:, 1:])                 # (laid out anew in a workspace)
        return [*binding.onnx_quantize_rows(X), binding.onnx_gemm_int8(A, sa, B, sb, su), binding.onnx_gated_int8(A, sa, B, sb, Bu, su, dtype=t),
                *binding.onnx_gated(X, Wg, Wu, save=True), binding.onnx_gated(*odd), *binding.onnx_gated_backward(dH, X, Wg, Wu, G, U),
                *binding.onnx_gated_backward(dH, *odd, G, U)]

    own = inputs(92)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = calls(*own)
    for seed in (93, 94):
        fresh = inputs(seed)
        for mine, other in zip(own, fresh):
            mine.copy_(other)
        graph.replay()
        want = calls(*fresh)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, want))
    assert binding.last_device_status() == 0
