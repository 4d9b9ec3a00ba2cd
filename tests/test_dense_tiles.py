"""Every tile shape of the tensor-core kernel of the dense layers, and every number of parts that dX's reduction is shared by, pinned
through the environment: results against the definitions in 64 bits (dense_reference.py)."""
import math

import pytest
import torch

import dense_reference as ref
from paper_2008_08272_b200 import binding

pytestmark = pytest.mark.gpu
TILES = ["1x32", "1x64", "1x96", "1x128", "1x160", "1x192", "1x224", "1x256", "2x64", "2x128", "2x192", "2x256"]
# (tokens, width, channels): one tile and many, more tiles than SMs, last tiles of few rows and columns
SIZES = [(40, 200, 70), (300, 520, 700), (700, 72, 2100), (2600, 136, 1300)]


def normal(g, *size):
    return torch.randn(*size, generator=g, device="cuda")


def check_forward(size):
    M, K, F = size
    g = torch.Generator(device="cuda").manual_seed(23)
    A, B, Bu = (torch.randint(-128, 128, (n, (K + 15) // 16 * 16), generator=g, device="cuda", dtype=torch.int8)[:, :K] for n in (M, F, F))
    sa, sb, su = (torch.rand(n, generator=g, device="cuda") / 99 for n in (M, F, F))
    for y_type in (torch.float32, torch.float16):
        assert ref.worst(binding.onnx_gemm_int8(A, sa, B, sb, sb, dtype=y_type), ref.gemm_int8(A, sa, B, sb, sb, False, y_type)) <= 1
        assert ref.worst(binding.onnx_gated_int8(A, sa, B, sb / 9, Bu, su, dtype=y_type), ref.gated_int8(A, sa, B, sb / 9, Bu, su, "silu", y_type)) <= 1
    for t in (torch.bfloat16, torch.float16):
        X, Wg, Wu = normal(g, M, K).to(t), (normal(g, F, K) / math.sqrt(K)).to(t), (normal(g, F, K) / math.sqrt(K)).to(t)
        got = binding.onnx_gated(X, Wg, Wu, save=True)
        for y, pair in zip(got, ref.gated(X, Wg, Wu, "silu")):
            assert ref.worst(y, pair) <= 1
        assert torch.equal(binding.onnx_gated(X, Wg, Wu), got[0])
    assert binding.last_device_status() == 0


# one reduction shared by a cluster: (tokens, width, channels) of few tiles, parts that are not equally long
LONG = [(20, 5000, 33), (40, 2000, 70), (130, 3001, 200), (300, 4104, 130), (128, 2200, 256), (150, 4096, 200)]


@pytest.mark.parametrize("size", LONG + [(70, 256, 100), (1000, 512, 640), (40, 2048, 72), (33, 704, 1000), (90, 320, 136)], ids=str)
@pytest.mark.parametrize("ks", [1, 2, 4])
@pytest.mark.parametrize("tile", ["1x32", "1x64", "1x128", "2x64", "2x128", "1x64/2"])
def test_blocks_per_stage(tile, ks, size, monkeypatch):
    """Stages of several K blocks, whole ones and the last of a reduction."""
    monkeypatch.setenv("ONNXB_DENSE_TILE", tile)
    monkeypatch.setenv("ONNXB_DENSE_KS", str(ks))
    check_forward(size)


@pytest.mark.parametrize("size", LONG, ids=str)
@pytest.mark.parametrize("split", [2, 4, 8])
@pytest.mark.parametrize("tile", ["1x32", "1x64", "1x128", "1x256"])
def test_shared_reductions(tile, split, size, monkeypatch):
    monkeypatch.setenv("ONNXB_DENSE_TILE", f"{tile}/{split}")
    check_forward(size)


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("tile", TILES)
def test_tile_shapes(tile, size, monkeypatch):
    monkeypatch.setenv("ONNXB_DENSE_TILE", tile)
    M, K, F = size
    g = torch.Generator(device="cuda").manual_seed(21)
    t = torch.bfloat16
    A, B, Bu = (torch.randint(-128, 128, (n, (K + 15) // 16 * 16), generator=g, device="cuda", dtype=torch.int8)[:, :K] for n in (M, F, F))
    sa, sb, su = torch.rand(M, generator=g, device="cuda") / 99, torch.rand(F, generator=g, device="cuda") / 99, torch.rand(F, generator=g, device="cuda") / 99
    for y_type in (torch.float32, t):
        assert ref.worst(binding.onnx_gemm_int8(A, sa, B, sb, sb, dtype=y_type), ref.gemm_int8(A, sa, B, sb, sb, False, y_type)) <= 1
        assert ref.worst(binding.onnx_gated_int8(A, sa, B, sb, Bu, su, dtype=y_type), ref.gated_int8(A, sa, B, sb, Bu, su, "silu", y_type)) <= 1
    X, Wg, Wu = normal(g, M, K).to(t), (normal(g, F, K) / math.sqrt(K)).to(t), (normal(g, F, K) / math.sqrt(K)).to(t)
    H, G, U = binding.onnx_gated(X, Wg, Wu, save=True)
    for y, pair in zip((H, G, U), ref.gated(X, Wg, Wu, "silu")):
        assert ref.worst(y, pair) <= 1
    dH = normal(g, M, F).to(t)
    for y, pair in zip(binding.onnx_gated_backward(dH, X, Wg, Wu, G, U), ref.gated_backward(dH, X, Wg, Wu, G, U, "silu")):
        assert ref.worst(y, pair) <= 1
    assert binding.last_device_status() == 0


@pytest.mark.parametrize("size", [(30, 64, 512), (300, 204, 900), (129, 77, 1030), (520, 328, 2056)], ids=str)
@pytest.mark.parametrize("parts", [1, 2, 4, 8])
@pytest.mark.parametrize("tile", ["1x64", "2x128", "2x256"])
def test_parts_of_the_reduction(tile, parts, size, monkeypatch):
    """dX in parts of its reduction, alone and beside the weights' gradients; both at once give what each gives by itself."""
    monkeypatch.setenv("ONNXB_DENSE_TILE", tile)
    monkeypatch.setenv("ONNXB_DENSE_PARTS", str(parts))
    M, K, F = size
    g = torch.Generator(device="cuda").manual_seed(22)
    t = torch.float16
    X, Wg, Wu = normal(g, M, K).to(t), (normal(g, F, K) / math.sqrt(K)).to(t), (normal(g, F, K) / math.sqrt(K)).to(t)
    dH, G, U = normal(g, M, F).to(t), normal(g, M, F).to(t), normal(g, M, F).to(t)
    want = ref.gated_backward(dH, X, Wg, Wu, G, U, "gelu")
    got = binding.onnx_gated_backward(dH, X, Wg, Wu, G, U, activation="gelu")
    alone = binding.onnx_gated_backward(dH, X, Wg, Wu, G, U, activation="gelu", wanted=(True, False, False))[0]
    weights = binding.onnx_gated_backward(dH, X, Wg, Wu, G, U, activation="gelu", wanted=(False, True, True))[1:]
    for y, pair in zip(got, want):
        assert ref.worst(y, pair) <= 1
    assert torch.equal(alone, got[0]) and all(torch.equal(a, b) for a, b in zip(weights, got[1:]))
    assert binding.last_device_status() == 0


@pytest.mark.parametrize("size", [(40, 200, 70), (300, 520, 700), (129, 77, 1030), (700, 136, 64), (64, 64, 2056)], ids=str)
@pytest.mark.parametrize("ks", [1, 2])
@pytest.mark.parametrize("tile", ["1x64", "1x128", "2x128", "2x256"])
def test_gradients_by_blocks_per_stage(tile, ks, size, monkeypatch):
    monkeypatch.setenv("ONNXB_DENSE_TILE", tile)
    monkeypatch.setenv("ONNXB_DENSE_KS", str(ks))
    M, K, F = size
    g = torch.Generator(device="cuda").manual_seed(24)
    t = torch.bfloat16
    X, Wg, Wu = normal(g, M, K).to(t), (normal(g, F, K) / math.sqrt(K)).to(t), (normal(g, F, K) / math.sqrt(K)).to(t)
    dH, G, U = normal(g, M, F).to(t), normal(g, M, F).to(t), normal(g, M, F).to(t)
    want = ref.gated_backward(dH, X, Wg, Wu, G, U, "relu")
    for parts in ("1", "4"):
        monkeypatch.setenv("ONNXB_DENSE_PARTS", parts)
        for y, pair in zip(binding.onnx_gated_backward(dH, X, Wg, Wu, G, U, activation="relu"), want):
            assert ref.worst(y, pair) <= 1
    assert binding.last_device_status() == 0


@pytest.mark.parametrize("size", [(1, 4096, 700), (3, 200, 33), (8, 1030, 257), (9, 520, 100), (16, 2056, 300), (12, 24, 40)], ids=str)
@pytest.mark.parametrize("warps", [4, 8, 16])
def test_few_tokens_by_warps(warps, size, monkeypatch):
    """Every number of warps that a block of the kernel for a few tokens may have; and the other kernel for the same tokens."""
    monkeypatch.setenv("ONNXB_DENSE_FEW_WARPS", str(warps))
    monkeypatch.setenv("ONNXB_DENSE_FEW", "16")
    check_forward(size)
    monkeypatch.setenv("ONNXB_DENSE_FEW", "0")
    check_forward(size)
