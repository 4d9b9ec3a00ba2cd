"""A token with a NaN or an infinity on its way through layers of 8-bit operands: NaN everywhere but behind a fused Relu; the other tokens as they were."""
import math

import pytest
import torch

from paper_2008_08272_b200 import binding


@pytest.mark.gpu
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("M", [3, 12, 70, 300])
def test_a_bad_token_stays_nan(M, value):
    g = torch.Generator(device="cuda").manual_seed(71)
    X, Wg, Wu = (torch.randn(n, 100, generator=g, device="cuda") for n in (M, 130, 130))
    (Qg, sg), (Qu, su) = binding.onnx_quantize_rows(Wg), binding.onnx_quantize_rows(Wu)
    bad = X.clone()
    bad[1, 99] = value
    others = [i for i in range(M) if i != 1]

    def layers(x):
        q, s = binding.onnx_quantize_rows(x)
        out = [binding.onnx_gemm_int8(q, s, Qg, sg, su)]
        out += [binding.onnx_gated_int8(q, s, Qg, sg, Qu, su, activation=kind, dtype=torch.bfloat16) for kind in binding.ACTIVATIONS]
        again, s2 = binding.onnx_quantize_rows(out[1])
        return out + [binding.onnx_gemm_int8(again, s2, again[2:3], s2[2:3])], binding.onnx_gemm_int8(q, s, Qg, sg, su, fuse_relu=True)

    (got, relu), (want, clean) = layers(bad), layers(X)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert bool(a[1].isnan().all()) and torch.equal(a[others], b[others])
    assert bool((relu[1] == 0).all()) and torch.equal(relu[others], clean[others])
