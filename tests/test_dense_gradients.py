"""The gated block's gradients where what one call computes must not go by what it does besides: which results are wanted, how many tokens
there are."""
import itertools
import math

import pytest
import torch

import dense_reference as ref
from paper_2008_08272_b200 import binding
from paper_2008_08272_b200.binding import Matrix

# (tokens, width, channels), dX's long reduction in parts by the rule: short and long rows, whole K blocks and odd ones
IN_PARTS = [(64, 4096, 10240), (96, 264, 3001), (128, 512, 1024), (200, 1024, 2816), (512, 1024, 4096), (512, 512, 1090), (1024, 1024, 4096)]
FORMS = [w for w in itertools.product((True, False), repeat=3) if w[0]]


def normal(g, *size):
    return torch.randn(*size, generator=g, device="cuda")


def views(*sizes):
    """bfloat16 views at addresses of their own, rows at multiples of 16 bytes (nothing is launched on them)."""
    return [Matrix((i + 1) << 24, rows, cols, (cols + 7) // 8 * 8, 16, 0) for i, (rows, cols) in enumerate(sizes)]


@pytest.mark.parametrize("size", IN_PARTS, ids=str)
def test_parts_of_dX_do_not_go_by_what_else_is_wanted(size):
    """Each part has a plane of fp32 in the workspace, whole tiles of 128 or 256 rows: as many parts in every form (no GPU needed)."""
    M, K, F = size
    dH, X, W, dX, dW = views((M, F), (M, K), (F, K), (M, K), (F, K))
    lib, found = binding.load(), set()
    for _, g, u in FORMS:
        need = lib.onnx_gated_backward_workspace_bytes(dH, X if g or u else None, W, W, dX, dW if g else None, dW if u else None)
        planes = (need - 2 * M * dH.ld * 2) / ((K + 3) // 4 * 4 * 4)
        fits = {planes / rows for rows in (-(-M // 128) * 128, -(-M // 256) * 256)} & {2.0, 4.0, 8.0}
        assert fits, (size, planes)
        found.add(frozenset(fits))
    assert frozenset.intersection(*found), found


@pytest.mark.gpu
@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("size", IN_PARTS + [(2048, 1024, 4096), (1, 4096, 10240), (20, 1024, 4096), (32, 512, 2816)], ids=str)
def test_dX_is_the_same_whatever_else_is_wanted(size, t):
    """Bit by bit, with nothing pinned: a weight that is frozen does not change the other gradients."""
    g = torch.Generator(device="cuda").manual_seed(61)
    M, K, F = size
    X, Wg, Wu = normal(g, M, K).to(t), (normal(g, F, K) / math.sqrt(K)).to(t), (normal(g, F, K) / math.sqrt(K)).to(t)
    dH, G, U = normal(g, M, F).to(t), normal(g, M, F).to(t), normal(g, M, F).to(t)
    every = binding.onnx_gated_backward(dH, X, Wg, Wu, G, U)
    for wanted in itertools.product((True, False), repeat=3):
        if not any(wanted):
            continue
        some = binding.onnx_gated_backward(dH, X, Wg, Wu, G, U, wanted=wanted)
        for w, a, b in zip(wanted, some, every):
            assert (a is None) == (not w) and (a is None or torch.equal(a, b)), wanted
    assert binding.last_device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("M", [1, 5, 32, 33, 150])
def test_infinite_operands_give_what_the_sums_give(M, t):
    """An infinity (or NaN) among X or the weights: the results it goes into are infinite with the sign of dG or dU, or NaN, as the definition
    has it, up to 32 tokens as above; all others are as they were."""
    g = torch.Generator(device="cuda").manual_seed(62)
    K, F = 72, 200
    X, Wg, Wu = normal(g, M, K).to(t), (normal(g, F, K) / 9).to(t), (normal(g, F, K) / 9).to(t)
    dH, G, U = ((1 + torch.rand(M, F, generator=g, device="cuda")).to(t) * normal(g, M, F).sign().to(t) for _ in range(3))
    clean = binding.onnx_gated_backward(dH, X, Wg, Wu, G, U, activation="gelu")
    value, slope = ref.act("gelu", G.double())
    dG, dU = dH.double() * U.double() * slope, dH.double() * value       # none of them 0
    for where, at, v in (("X", (0, 7), math.inf), ("X", (M - 1, 71), -math.inf), ("X", (M // 2, 0), math.nan), ("Wg", (9, 3), math.inf),
                         ("Wu", (199, 64), -math.inf), ("Wg", (100, 70), math.nan)):
        own = {"X": X, "Wg": Wg, "Wu": Wu}
        own[where] = own[where].clone()
        own[where][at] = v
        got = binding.onnx_gated_backward(dH, own["X"], own["Wg"], own["Wu"], G, U, activation="gelu")
        torch.cuda.synchronize()
        column, factor = at[1], {"X": None, "Wg": dG[:, at[0]], "Wu": dU[:, at[0]]}[where]
        want = [c.double() for c in clean]
        if where == "X":
            want[1][:, column], want[2][:, column] = dG[at[0]] * v, dU[at[0]] * v
        else:
            want[0][:, column] = factor * v
        for y, w in zip(got, want):
            assert torch.equal(y.double().nan_to_num(7.0, 3e38, -3e38), w.nan_to_num(7.0, 3e38, -3e38)) and torch.equal(y.isnan(), w.isnan()), (where, at, v)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [4, 40])
def test_dG_beyond_the_types_range(M):
    """dG and dU are held in the operands' type: one above float16's largest number is infinite, and so is what it goes into (dX of its token,
    dWg of its channel), no more than that; bfloat16 takes it."""
    g = torch.Generator(device="cuda").manual_seed(63)
    K, F = 64, 96
    X, Wg, Wu, dH, G, U = (normal(g, *s) for s in ((M, K), (F, K), (F, K), (M, F), (M, F), (M, F)))
    large, G[2, 9], U[2, 9] = dH.clone(), 8.0, 4.0
    large[2, 9] = 30000.0
    rows, channels = [i for i in range(M) if i != 2], [j for j in range(F) if j != 9]
    for t in (torch.float16, torch.bfloat16):
        clean, got = ([y.float() for y in binding.onnx_gated_backward(*(v.to(t) for v in (d, X, Wg, Wu, G, U)))] for d in (dH, large))
        torch.cuda.synchronize()
        assert torch.equal(got[0][rows], clean[0][rows]) and all(torch.equal(a[channels], b[channels]) for a, b in zip(got[1:], clean[1:]))
        if t == torch.bfloat16:
            assert all(bool(y.isfinite().all()) for y in got)
        else:
            assert not bool(got[0][2].isfinite().any()) and not bool(got[1][9].isfinite().any())


class Gated(torch.autograd.Function):
    """The gated block with its gradients, as a training program has them."""

    @staticmethod
    def forward(ctx, X, Wg, Wu):
        H, G, U = binding.onnx_gated(X, Wg, Wu, save=True)
        ctx.save_for_backward(X, Wg, Wu, G, U)
        return H

    @staticmethod
    def backward(ctx, dH):
        return binding.onnx_gated_backward(dH.contiguous(), *ctx.saved_tensors, wanted=ctx.needs_input_grad)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [7, 90])
def test_within_autograd(M):
    """The calls leave autograd alone (no graph, of parameters neither), and serve as a function of it, a frozen weight among the inputs."""
    g = torch.Generator(device="cuda").manual_seed(64)
    X, Wg, Wu, dH = (normal(g, *s).bfloat16() for s in ((M, 72), (96, 72), (96, 72), (M, 96)))
    leaves = [torch.nn.Parameter(v) for v in (X, Wg, Wu)]
    assert not any(y.requires_grad for y in binding.onnx_gated(*leaves, save=True))
    H, G, U = binding.onnx_gated(X, Wg, Wu, save=True)
    for frozen, dH in ((None, dH), (1, dH), (None, torch.ones_like(dH[:1, :1]).expand(M, 96))):
        want = binding.onnx_gated_backward(dH.contiguous(), X, Wg, Wu, G, U)
        for i, leaf in enumerate(leaves):
            leaf.grad = None
            leaf.requires_grad_(i != frozen)
        y = Gated.apply(*leaves)
        y.backward(dH)
        torch.cuda.synchronize()
        assert torch.equal(y, H) and all(leaf.grad is None if i == frozen else torch.equal(leaf.grad, w) for i, (leaf, w) in enumerate(zip(leaves, want)))
