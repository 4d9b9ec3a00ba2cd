"""Products whose weights go by the row's group, and their gradients, against their definition in 64 bits."""
import math

import pytest
import torch

from paper_2008_08272_b200 import binding

TYPES = {"float16": torch.float16, "bfloat16": torch.bfloat16}
U = 2.0 ** -24
gpu = pytest.mark.gpu


def half_step(t):
    return torch.finfo(t).eps / 2


def smallest(t):
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2


def activation(kind, g):
    """act(g) and act'(g) in 64 bits."""
    if kind == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p))
    if kind == "gelu":
        p = torch.special.erfc(-g / math.sqrt(2)) / 2
        return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        th = torch.tanh(c * (g + 0.044715 * g ** 3))
        return g * (1 + th) / 2, (1 + th) / 2 + g / 2 * (1 - th * th) * c * (1 + 3 * 0.044715 * g * g)
    return g.clamp(min=0), (g > 0).double()


class Case:
    """sizes: of the groups, one after the other; before, behind: rows of no group, which hold NaN as they lie."""

    def __init__(self, sizes, K, N, t, seed=0, before=0, behind=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *s: torch.randn(*s, generator=g, device="cuda")
        self.sizes, self.K, self.N, self.t = sizes, K, N, t
        R = self.R = before + sum(sizes) + behind
        ends = [before]
        for s in sizes:
            ends.append(ends[-1] + s)
        self.ends = ends
        self.offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
        self.X, self.dY, self.G, self.U = (normal(R, c).to(t) for c in (K, N, N, N))
        self.W, self.Wu = ((normal(len(sizes), N, K) / math.sqrt(K)).to(t) for _ in range(2))
        for x in (self.X, self.dY, self.G, self.U):
            x[:before] = float("nan")
            x[ends[-1]:] = float("nan")

    def rows(self):
        return slice(self.ends[0], self.ends[-1])

    def by_row(self, a, W):              # a[i] W[g]^T; W [groups, cols of the result, cols of a], all in 64 bits
        parts = [a[b:e] @ w.T for b, e, w in zip(self.ends, self.ends[1:], W)]
        return torch.cat(parts)

    def by_group(self, a, b):            # the sums of a[i]^T b[i]
        return torch.stack([a[s:e].T @ b[s:e] for s, e in zip(self.ends, self.ends[1:])])


def close(got, want, size, terms, t, extra=0.0):
    """Off by one rounding of the result and one of 32 bits (twice: the tensor cores may cut off) for each addition of `size`, the sum of magnitudes."""
    tol = half_step(t) * want.abs() + 2 * U * terms * size + extra + smallest(t)
    off = (got.double() - want).abs()
    assert (off <= 1.01 * tol).all(), (float((off / tol).nan_to_num(nan=float("inf")).max()), int((~(off <= 1.01 * tol)).sum()))


def in_norm(got, want, t, roundings=1):
    """Roundings of many values are at most half a step / sqrt(3) in the mean square."""
    if want.numel() >= 4096 and want.norm() > 0:
        assert float((got.double() - want).norm() / want.norm()) < 1.05 * half_step(t) / math.sqrt(3) * math.sqrt(roundings)


def check_gemm(c, Y):
    r = c.rows()
    want, size = c.by_row(c.X.double(), c.W.double()), c.by_row(c.X.double().abs(), c.W.double().abs())
    close(Y[r], want, size, c.K, c.t)
    in_norm(Y[r], want, c.t)


def check_gated(c, H, G, Up, kind):
    r = c.rows()
    X = c.X.double()
    g, u = c.by_row(X, c.W.double()), c.by_row(X, c.Wu.double())
    sg, su = c.by_row(X.abs(), c.W.double().abs()), c.by_row(X.abs(), c.Wu.double().abs())
    if G is not None:
        close(G[r], g, sg, c.K, c.t)
        close(Up[r], u, su, c.K, c.t)
    a, _ = activation(kind, g)
    # slopes are at most 1.13 in magnitude; the activation itself is right to 1e-5
    close(H[r], a * u, 0 * u, 0, c.t, extra=2 * U * c.K * (1.13 * sg * (u.abs() + 2 * U * c.K * su) + a.abs() * su) + 1e-5 * (a * u).abs() + 1e-7 * u.abs())
    in_norm(H[r], a * u, c.t)


def check_gemm_backward(c, dX, dW):
    dY = c.dY.double()
    if dX is not None:
        W = c.W.double().transpose(1, 2)
        close(dX[c.rows()], c.by_row(dY, W), c.by_row(dY.abs(), W.abs()), c.N, c.t)
        in_norm(dX[c.rows()], c.by_row(dY, W), c.t)
    if dW is not None:
        want = c.by_group(dY, c.X.double())
        close(dW, want, c.by_group(dY.abs(), c.X.double().abs()), max(c.sizes), c.t)
        in_norm(dW, want, c.t)


def check_gated_backward(c, dX, dWg, dWu, kind):
    dH, g, u, X = (x.double() for x in (c.dY, c.G, c.U, c.X))
    a, slope = activation(kind, g)
    dG, dU = dH * u * slope, dH * a
    # what rounding dG and dU makes of them, and the activation's own error
    off = [half_step(c.t) * d.abs() + 1e-5 * d.abs() + 1e-6 * (dH * f).abs() + smallest(c.t) for d, f in ((dG, u), (dU, torch.ones_like(u)))]
    if dX is not None:
        W = [w.double().transpose(1, 2) for w in (c.W, c.Wu)]
        want = sum(c.by_row(d, w) for d, w in zip((dG, dU), W))
        size = sum(c.by_row(d.abs(), w.abs()) for d, w in zip((dG, dU), W))
        close(dX[c.rows()], want, size, 2 * c.N, c.t, extra=sum(c.by_row(o, w.abs()) for o, w in zip(off, W)))
        in_norm(dX[c.rows()], want, c.t, 2)
    for got, d, o in ((dWg, dG, off[0]), (dWu, dU, off[1])):
        if got is not None:
            want = c.by_group(d, X)
            close(got, want, c.by_group(d.abs(), X.abs()), max(c.sizes), c.t, extra=c.by_group(o, X.abs()))
            in_norm(got, want, c.t, 2)


def check_all(c, kind="silu"):
    check_gemm(c, binding.onnx_grouped_gemm(c.X, c.W, c.offsets))
    H, G, Up = binding.onnx_grouped_gated(c.X, c.W, c.Wu, c.offsets, activation=kind, save=True)
    check_gated(c, H, G, Up, kind)
    alone = binding.onnx_grouped_gated(c.X, c.W, c.Wu, c.offsets, activation=kind)
    assert torch.equal(alone[c.rows()], H[c.rows()])
    check_gemm_backward(c, *binding.onnx_grouped_gemm_backward(c.dY, c.X, c.W, c.offsets))
    check_gated_backward(c, *binding.onnx_grouped_gated_backward(c.dY, c.X, c.W, c.Wu, c.G, c.U, c.offsets, activation=kind), kind)


@pytest.fixture(params=["0", "5000"], ids=["tensor-cores", "few"])
def few(request, monkeypatch):
    """By either kernel."""
    monkeypatch.setenv("ONNXB_GROUPED_FEW", request.param)


SHAPES = [([1], 8, 8), ([3], 64, 64), ([2, 0, 1], 72, 40), ([0, 5, 0, 0, 17, 16, 15, 1, 0], 128, 200), ([64, 65, 63, 1, 128], 192, 136),
          ([100, 0, 300, 129, 256], 256, 384), ([1000, 24], 320, 520), ([40] * 33, 64, 128), ([0] * 40 + [70, 2] + [0] * 30, 136, 264)]


@gpu
@pytest.mark.parametrize("sizes,K,N", SHAPES, ids=lambda v: str(v) if not isinstance(v, list) else f"{len(v)}groups")
@pytest.mark.parametrize("t", list(TYPES))
def test_groups(sizes, K, N, t, few):
    check_all(Case(sizes, K, N, TYPES[t], seed=K + N))


@gpu
@pytest.mark.parametrize("tile", ["1x16", "1x48", "1x128", "2x32", "2x96", "2x128", "2x256"])
@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh", "relu"])
def test_every_tile(tile, kind, monkeypatch):
    monkeypatch.setenv("ONNXB_GROUPED_TILE", tile)
    check_all(Case([130, 0, 1, 77, 300, 16], 200, 328, torch.bfloat16, seed=3, before=5, behind=70), kind)


@gpu
@pytest.mark.parametrize("tile", ["1x16", "1x48", "1x128", "2x32", "2x96", "2x128", "2x256"])
@pytest.mark.parametrize("blocks", ["1", "2"])
def test_blocks_of_a_stage(tile, blocks, monkeypatch):
    """Reductions of whole blocks of 64, of an odd and an even number, in stages of one and of two; groups that end in either of a stage's blocks."""
    monkeypatch.setenv("ONNXB_GROUPED_TILE", tile)
    monkeypatch.setenv("ONNXB_GROUPED_KS", blocks)
    check_all(Case([130, 0, 1, 77, 300, 16, 64, 192], 320, 448, torch.bfloat16, seed=3, before=5, behind=70))
    check_all(Case([257, 63], 128, 64, torch.float16, seed=5))


@gpu
@pytest.mark.parametrize("parts", ["2", "3", "16", "3,1", "1,3"])
@pytest.mark.parametrize("tile", ["1x48", "2x32", "2x256"])
@pytest.mark.parametrize("t", list(TYPES))
def test_parts_of_the_sums(parts, tile, t, monkeypatch):
    """Reductions in parts, some of which have no stages: of groups with few rows or none, and with the last stage in either; rows of no group stay as they were."""
    monkeypatch.setenv("ONNXB_GROUPED_TILE", tile)
    monkeypatch.setenv("ONNXB_GROUPED_PARTS", parts)
    cases = (Case([130, 0, 1, 77, 300, 16, 64, 192], 320, 448, TYPES[t], seed=3, before=5, behind=70), Case([257, 63, 129], 129, 65, TYPES[t], seed=5, behind=1),
             Case([5], 1000, 8, TYPES[t], seed=6), Case([1500, 700], 40, 136, TYPES[t], seed=7))
    for case, kind in zip(cases, ("silu", "gelu", "gelu_tanh", "relu")):
        check_all(case, kind)
        outside = torch.ones(case.R, dtype=torch.bool, device="cuda")
        outside[case.rows()] = False
        Y, H, G, Up, dX = (torch.full((case.R, n), 7.0, dtype=case.t, device="cuda") for n in (case.N, case.N, case.N, case.N, case.K))
        binding.onnx_grouped_gemm(case.X, case.W, case.offsets, Y=Y)
        binding.onnx_grouped_gated(case.X, case.W, case.Wu, case.offsets, H=H, G=G, U=Up)
        binding.onnx_grouped_gemm_backward(case.dY, case.X, case.W, case.offsets, dX=dX)
        for y in (Y, H, G, Up, dX):
            assert (y[outside] == 7.0).all()
        every = binding.onnx_grouped_gated_backward(case.dY, case.X, case.W, case.Wu, case.G, case.U, case.offsets)
        for i in range(1, 7):
            wanted = [bool(i & b) for b in (1, 2, 4)]
            some = binding.onnx_grouped_gated_backward(case.dY, case.X, case.W, case.Wu, case.G, case.U, case.offsets, wanted=wanted)
            for w, a, b in zip(wanted, some, every):
                assert not w or torch.equal(a[outside.logical_not()] if a.dim() == 2 else a, b[outside.logical_not()] if b.dim() == 2 else b)


@gpu
def test_long_sums_of_few_tiles():
    """Sizes whose sums are in parts by themselves, also of views, of offsets that do not rise and of a group that has all rows."""
    for c in (Case([2000, 1500], 4224, 64, torch.bfloat16, seed=1), Case([4000], 64, 200, torch.float16, seed=2, before=3, behind=9),
              Case([0, 900, 3], 72, 4104, torch.bfloat16, seed=3), Case([120, 0, 130, 7], 64, 5184, torch.bfloat16, seed=8), Case([3, 0, 0, 3000], 96, 96, torch.bfloat16, seed=4)):
        check_all(c)
        wide = torch.full((c.R, c.N + 3), 7.0, dtype=c.t, device="cuda")
        binding.onnx_grouped_gemm(c.X, c.W, c.offsets, Y=wide[:, 1:1 + c.N])
        check_gemm(c, wide[:, 1:1 + c.N])
        assert (wide[:, 0] == 7.0).all() and (wide[:, 1 + c.N:] == 7.0).all()
        both = torch.full((c.R, 3 * c.N + 1), 7.0, dtype=c.t, device="cuda")
        H, G, Up = (both[:, 1 + i * c.N:1 + (i + 1) * c.N] for i in range(3))
        binding.onnx_grouped_gated(c.X, c.W, c.Wu, c.offsets, activation="gelu", H=H, G=G, U=Up)
        check_gated(c, H, G, Up, "gelu")
        assert (both[:, 0] == 7.0).all()
        store = torch.full((len(c.sizes), c.N + 1, c.K + 5), 7.0, dtype=c.t, device="cuda")
        dX, dW = binding.onnx_grouped_gemm_backward(c.dY, c.X, c.W, c.offsets, dW=store[:, :c.N, :c.K])
        check_gemm_backward(c, dX, dW)
        assert (store[:, c.N:] == 7.0).all() and (store[:, :, c.K:] == 7.0).all()
    c.ends, c.sizes = [0, 50, 50, 3003, 3003], [50, 0, 2953, 0]
    c.offsets = torch.tensor([-7, 50, 20, 2 ** 31 - 1, 5], dtype=torch.int32, device="cuda")
    check_all(c)


@gpu
@pytest.mark.parametrize("K,N", [(1, 1), (7, 9), (65, 33), (100, 101), (777, 130), (130, 777)])
@pytest.mark.parametrize("t", list(TYPES))
def test_odd_widths(K, N, t, few):
    check_all(Case([20, 0, 33, 1], K, N, TYPES[t], seed=K, behind=3))


@gpu
@pytest.mark.parametrize("tile", ["1x128", "2x128", "2x256"])
def test_rows_of_no_group_are_left(tile, monkeypatch):
    monkeypatch.setenv("ONNXB_GROUPED_TILE", tile)
    c = Case([33, 0, 90], 96, 200, torch.float16, before=9, behind=50)
    outside = torch.ones(c.R, dtype=torch.bool, device="cuda")
    outside[c.rows()] = False

    def filled(cols):
        return torch.full((c.R, cols), 7.0, dtype=c.t, device="cuda")

    Y, H, G, Up, dX, dX2 = filled(c.N), filled(c.N), filled(c.N), filled(c.N), filled(c.K), filled(c.K)
    binding.onnx_grouped_gemm(c.X, c.W, c.offsets, Y=Y)
    binding.onnx_grouped_gated(c.X, c.W, c.Wu, c.offsets, H=H, G=G, U=Up)
    _, dW = binding.onnx_grouped_gemm_backward(c.dY, c.X, c.W, c.offsets, dX=dX)
    grads = binding.onnx_grouped_gated_backward(c.dY, c.X, c.W, c.Wu, c.G, c.U, c.offsets, dX=dX2)
    for y in (Y, H, G, Up, dX, dX2):
        assert (y[outside] == 7.0).all()
    check_gemm(c, Y)
    check_gated(c, H, G, Up, "silu")
    check_gemm_backward(c, dX, dW)
    check_gated_backward(c, *grads, "silu")


@gpu
@pytest.mark.parametrize("tile", ["1x16", "1x128", "2x128", "2x256"])
def test_what_is_not_finite_stays_in_its_group(tile, monkeypatch):
    """A group's rows, results and gradients are its own, wherever another's rows lie in the same tile or stage."""
    monkeypatch.setenv("ONNXB_GROUPED_TILE", tile)
    c = Case([21, 30, 5, 64, 9], 104, 136, torch.bfloat16, seed=9)
    clean = [binding.onnx_grouped_gemm(c.X, c.W, c.offsets), *binding.onnx_grouped_gemm_backward(c.dY, c.X, c.W, c.offsets),
             *binding.onnx_grouped_gated_backward(c.dY, c.X, c.W, c.Wu, c.G, c.U, c.offsets)]
    for g in (1, 3):
        rows = slice(c.ends[g], c.ends[g + 1])
        for x, bad in ((c.X, float("nan")), (c.dY, float("inf")), (c.G, float("nan")), (c.U, float("-inf"))):
            x[rows] = bad
        c.W[g], c.Wu[g] = float("nan"), float("inf")
    dirty = [binding.onnx_grouped_gemm(c.X, c.W, c.offsets), *binding.onnx_grouped_gemm_backward(c.dY, c.X, c.W, c.offsets),
             *binding.onnx_grouped_gated_backward(c.dY, c.X, c.W, c.Wu, c.G, c.U, c.offsets)]
    for a, b in zip(clean, dirty):
        for g in (0, 2, 4):
            at = g if a.dim() == 3 else slice(c.ends[g], c.ends[g + 1])
            assert torch.equal(a[at], b[at])
        for g in (1, 3):
            assert not b[g if a.dim() == 3 else slice(c.ends[g], c.ends[g + 1])].isfinite().any()


@gpu
@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh", "relu"])
def test_few_rows(kind):
    """Rows of no group before and behind, groups of more rows than are taken at once, and more groups than a block has threads."""
    for sizes, before, behind in (([1], 0, 0), ([0, 3, 0, 1], 2, 2), ([8], 0, 0), ([0] * 700 + [2] + [0] * 300 + [5], 1, 0)):
        check_all(Case(sizes, 104, 70, torch.float16, seed=len(sizes), before=before, behind=behind), kind)


@gpu
def test_views(few, request):
    """Halves of one tensor, all groups' first rows first, and rows and groups that begin anywhere.  The tensor cores have copies of such, laid out alike,
    and give the same bit by bit; the kernel for few rows reads them as they lie, and adds up their terms in another order."""
    same_order = "tensor-cores" in request.node.name
    c = Case([50, 3, 0, 140], 72, 88, torch.bfloat16, seed=4)
    E, N, K = c.W.shape
    both = torch.cat([c.W, c.Wu], 1)                                     # [E, 2N, K]
    across = c.W.transpose(0, 1).contiguous().transpose(0, 1)            # [E, N, K], groups K apart
    odd = torch.full((E * (N + 1) * (K + 3) + 1,), float("nan"), dtype=c.t, device="cuda")[1:].view(E, N + 1, K + 3)[:, :N, :K]
    odd.copy_(c.W)
    Y = binding.onnx_grouped_gemm(c.X, c.W, c.offsets)
    want = binding.onnx_grouped_gemm_backward(c.dY, c.X, c.W, c.offsets)
    for w in (both[:, :N], across, odd):
        got = binding.onnx_grouped_gemm(c.X, w, c.offsets)
        check_gemm(c, got)
        assert not same_order or torch.equal(Y, got)
        store = torch.full((E, N + 1, K + 5), 7.0, dtype=c.t, device="cuda")
        dX, dW = binding.onnx_grouped_gemm_backward(c.dY, c.X, w, c.offsets, dW=store[:, :N, :K])
        assert torch.equal(dX, want[0]) and torch.equal(dW, want[1]) and (store[:, N:] == 7.0).all() and (store[:, :, K:] == 7.0).all()
    H = binding.onnx_grouped_gated(c.X, c.W, c.Wu, c.offsets)
    assert torch.equal(H, binding.onnx_grouped_gated(c.X, both[:, :N], both[:, N:], c.offsets))
    wide = torch.full((c.R, K + 5), float("nan"), dtype=c.t, device="cuda")
    wide[:, 2:2 + K] = c.X
    out = torch.full((c.R, N + 3), 7.0, dtype=c.t, device="cuda")
    binding.onnx_grouped_gemm(wide[:, 2:2 + K], c.W, c.offsets, Y=out[:, 1:1 + N])
    check_gemm(c, out[:, 1:1 + N])
    assert not same_order or torch.equal(out[:, 1:1 + N], Y)
    assert (out[:, 0] == 7.0).all() and (out[:, 1 + N:] == 7.0).all()


@gpu
def test_wanted():
    """A result is the same bit by bit whichever others are wanted."""
    c = Case([50, 3, 0, 140], 72, 88, torch.float16, seed=4)
    both = binding.onnx_grouped_gemm_backward(c.dY, c.X, c.W, c.offsets)
    dX, none = binding.onnx_grouped_gemm_backward(c.dY, None, c.W, c.offsets, wanted=(True, False))
    assert none is None and torch.equal(dX, both[0])
    none, dW = binding.onnx_grouped_gemm_backward(c.dY, c.X, None, c.offsets, wanted=(False, True), dW=torch.empty_like(c.W))
    assert none is None and torch.equal(dW, both[1])
    every = binding.onnx_grouped_gated_backward(c.dY, c.X, c.W, c.Wu, c.G, c.U, c.offsets)
    for i in range(1, 7):
        wanted = [bool(i & b) for b in (1, 2, 4)]
        some = binding.onnx_grouped_gated_backward(c.dY, c.X if wanted[1] or wanted[2] else None, c.W, c.Wu, c.G, c.U, c.offsets, wanted=wanted)
        for w, a, b in zip(wanted, some, every):
            assert (a is None) if not w else torch.equal(a, b)


@gpu
def test_no_rows():
    c = Case([0, 0], 16, 24, torch.float16)
    assert binding.onnx_grouped_gemm(c.X, c.W, c.offsets).shape == (0, 24)
    dX, dW = binding.onnx_grouped_gemm_backward(c.dY, c.X, c.W, c.offsets)
    assert dX.shape == (0, 16) and dW.shape == c.W.shape and not dW.any()
    c = Case([0, 0], 16, 24, torch.float16, behind=40)          # rows, but no group has one
    Y = torch.full((40, 24), 7.0, dtype=c.t, device="cuda")
    binding.onnx_grouped_gemm(c.X, c.W, c.offsets, Y=Y)
    dX, dWg, dWu = binding.onnx_grouped_gated_backward(c.dY, c.X, c.W, c.Wu, c.G, c.U, c.offsets)
    assert (Y == 7.0).all() and not dWg.any() and not dWu.any()


@gpu
@pytest.mark.parametrize("offsets,ends", [([-5, 10, 300, 20], [0, 10, 60, 60]), ([20, 50, 30, 55], [20, 50, 50, 55]), ([59, 10, 5, 0], [59, 59, 59, 59]),
                                          ([0, 2 ** 31 - 1, -2 ** 31, 7], [0, 60, 60, 60])])
def test_few_rows_whose_offsets_do_not_rise(offsets, ends, few):
    c = Case([10, 20, 30], 64, 72, torch.bfloat16)
    c.ends, c.sizes = ends, [b - a for a, b in zip(ends, ends[1:])]
    c.offsets = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    Y = torch.full((c.R, c.N), 7.0, dtype=c.t, device="cuda")
    binding.onnx_grouped_gemm(c.X, c.W, c.offsets, Y=Y)
    assert (Y[:ends[0]] == 7.0).all() and (Y[ends[-1]:] == 7.0).all()
    if ends[0] < ends[-1]:
        check_gemm(c, Y)


@gpu
@pytest.mark.parametrize("offsets,ends", [([-5, 10, 300, 20], [0, 10, 100, 100]), ([20, 50, 30, 90], [20, 50, 50, 90]),
                                          ([90, 10, 5, 0], [90, 90, 90, 90]), ([0, 2 ** 31 - 1, -2 ** 31, 7], [0, 100, 100, 100])])
@pytest.mark.parametrize("tile", ["1x128", "2x128", "2x256"])
def test_offsets_that_do_not_rise(offsets, ends, tile, monkeypatch):
    """What is outside of 0 and the rows counts as the nearest end, one below the one before it as that: no row beyond the tensors is touched."""
    monkeypatch.setenv("ONNXB_GROUPED_TILE", tile)
    c = Case([10, 20, 70], 64, 72, torch.bfloat16)
    c.ends, c.sizes = ends, [b - a for a, b in zip(ends, ends[1:])]
    c.offsets = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    if c.ends[0] == c.ends[-1]:
        assert not binding.onnx_grouped_gemm_backward(c.dY, c.X, c.W, c.offsets)[1].any()
    else:
        check_all(c)


@gpu
def test_captured_with_offsets_that_change():
    """One graph, replayed with other offsets and inputs; two graphs on two streams with workspaces of their own."""
    runs = []
    for seed in (1, 2):
        c = Case([100, 30, 0, 70], 136, 200, torch.bfloat16, seed=seed)
        s = torch.cuda.Stream()
        ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            H, G, Up = binding.onnx_grouped_gated(c.X, c.W, c.Wu, c.offsets, save=True)
            grads = binding.onnx_grouped_gated_backward(c.dY, c.X, c.W, c.Wu, c.G, c.U, c.offsets, workspace=ws)
        runs.append((c, s, g, H, G, Up, grads, ws))
    for sizes in ([1, 0, 199, 0], [64, 64, 64, 8]):
        for c, *_ in runs:
            c.sizes, c.ends = sizes, [0] + torch.tensor(sizes).cumsum(0).tolist()
            c.offsets.copy_(torch.tensor(c.ends, dtype=torch.int32))
            c.X.copy_(torch.randn_like(c.X))
        torch.cuda.synchronize()
        for c, s, g, *_ in runs:
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for c, s, g, H, G, Up, grads, ws in runs:
            check_gated(c, H, G, Up, "silu")
            check_gated_backward(c, *grads, "silu")


@gpu
def test_checked_path_and_another_stream(monkeypatch):
    c = Case([50, 3, 0, 140], 72, 88, torch.float16, seed=4, behind=8)

    def calls(stream):
        H, G, Up = binding.onnx_grouped_gated(c.X, c.W, c.Wu, c.offsets, activation="gelu", save=True, stream=stream)
        out = [binding.onnx_grouped_gemm(c.X, c.W, c.offsets, stream=stream)[c.rows()], H[c.rows()], G[c.rows()], Up[c.rows()]]
        for grads in (binding.onnx_grouped_gemm_backward(c.dY, c.X, c.W, c.offsets, stream=stream),
                      binding.onnx_grouped_gated_backward(c.dY, c.X, c.W, c.Wu, c.G, c.U, c.offsets, activation="gelu", stream=stream)):
            out += [grads[0][c.rows()], *grads[1:]]
        return out

    native = calls(None)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        on_side = calls(side)
    torch.cuda.synchronize()
    monkeypatch.setattr(binding, "_fast_mod", binding._Declined())
    checked = calls(None)
    torch.cuda.synchronize()
    for a, b, d in zip(native, on_side, checked):
        assert a.dtype == b.dtype == d.dtype and torch.equal(a, b) and torch.equal(a, d)


@gpu
def test_a_layer_with_its_gradients():
    """Norm, router, gated block, down products and their sum, forward and backward, against torch's gradients in 64 bits; captured as a graph, too."""
    T, K, F, E, top = 300, 128, 192, 6, 2
    t = torch.float16
    g = torch.Generator(device="cuda").manual_seed(11)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x, scale, bias = normal(T, K).to(t), 1 + 0.1 * normal(K), 0.1 * normal(K)
    Wg, Wu, Wd = ((normal(*s) / math.sqrt(s[2])).to(t) for s in ((E, F, K), (E, F, K), (E, K, F)))
    share, expert = torch.softmax(normal(T, E), 1).topk(top)
    order = expert.flatten().argsort(stable=True)
    token, weight = order // top, share.flatten()[order]
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), torch.bincount(expert.flatten(), minlength=E).cumsum(0)]).to(torch.int32)
    dout = normal(T, K).to(t)

    def layer():
        y, mean, inv_std = binding.onnx_layer_normalization(x, scale, bias, save=True)
        rows = y[token]
        h, gate, up = binding.onnx_grouped_gated(rows, Wg, Wu, offsets, save=True)
        down = binding.onnx_grouped_gemm(h, Wd, offsets)
        out = torch.zeros(T, K, dtype=torch.float32, device="cuda").index_add_(0, token, down.float() * weight[:, None])
        ddown = (dout[token].float() * weight[:, None]).to(t)
        dh, dWd = binding.onnx_grouped_gemm_backward(ddown, h, Wd, offsets)
        drows, dWg, dWu = binding.onnx_grouped_gated_backward(dh, rows, Wg, Wu, gate, up, offsets)
        dy = torch.zeros(T, K, dtype=torch.float32, device="cuda").index_add_(0, token, drows.float()).to(t)
        return out, *binding.onnx_layer_normalization_backward(dy, x, scale, mean, inv_std), dWg, dWu, dWd

    leaves = [v.double().requires_grad_() for v in (x, scale, bias, Wg, Wu, Wd)]
    X, S, B, G, Up, D = leaves
    rows = torch.nn.functional.layer_norm(X, (K,), S, B, 1e-5)[token]
    ends = offsets.tolist()
    down = torch.cat([(torch.nn.functional.silu(rows[b:e] @ G[i].T) * (rows[b:e] @ Up[i].T)) @ D[i].T for i, (b, e) in enumerate(zip(ends, ends[1:]))])
    out = torch.zeros(T, K, dtype=torch.float64, device="cuda").index_add(0, token, down * weight.double()[:, None])
    out.backward(dout.double())
    want = [out.detach()] + [v.grad for v in leaves]

    def compare(got):
        # a result goes through at most nine roundings to 16 bits, each of at most half a step / sqrt(3) in the mean square
        for a, b in zip(got, want):
            assert float((a.double() - b).norm() / b.norm()) < half_step(t) / math.sqrt(3) * 9

    compare(layer())
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        layer()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = layer()
    graph.replay()
    torch.cuda.synchronize()
    compare(got)


@gpu
def test_gradients_against_differences():
    """The formula that the kernels are compared with, against differences of the forward formula in 64 bits."""
    c = Case([3, 0, 4], 5, 6, torch.float16, seed=2)
    X, W, Wu, dH = (v.double() for v in (c.X, c.W, c.Wu, c.dY))

    def loss(X, W, Wu):
        return float((activation("silu", c.by_row(X, W))[0] * c.by_row(X, Wu) * dH).sum())

    c.G, c.U = c.by_row(X, W).to(c.t), c.by_row(X, Wu).to(c.t)
    grads = binding.onnx_grouped_gated_backward(c.dY, c.X, c.W, c.Wu, c.G, c.U, c.offsets)
    h = 1e-4
    for which, grad in enumerate(grads):
        for i in range(grad.numel()):
            sides = []
            for sign in (h, -h):
                a = [X.clone(), W.clone(), Wu.clone()]
                a[which].view(-1)[i] += sign
                sides.append(loss(*a))
            # G, U, dG, dU and the result are rounded to 16 bits on the way
            assert abs((sides[0] - sides[1]) / (2 * h) - float(grad.view(-1)[i])) < 20 * half_step(c.t) * (1 + float(grad.abs().max()))


@gpu
def test_more_than_2_31_elements():
    """Rows behind the 2^31-th element of X, and of dX; a group's weights behind that of W."""
    R, K, N = (1 << 20) + 40, 2056, 8
    g = torch.Generator(device="cuda").manual_seed(3)
    X = torch.zeros(R, K, dtype=torch.float16, device="cuda")
    x, dy = torch.randn(60, K, generator=g, device="cuda").half(), torch.randn(60, N, generator=g, device="cuda").half()
    X[-60:] = x
    dY = torch.zeros(R, N, dtype=torch.float16, device="cuda")
    dY[-60:] = dy
    W = (torch.randn(2, N, K, generator=g, device="cuda") / math.sqrt(K)).half()
    offsets = torch.tensor([0, R - 60, R], dtype=torch.int32, device="cuda")
    c = Case([60], K, N, torch.float16)
    c.X, c.dY, c.W = x, dy, W[1:]
    check_gemm(c, binding.onnx_grouped_gemm(X, W, offsets)[-60:])
    dX, dW = binding.onnx_grouped_gemm_backward(dY, X, W, offsets)
    check_gemm_backward(c, dX[-60:], dW[1:])
    assert not dX[:-60].any() and not dW[0].any()
    del X, dX
    W = torch.zeros(900, 2400, 1000, dtype=torch.float16, device="cuda")
    c = Case([0] * 899 + [33], 1000, 2400, torch.float16)
    W[899] = c.W[899]
    c.W, c.Wu = W, W
    check_gemm(c, binding.onnx_grouped_gemm(c.X, W, c.offsets))
    dX, _ = binding.onnx_grouped_gemm_backward(c.dY, c.X, W, c.offsets, wanted=(True, False))
    check_gemm_backward(c, dX, None)


@gpu
def test_two_streams_at_once():
    """Calls that overlap in time leave one another's results alone."""
    cases = [Case([300, 0, 50, 700], 512, 384, torch.bfloat16, seed=1), Case([3, 2, 0, 1], 1024, 512, torch.bfloat16, seed=2)]

    def run(c):
        H, G, Up = binding.onnx_grouped_gated(c.X, c.W, c.Wu, c.offsets, save=True)
        return [H, G, Up, binding.onnx_grouped_gemm(c.X, c.W, c.offsets), *binding.onnx_grouped_gated_backward(c.dY, c.X, c.W, c.Wu, c.G, c.U, c.offsets)]

    want = [run(c) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = run(cases[i])
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert binding.last_device_status() == 0


@gpu
@pytest.mark.parametrize("tile", ["1x32", "1x64", "1x96", "2x160", "2x192"])
@pytest.mark.parametrize("kind", ["silu", "relu"])
def test_gated_exchange_from_tile_to_tile(tile, kind, monkeypatch):
    """Several short tiles a CTA, one after the other, whose warps exchange an odd number of blocks in each: what one gives in a tile is not what the other still
    reads of the tile before."""
    monkeypatch.setenv("ONNXB_GROUPED_TILE", tile)
    c = Case([1500, 33, 1, 0, 900, 161], 64, 1000, torch.bfloat16, seed=12)
    H, G, Up = binding.onnx_grouped_gated(c.X, c.W, c.Wu, c.offsets, activation=kind, save=True)
    check_gated(c, H, G, Up, kind)
    for _ in range(50):
        assert torch.equal(H, binding.onnx_grouped_gated(c.X, c.W, c.Wu, c.offsets, activation=kind))


@gpu
@pytest.mark.parametrize("tile", ["1x16", "1x128", "2x32", "2x256"])
@pytest.mark.parametrize("sizes", [[0] * 899 + [950], [700] + [0] * 600, [0] * 300 + [40] * 10 + [0] * 300], ids=["last", "first", "middle"])
def test_most_of_the_grid_has_no_tile(tile, sizes, monkeypatch):
    """Few groups have rows: the grid has thousands of blocks behind the last tile, which are passed over, and no tile with them; also in parts of the sums."""
    monkeypatch.setenv("ONNXB_GROUPED_TILE", tile)
    c = Case(sizes, 136, 1032, torch.bfloat16, seed=13)
    check_all(c)
    dX, _ = binding.onnx_grouped_gemm_backward(c.dY, None, c.W, c.offsets, wanted=(True, False))
    check_gemm_backward(c, dX, None)
    monkeypatch.setenv("ONNXB_GROUPED_PARTS", "2")
    check_all(c)


@gpu
@pytest.mark.parametrize("tile", ["1x16", "1x64", "1x128", "2x128", "2x256"])
@pytest.mark.parametrize("parts", [None, "2"])
@pytest.mark.parametrize("kind", ["silu", "relu"])
def test_gated_block_of_what_is_not_finite(tile, parts, kind, monkeypatch):
    """A group's rows and weights that are not finite: the other groups' H, G and U are the same bit by bit, whichever values the warps exchange."""
    monkeypatch.setenv("ONNXB_GROUPED_TILE", tile)
    if parts:
        monkeypatch.setenv("ONNXB_GROUPED_PARTS", parts)
    c = Case([21, 30, 5, 64, 9, 100], 136, 200, torch.bfloat16, seed=9, before=3, behind=4)
    clean = binding.onnx_grouped_gated(c.X, c.W, c.Wu, c.offsets, activation=kind, save=True)
    for g, bad in ((1, float("nan")), (3, float("inf"))):
        c.X[c.ends[g]:c.ends[g + 1]] = bad
        c.W[g], c.Wu[g] = bad, -bad
    dirty = binding.onnx_grouped_gated(c.X, c.W, c.Wu, c.offsets, activation=kind, save=True)
    for a, b in zip(clean, dirty):
        for g in (0, 2, 4, 5):
            assert torch.equal(a[c.ends[g]:c.ends[g + 1]], b[c.ends[g]:c.ends[g + 1]])
        for g in (1, 3):
            assert not b[c.ends[g]:c.ends[g + 1]].isfinite().any()


@gpu
def test_more_than_2_31_elements_of_gradients():
    """Weights' gradients behind the 2^31-th element of dW, by group and by row."""
    for sizes, N, K in (([70, 0, 33, 201], 24000, 24008), ([130], 46400, 46408)):
        E, R, t = len(sizes), sum(sizes), torch.bfloat16
        g = torch.Generator(device="cuda").manual_seed(5)
        X, dY = torch.randn(R, K, generator=g, device="cuda").to(t), torch.randn(R, N, generator=g, device="cuda").to(t)
        ends = [0] + torch.tensor(sizes).cumsum(0).tolist()
        dW = torch.full((E, N, K), 7.0, dtype=t, device="cuda")
        binding.onnx_grouped_gemm_backward(dY, X, None, torch.tensor(ends, dtype=torch.int32, device="cuda"), wanted=(False, True), dW=dW)
        for e in range(E):
            x, d = X[ends[e]:ends[e + 1]].double(), dY[ends[e]:ends[e + 1]].double()
            for n in (slice(0, 300), slice(N // 2, N // 2 + 300), slice(N - 300, N)):
                close(dW[e, n], d[:, n].T @ x, d[:, n].abs().T @ x.abs(), max(sizes), t)
        del dW


@gpu
def test_planes_of_more_than_2_31_elements(monkeypatch):
    """Parts of the sums behind the 2^31-th element of their planes: of the weights' gradients, and of results by row."""
    t = torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(6)
    monkeypatch.setenv("ONNXB_GROUPED_PARTS", "1,4")
    N, K, sizes = 16000, 17000, [300, 210]
    X, dY = torch.randn(510, K, generator=g, device="cuda").to(t), torch.randn(510, N, generator=g, device="cuda").to(t)
    dW = torch.full((2, N, K), 7.0, dtype=t, device="cuda")
    binding.onnx_grouped_gemm_backward(dY, X, None, torch.tensor([0, 300, 510], dtype=torch.int32, device="cuda"), wanted=(False, True), dW=dW)
    for e, rows in enumerate((slice(0, 300), slice(300, 510))):
        x, d = X[rows].double(), dY[rows].double()
        for n in (slice(0, 300), slice(N // 2, N // 2 + 300), slice(N - 300, N)):
            close(dW[e, n], d[:, n].T @ x, d[:, n].abs().T @ x.abs(), 300, t)
    del dW
    monkeypatch.setenv("ONNXB_GROUPED_PARTS", "4")
    R, K, N = 40000, 320, 13600
    X, W = torch.randn(R, K, generator=g, device="cuda").to(t), (torch.randn(2, N, K, generator=g, device="cuda") / math.sqrt(K)).to(t)
    offsets = torch.tensor([0, 20000, R], dtype=torch.int32, device="cuda")
    Y = binding.onnx_grouped_gemm(X, W, offsets)
    H, G, Up = binding.onnx_grouped_gated(X, W, W, offsets, save=True)
    for first, e in ((0, 0), (20000, 1), (R - 100, 1)):
        c = Case([100], K, N, t)
        c.X, c.W, c.Wu = X[first:first + 100], W[e:e + 1], W[e:e + 1]
        check_gemm(c, Y[first:first + 100])
        check_gated(c, *(v[first:first + 100] for v in (H, G, Up)), "silu")


@gpu
def test_the_same_bit_by_bit_from_call_to_call():
    """Which CTA has which tile goes by no order; the results do not depend on it."""
    for sizes, K, N, t in (([700, 0, 33, 1, 300, 512], 520, 1000, torch.bfloat16), ([3000], 192, 2000, torch.float16), ([2, 0, 5], 1032, 600, torch.bfloat16)):
        c = Case(sizes, K, N, t, seed=3)

        def calls():
            return [binding.onnx_grouped_gemm(c.X, c.W, c.offsets), *binding.onnx_grouped_gated(c.X, c.W, c.Wu, c.offsets, save=True),
                    *binding.onnx_grouped_gemm_backward(c.dY, c.X, c.W, c.offsets),
                    *binding.onnx_grouped_gated_backward(c.dY, c.X, c.W, c.Wu, c.G, c.U, c.offsets)]

        first = calls()
        for _ in range(20):
            assert all(torch.equal(a, b) for a, b in zip(first, calls()))
