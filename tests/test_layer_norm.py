"""Layer normalisation and its gradients against their definition in 64 bits, element by element."""
import pytest
import torch

from paper_2008_08272_b200 import binding

TYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
U = 2.0 ** -24                               # half a step of a 32-bit float
gpu = pytest.mark.gpu


def half_step(t):
    return torch.finfo(t).eps / 2


def smallest(t):                             # half of the smallest step that a type's numbers next to zero have
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2


def additions(K):
    """Roundings on the way of a term into a row's sum: at most 32 or K / 1024 in a thread, some in the tree, a few for the term and the result."""
    return max(32, K / 1024) + 24


def inputs(M, K, t, w, seed=0, far=0.0, bias=True):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    X = (torch.randn(M, K, generator=gen, device="cuda") * torch.exp(0.5 * torch.randn(K, generator=gen, device="cuda")) + far).to(t)
    scale = (1 + 0.3 * torch.randn(K, generator=gen, device="cuda")).to(w)
    B = torch.randn(K, generator=gen, device="cuda").to(w) if bias else None
    dY = torch.randn(M, K, generator=gen, device="cuda").to(t)
    return X, scale, B, dY


def definition(X, scale, B, epsilon):
    x = X.double()
    mean = x.mean(1, keepdim=True)
    inv_std = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + epsilon)
    n = (x - mean) * inv_std
    return n * scale.double() + (0 if B is None else B.double()), mean, inv_std, n


def check_forward(X, scale, B, epsilon, got):
    Y, m, r = got
    K, D = X.shape[1], additions(X.shape[1])
    y, mean, inv_std, n = definition(X, scale, B, epsilon)
    level = X.double().abs().mean(1, keepdim=True)
    # the mean is off by D roundings of the magnitudes' mean; a deviation by that and its own rounding; the variance, of squares of deviations, by 2 of
    # the former relative to the deviations, and D roundings of its own; inv_std by half of it
    off = U * (D * level + (X.double() - mean).abs() + mean.abs())
    rel = U * (D + 4) + inv_std * U * D * level
    s = scale.double().abs()
    tol = (off * inv_std + n.abs() * rel) * s + 3 * U * ((n * scale.double()).abs() + y.abs()) + half_step(Y.dtype) * y.abs() + smallest(Y.dtype)
    assert ((Y.double() - y).abs() <= 1.01 * tol).all(), float(((Y.double() - y).abs() / tol).max())
    if m is not None:
        assert ((m.double() - mean[:, 0]).abs() <= (U * (D * level + mean.abs()))[:, 0]).all()
        assert ((r.double() / inv_std[:, 0] - 1).abs() <= 1.01 * rel[:, 0] + U).all()


SIZES = [(1, 1), (3, 2), (1, 4096), (2, 777), (33, 40), (5, 8), (9, 250), (300, 512), (297, 1001), (64, 1024), (640, 4096), (301, 8192), (7, 12288), (3, 16384),
         (2, 25600), (2, 33000), (1, 70001), (2, 131072)]


@gpu
@pytest.mark.parametrize("M,K", SIZES)
@pytest.mark.parametrize("t,w", [("float32", "float32"), ("float16", "float16"), ("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float16", "float32")])
def test_forward(M, K, t, w):
    X, scale, B, _ = inputs(M, K, TYPES[t], TYPES[w], seed=M + K)
    got = binding.onnx_layer_normalization(X, scale, B, epsilon=1e-5, save=True)
    check_forward(X, scale, B, 1e-5, got)
    assert torch.equal(got[0], binding.onnx_layer_normalization(X, scale, B, epsilon=1e-5))
    no_bias = binding.onnx_layer_normalization(X, scale, epsilon=0.25)
    check_forward(X, scale, None, 0.25, (no_bias, None, None))


def check_backward(dY, X, scale, mean, inv_std, got):
    dX, dS, dB = got
    M, K = X.shape
    D = additions(K)
    g, r = dY.double(), inv_std.double()[:, None]
    n, d = (X.double() - mean.double()[:, None]) * r, dY.double() * scale.double()
    level, along = d.mean(1, keepdim=True), (d * n).mean(1, keepdim=True)
    dx = r * (d - level - n * along)
    if dX is not None:
        tol = U * r * (6 * d.abs() + D * d.abs().mean(1, keepdim=True) + (D + 8) * n.abs() * (d * n).abs().mean(1, keepdim=True)
                       + 6 * n.abs() * along.abs()) + half_step(dX.dtype) * dx.abs() + smallest(dX.dtype)
        assert ((dX.double() - dx).abs() <= 1.01 * tol).all(), float(((dX.double() - dx).abs() / tol).max())
    # columns' sums: at most one addition for each of a block's rows (148 blocks have rows where there are so many), for its warps and for the blocks
    adds = M / 64 + 64
    for got_sum, terms in ((dS, g * n), (dB, g)):
        if got_sum is None:
            continue
        want = terms.sum(0)
        tol = U * (adds + 4) * terms.abs().sum(0) + half_step(got_sum.dtype) * want.abs() + smallest(got_sum.dtype)
        assert ((got_sum.double() - want).abs() <= 1.01 * tol).all(), float(((got_sum.double() - want).abs() / tol).max())


@gpu
@pytest.mark.parametrize("M,K", SIZES + [(5000, 512), (2000, 4096), (1200, 20000)])
@pytest.mark.parametrize("t,w", [("float32", "float32"), ("float16", "float16"), ("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float16", "float32")])
def test_backward(M, K, t, w):
    X, scale, B, dY = inputs(M, K, TYPES[t], TYPES[w], seed=M + K)
    x = X.double()
    mean = x.mean(1).float()
    inv_std = (1 / torch.sqrt(x.var(1, unbiased=False) + 1e-5)).float()
    got = binding.onnx_layer_normalization_backward(dY, X, scale, mean, inv_std)
    assert got[0].dtype == X.dtype and got[1].dtype == got[2].dtype == scale.dtype
    check_backward(dY, X, scale, mean, inv_std, got)
    for wanted in ((True, False, False), (False, True, False), (False, False, True), (True, False, True)):
        some = binding.onnx_layer_normalization_backward(dY, X, scale, mean, inv_std, wanted=wanted)
        for want, one, all_of_them in zip(wanted, some, got):
            assert (one is None) == (not want)
            assert one is None or torch.equal(one, all_of_them)


@gpu
@pytest.mark.parametrize("far", [100.0, -5000.0])
def test_rows_far_from_zero(far):
    """The mean is taken away before the squares are added up."""
    X, scale, B, _ = inputs(50, 1000, torch.float32, torch.float32, far=far)
    check_forward(X, scale, B, 1e-5, binding.onnx_layer_normalization(X, scale, B, save=True))


@gpu
def test_gradients_against_differences():
    """The forward kernel's own results, a little to both sides, in 32 bits (steps of 2^-6: what is left of the third derivative is 2^-12 of its size,
    what the results' rounding makes of the quotient about 2^-24 * 2^6 * sqrt(MK))."""
    M, K = 3, 20
    X, scale, B, dY = inputs(M, K, torch.float32, torch.float32, seed=5)
    _, mean, inv_std = binding.onnx_layer_normalization(X, scale, B, save=True)
    dX, dS, dB = binding.onnx_layer_normalization_backward(dY, X, scale, mean, inv_std)

    def loss(x, s, b):
        return float((binding.onnx_layer_normalization(x, s, b).double() * dY.double()).sum())

    h = 2.0 ** -6
    for grad, which in ((dX, 0), (dS, 1), (dB, 2)):
        for i in range(0, grad.numel(), 3):
            sides = []
            for sign in (1, -1):
                a = [X.clone(), scale.clone(), B.clone()]
                a[which].view(-1)[i] += sign * h
                sides.append(loss(*a))
            assert abs((sides[0] - sides[1]) / (2 * h) - float(grad.view(-1)[i])) < 2e-3 * (1 + float(dY.abs().max()) * float(inv_std.max()))


@gpu
@pytest.mark.parametrize("t", list(TYPES))
def test_views(t):
    """Rows that begin anywhere, with other values between them that are neither read nor written."""
    t = TYPES[t]
    for M, K, ld, at in ((20, 100, 107, 3), (5, 64, 72, 8), (400, 1000, 1001, 0)):
        X, scale, B, dY = inputs(M, K, t, t, seed=ld)

        def view(x, fill):
            store = torch.full((M * ld + at + ld,), fill, dtype=t, device="cuda")
            v = store[at:at + M * ld].view(M, ld)[:, :K]
            if x is not None:
                v.copy_(x)
            return store, v

        xs, xv = view(X, float("nan"))
        gs, gv = view(dY, float("nan"))
        ys, yv = view(None, 7.0)
        ds, dv = view(None, 7.0)
        odd = torch.empty(K + 1, dtype=t, device="cuda")[1:]
        odd.copy_(scale)
        Y, m, r = binding.onnx_layer_normalization(xv, odd, B, save=True, Y=yv)
        check_forward(X, scale, B, 1e-5, (Y, m, r))
        got = binding.onnx_layer_normalization_backward(gv, xv, odd, m, r, dX=dv)
        check_backward(dY, X, scale, m, r, got)
        for store, v in ((ys, yv), (ds, dv)):
            v.fill_(7.0)
            assert (store == 7.0).all()


@gpu
def test_rows_without_numbers():
    """A row of one value, of infinities or with a NaN: what the formula gives, and nothing of it in other rows."""
    X, scale, B, dY = inputs(6, 300, torch.float32, torch.float32)
    X[1] = 2.5
    X[2, 7] = float("nan")
    X[4, 0] = float("inf")
    Y, m, r = binding.onnx_layer_normalization(X, scale, B, save=True)
    assert torch.equal(Y[1], B)
    assert Y[2].isnan().all() and Y[4].isnan().all() and Y[[0, 1, 3, 5]].isfinite().all()
    dX, dS, dB = binding.onnx_layer_normalization_backward(dY, X, scale, m, r)
    assert dX[[2, 4]].isnan().all() and dX[[0, 1, 3, 5]].isfinite().all() and dB.isfinite().all() and dS.isnan().all()


@gpu
def test_no_rows():
    X, scale, B, _ = inputs(1, 64, torch.float16, torch.float32)
    Y, m, r = binding.onnx_layer_normalization(X[:0], scale, B, save=True)
    assert Y.shape == (0, 64) and m.shape == r.shape == (0,)
    dX, dS, dB = binding.onnx_layer_normalization_backward(X[:0], X[:0], scale, m, r)
    assert dX.shape == (0, 64) and not dS.any() and not dB.any()


@gpu
def test_captured_and_replayed():
    """Graphs of the same calls with workspaces of their own, replayed on inputs that have changed, on two streams."""
    runs = []
    for seed in (1, 2):
        X, scale, B, dY = inputs(700, 2048, torch.bfloat16, torch.float32, seed=seed)
        ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            binding.onnx_layer_normalization(X, scale, B, save=True)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            Y, m, r = binding.onnx_layer_normalization(X, scale, B, save=True)
            got = binding.onnx_layer_normalization_backward(dY, X, scale, m, r, workspace=ws)
        runs.append((g, s, X, scale, B, dY, Y, m, r, got, ws))
    for g, s, X, scale, B, dY, *_ in runs:
        X.copy_(torch.randn_like(X))
        dY.copy_(torch.randn_like(dY))
    torch.cuda.synchronize()
    for g, s, *_ in runs:
        with torch.cuda.stream(s):
            g.replay()
    torch.cuda.synchronize()
    for g, s, X, scale, B, dY, Y, m, r, got, ws in runs:
        check_forward(X, scale, B, 1e-5, (Y, m, r))
        check_backward(dY, X, scale, m, r, got)


@gpu
def test_on_another_stream():
    X, scale, B, dY = inputs(500, 1024, torch.float16, torch.float16)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    Y, m, r = binding.onnx_layer_normalization(X, scale, B, save=True, stream=s)
    got = binding.onnx_layer_normalization_backward(dY, X, scale, m, r, stream=s)
    s.synchronize()
    check_forward(X, scale, B, 1e-5, (Y, m, r))
    check_backward(dY, X, scale, m, r, got)


@gpu
def test_refusals():
    X, scale, B, dY = inputs(4, 64, torch.float16, torch.float32)
    norm, back = binding.onnx_layer_normalization, binding.onnx_layer_normalization_backward
    m, r = torch.zeros(4, device="cuda"), torch.ones(4, device="cuda")
    bad = [(TypeError, lambda: norm(X.double(), scale)), (TypeError, lambda: norm(X.cpu(), scale)), (TypeError, lambda: norm(X[0], scale)),
           (TypeError, lambda: norm(X.T, scale)), (TypeError, lambda: norm(X, scale.bfloat16())), (TypeError, lambda: norm(X, scale, B.half())),
           (TypeError, lambda: norm(X.float(), scale.half())), (TypeError, lambda: norm(X, scale[None])), (binding.OnnxB200Error, lambda: norm(X, None)),
           (binding.OnnxB200Error, lambda: norm(X, scale[:63])), (binding.OnnxB200Error, lambda: norm(X, scale, B[:1])),
           (binding.OnnxB200Error, lambda: norm(X, scale, epsilon=-1e-5)), (binding.OnnxB200Error, lambda: norm(X, scale, epsilon=float("nan"))),
           (binding.OnnxB200Error, lambda: norm(X, scale, Y=X)), (binding.OnnxB200Error, lambda: norm(X, scale, Y=X.new_empty(4, 65))),
           (TypeError, lambda: norm(X, scale, Y=X.float())), (binding.OnnxB200Error, lambda: norm(X, scale, mean=m, inv_std=m)),
           (binding.OnnxB200Error, lambda: norm(X, scale, mean=m[:3])), (TypeError, lambda: norm(X, scale, mean=m.half())),
           (binding.OnnxB200Error, lambda: back(dY, X, scale, m, r, wanted=(False,) * 3)), (ValueError, lambda: back(dY, X, scale, m, r, wanted=(True,))),
           (binding.OnnxB200Error, lambda: back(dY, X, None, m, r)), (binding.OnnxB200Error, lambda: back(dY, X, scale, None, r)),
           (binding.OnnxB200Error, lambda: back(dY[:3], X, scale, m, r)), (TypeError, lambda: back(dY.float(), X, scale, m, r)),
           (binding.OnnxB200Error, lambda: back(dY, X, scale, m, r, dX=X)), (binding.OnnxB200Error, lambda: back(dY, X, scale, m, r, dX=dY)),
           (binding.OnnxB200Error, lambda: back(dY, X, scale, m, r, dScale=scale)), (binding.OnnxB200Error, lambda: back(dY, X, scale, m, r, dScale=B, dB=B)),
           (TypeError, lambda: back(dY, X, scale, m, r, dScale=B.half())),
           (binding.OnnxB200Error, lambda: back(dY, X, scale, m, r, workspace=torch.empty(64, dtype=torch.uint8, device="cuda")))]
    for error, call in bad:
        with pytest.raises(error):
            call()
    # without scale dScale and dB are of X's type
    _, dS, dB = back(dY, X, None, m, r, wanted=(False, True, True))
    assert dS.dtype == dB.dtype == X.dtype
    check_backward(dY, X, scale, m, r, (None, dS, dB))


def test_no_cpu_path():
    with pytest.raises(TypeError):
        binding.onnx_layer_normalization(torch.zeros(2, 4), torch.ones(4))
    with pytest.raises(TypeError):
        binding.onnx_layer_normalization_backward(torch.zeros(2, 4), torch.zeros(2, 4), torch.ones(4), torch.zeros(2), torch.ones(2))


@gpu
def test_checked_path_gives_the_same(monkeypatch):
    X, scale, B, dY = inputs(70, 1000, torch.bfloat16, torch.float32)

    def calls():
        Y, m, r = binding.onnx_layer_normalization(X, scale, B, save=True)
        return [Y, m, r, binding.onnx_layer_normalization(X, scale), *binding.onnx_layer_normalization_backward(dY, X, scale, m, r)]

    native = calls()
    monkeypatch.setattr(binding, "_fast_mod", binding._Declined())
    for a, b in zip(native, calls()):
        assert a.dtype == b.dtype and torch.equal(a, b)


@gpu
def test_more_than_2_31_elements():
    """Rows behind the 2^31-th element, in a tensor whose other rows are zeros."""
    M, K = (1 << 20) + 3, 2056
    X = torch.zeros(M, K, dtype=torch.float16, device="cuda")
    dY = torch.zeros_like(X)
    x, scale, B, dy = inputs(5, K, torch.float16, torch.float32)
    X[-5:], dY[-5:] = x, dy
    Y, m, r = binding.onnx_layer_normalization(X, scale, B, save=True)
    check_forward(x, scale, B, 1e-5, (Y[-5:], m[-5:], r[-5:]))
    assert torch.equal(Y[:-5], B.to(torch.float16).expand(M - 5, K))
    del Y
    dX, dS, dB = binding.onnx_layer_normalization_backward(dY, X, scale, m, r)
    # (rows of zeros add nothing to the sums)
    check_backward(dy, x, scale, m[-5:], r[-5:], (dX[-5:], dS, dB))
    assert not dX[:-5].any()


@gpu
def test_two_streams_at_once():
    """Calls that overlap in time leave one another's results alone."""
    cases = [inputs(3000, 1024, torch.bfloat16, torch.float32, seed=1), inputs(500, 12288, torch.bfloat16, torch.float32, seed=2)]

    def run(case):
        X, scale, B, dY = case
        Y, m, r = binding.onnx_layer_normalization(X, scale, B, save=True)
        return [Y, *binding.onnx_layer_normalization_backward(dY, X, scale, m, r)]

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


@gpu
@pytest.mark.parametrize("M,K", [(3, 20), (2, 777), (5, 4096), (700, 1000), (640, 4096), (700, 1003), (3, 16384), (2, 25600), (2, 70001)])
@pytest.mark.parametrize("t,far", [("float32", 1e4), ("float32", -3e5), ("float16", 500.0), ("bfloat16", -60.0)])
def test_mean_far_from_zero(M, K, t, far):
    """The mean that is kept is off by its own rounding, and what is left of its error by roundings of the deviations alone, not of the mean."""
    X, scale, B, _ = inputs(M, K, TYPES[t], torch.float32, seed=M + K, far=far)
    Y, m, r = binding.onnx_layer_normalization(X, scale, B, save=True)
    y, mean, inv_std, n = definition(X, scale, B, 1e-5)
    D = additions(K)
    # the first mean is off by at most D roundings of the magnitudes' mean; deviations from it are rounded once and added up in D steps, and the mean of those is
    # rounded twice more
    first = U * D * X.double().abs().mean(1, keepdim=True)
    away = (X.double() - mean).abs()
    drift = U * (D + 3) * (away.mean(1, keepdim=True) + first)
    assert ((m.double() - mean[:, 0]).abs() <= 1.01 * (U * mean.abs() + drift)[:, 0]).all()
    # the variance: D roundings of the squares' sum, two of each square, and of what the first mean was off by, which is taken away again, as many; the deviations' sums
    # enter by their square; inv_std by half of it and its own
    rel = U * (D + 8) * (1 + (first * inv_std) ** 2) + (drift * inv_std) ** 2
    assert ((r.double() / inv_std[:, 0] - 1).abs() <= 1.01 * rel[:, 0]).all()
    s = scale.double().abs()
    tol = ((U * (away + first) + drift) * inv_std + n.abs() * rel) * s + 3 * U * ((n * scale.double()).abs() + y.abs()) + half_step(Y.dtype) * y.abs() + smallest(Y.dtype)
    assert ((Y.double() - y).abs() <= 1.01 * tol).all(), float(((Y.double() - y).abs() / tol).max())


@gpu
def test_squares_that_are_not_finite():
    """A row whose deviations have no square in 32 bits becomes the bias, however far from zero it is."""
    for K in (64, 1000, 4096, 70000):
        X = torch.full((2, K), 1e30, device="cuda")
        X[:, ::3] = -0.7e30
        scale, B = torch.ones(K, device="cuda"), torch.randn(K, device="cuda")
        Y, m, r = binding.onnx_layer_normalization(X, scale, B, save=True)
        assert torch.equal(Y, B.expand(2, K)) and not r.any() and m.isfinite().all()


@gpu
@pytest.mark.parametrize("M,K", [(3, 20), (2, 777), (5, 4096), (700, 1000), (640, 4096), (700, 1003), (3, 16384), (2, 25600), (2, 70001)])
@pytest.mark.parametrize("t", list(TYPES))
def test_mean_near_zero(M, K, t):
    """Rows of whole numbers, whose sums are exact in 32 bits: the mean is off by the rounding of 1 / K and its own alone."""
    gen = torch.Generator(device="cuda").manual_seed(K)
    X = torch.randint(-100, 101, (M, K), generator=gen, device="cuda").to(TYPES[t])
    scale = torch.ones(K, dtype=TYPES[t], device="cuda")
    _, m, _ = binding.onnx_layer_normalization(X, scale, save=True)
    mean = X.double().mean(1)
    assert ((m.double() - mean).abs() <= 2.01 * U * mean.abs()).all()
