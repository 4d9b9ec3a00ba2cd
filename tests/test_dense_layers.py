"""Dense layers of 8- and 16-bit operands (row quantisation, 8-bit Gemm, the gated block and its gradients) against their definitions
in 64 bits, through the binding; tolerances in dense_reference.py."""
import math

import pytest
import torch

import dense_reference as ref
from paper_2008_08272_b200 import binding

pytestmark = pytest.mark.gpu
HALVES = (torch.bfloat16, torch.float16)
FLOATS = (torch.float32,) + HALVES
# (tokens, width, channels): single tokens, the borders of tiles (8, 16, 32, 64, 128, 256), odd sizes, one of everything
SIZES = [(1, 1, 1), (1, 16, 8), (1, 64, 16), (1, 100, 33), (1, 4096, 48), (2, 257, 31), (5, 31, 300), (7, 520, 96), (8, 512, 64), (9, 1000, 130),
         (16, 128, 257), (17, 96, 128), (31, 72, 40), (33, 48, 65), (64, 1024, 64), (65, 200, 129), (100, 8, 500), (127, 130, 127), (128, 64, 128),
         (129, 65, 256), (200, 640, 264), (256, 256, 512), (257, 136, 513), (300, 1032, 200), (512, 128, 1024), (700, 333, 1111)]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *size):
    return torch.randn(*size, generator=g, device="cuda")


def pitched(x, extra, offset=0, fill=None):
    """x with rows `extra` elements further apart than they are long, the first `offset` elements into its storage; NaN (or 99) between."""
    rows, cols = x.shape
    fill = fill if fill is not None else 99 if x.dtype == torch.int8 else math.nan
    store = torch.full((offset + rows * (cols + extra),), fill, dtype=x.dtype, device=x.device)
    view = store[offset:].view(rows, cols + extra)[:, :cols]
    view.copy_(x)
    return view


def codes(g, rows, cols):
    """8-bit integers of every value, -128 among them."""
    return torch.randint(-128, 128, (rows, cols), generator=g, device="cuda", dtype=torch.int8)


def same(a, b):
    """Equal value by value, a NaN where the other has one."""
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0))


def done():
    torch.cuda.synchronize()
    assert binding.last_device_status() == 0


# --------------------------------------------------------------------- quantising
@pytest.mark.parametrize("t", FLOATS, ids=str)
@pytest.mark.parametrize("size", [(1, 1), (1, 7), (1, 4096), (3, 16), (5, 33), (4, 1000), (9, 255), (2, 8192), (3, 12289), (2, 70000), (300, 64), (1000, 129)])
def test_quantize_rows(t, size):
    g = gen(1)
    X = (normal(g, *size) * torch.exp(3 * normal(g, size[0], 1))).to(t)
    Q, scale = binding.onnx_quantize_rows(X)
    done()
    q, s = ref.quantize_rows(X)
    assert Q.shape == X.shape and (Q.stride(0) % 16 == 0 or size[0] == 1)
    assert same(scale, s) and torch.equal(Q, q)


def test_quantize_rows_next_to_halves():
    """Quotients at and right next to k + 1/2: the product with an inverse would round some of them the wrong way."""
    k = torch.arange(-126, 127, device="cuda", dtype=torch.float64) + 0.5
    rows = []
    for top in (127.0, 126.99999, 1.0, 3.3, 1e-30, 1e-41, 1e-44, 2e38, 1.7e-38):
        s = float(torch.tensor(top, dtype=torch.float64).float().double() / 127)
        s = float(torch.tensor(s, dtype=torch.float64).float())
        at = (k * s).float()
        inf = torch.tensor(math.inf, device="cuda")
        row = torch.cat([at, torch.nextafter(at, inf), torch.nextafter(at, -inf), torch.tensor([top], device="cuda", dtype=torch.float32)])
        rows.append(row)
    X = torch.stack(rows)
    Q, scale = binding.onnx_quantize_rows(X)
    done()
    q, s = ref.quantize_rows(X)
    assert same(scale, s) and torch.equal(Q, q)


def test_quantize_rows_without_a_scale():
    """Rows of zeros; rows with a NaN or an infinity, wherever it stands; the largest and smallest numbers."""
    X = normal(gen(2), 9, 300)
    X[0] = 0
    X[1, 5] = math.nan
    X[2, 299] = math.inf
    X[3, 0] = -math.inf
    X[4] = 0
    X[4, 7] = 1e-45
    X[5, 3] = torch.finfo(torch.float32).max
    X[6] = -0.0
    X[7, 100], X[7, 200] = math.nan, -math.inf
    Q, scale = binding.onnx_quantize_rows(X)
    done()
    q, s = ref.quantize_rows(X)
    assert torch.equal(Q, q) and same(scale, s)
    assert scale.isnan().tolist() == [False, True, True, True, False, False, False, True, False]


@pytest.mark.parametrize("t", FLOATS, ids=str)
@pytest.mark.parametrize("extra,offset", [(8, 0), (3, 0), (5, 1), (0, 3)])
def test_quantize_rows_strides(t, extra, offset):
    """Rows anywhere, of X and of Q; what lies between them stays as it was."""
    X = normal(gen(3), 37, 203).to(t)
    store = torch.full((offset + 37 * (203 + extra),), 55, dtype=torch.int8, device="cuda")
    Qv = store[offset:].view(37, 203 + extra)[:, :203]
    Q, scale = binding.onnx_quantize_rows(pitched(X, extra, offset), Q=Qv)
    done()
    q, s = ref.quantize_rows(X)
    assert Q is Qv and torch.equal(Q, q) and torch.equal(scale, s)
    assert bool((store[:offset] == 55).all()) and bool((store[offset:].view(37, 203 + extra)[:, 203:] == 55).all())


# --------------------------------------------------------------------- 8-bit Gemm
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("form", range(4))
def test_gemm_int8(size, form):
    M, K, N = size
    g = gen(4)
    t = FLOATS[form % 3]
    A, B = codes(g, M, K), codes(g, N, K)
    if form % 2:            # rows at multiples of 16 bytes, other values between them
        A, B = pitched(A, -K % 16), pitched(B, -K % 16 + 16)
    sa, sb = torch.exp(normal(g, M)) / 1000, torch.exp(normal(g, N)) / 127
    C = normal(g, N) if form >= 2 else None
    Y = binding.onnx_gemm_int8(A, sa, B, sb, C, fuse_relu=form == 3, dtype=t)
    done()
    assert Y.dtype == t
    assert ref.worst(Y, ref.gemm_int8(A, sa, B, sb, C, form == 3, t)) <= 1


@pytest.mark.parametrize("M", [1, 20, 150])
def test_gemm_int8_longest_sums(M):
    """The longest reduction, of the integers furthest from 0: the sum is next to 2^31."""
    K = 131071
    A = torch.full((M, K), -128, dtype=torch.int8, device="cuda")
    B = torch.full((40, K), -128, dtype=torch.int8, device="cuda")
    B[1::2] = 127
    one = torch.ones(150, device="cuda")
    Y = binding.onnx_gemm_int8(A, one[:M], B, one[:40])
    done()
    assert ref.worst(Y, ref.gemm_int8(A, one[:M], B, one[:40], None, False, torch.float32)) <= 1


def test_gemm_int8_scales_without_bounds():
    """A NaN scale makes its row NaN and no other; scales whose product is infinite leave a sum of 0 a 0; relu of NaN is 0."""
    g = gen(5)
    for M in (3, 40, 300):
        A, B = codes(g, M, 64), codes(g, 50, 64)
        A[2] = 0
        sa, sb = torch.ones(M, device="cuda"), torch.full((50,), 1e30, device="cuda")
        sa[1], sa[2] = math.nan, 1e30
        Y = binding.onnx_gemm_int8(A, sa, B, sb)
        Z = binding.onnx_gemm_int8(A, sa, B, sb, fuse_relu=True)
        done()
        assert bool(Y[1].isnan().all()) and bool((Y[2] == 0).all()) and bool(Y[3:].isfinite().all()) and bool((Z[1] == 0).all())


# --------------------------------------------------------------------- the gated block
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("form", range(4))
def test_gated(size, form):
    M, K, F = size
    g = gen(6)
    t, kind = HALVES[form % 2], ref.KINDS[(form + M) % 4]
    X, Wg, Wu = normal(g, M, K).to(t), (normal(g, F, K) * 2 / math.sqrt(K)).to(t), (normal(g, F, K) / math.sqrt(K)).to(t)
    want = ref.gated(X, Wg, Wu, kind)
    if form >= 2:
        X, Wg, Wu = pitched(X, -K % 8 + 8), pitched(Wg, -K % 8), pitched(Wu, -K % 8 + 16)
        got = binding.onnx_gated(X, Wg, Wu, activation=kind, save=True)
    else:
        got = (binding.onnx_gated(X, Wg, Wu, activation=kind),)
    done()
    for y, pair in zip(got, want):
        assert ref.worst(y, pair) <= 1


@pytest.mark.parametrize("kind", ref.KINDS)
@pytest.mark.parametrize("M", [2, 140])
def test_gated_activations_over_their_range(kind, M):
    """Gates from -60 to 60, where exponentials run over and quotients vanish, and zeros."""
    t = torch.float16
    Wg = torch.linspace(-60, 60, 241, device="cuda")[:, None].to(t)
    X, Wu = torch.ones(M, 1, device="cuda", dtype=t), torch.full((241, 1), 3.0, device="cuda", dtype=t)
    got = binding.onnx_gated(X, Wg, Wu, activation=kind, save=True)
    done()
    for y, pair in zip(got, ref.gated(X, Wg, Wu, kind)):
        assert ref.worst(y, pair) <= 1


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("form", range(3))
def test_gated_int8(size, form):
    M, K, F = size
    g = gen(7)
    t, kind = FLOATS[form], ref.KINDS[(form + M) % 4]
    A, Wg, Wu = codes(g, M, K), codes(g, F, K), codes(g, F, K)
    if form:
        A, Wg, Wu = pitched(A, -K % 16), pitched(Wg, -K % 16 + 32), pitched(Wu, -K % 16)
    sa, sg, su = torch.exp(normal(g, M)) / 75, torch.exp(normal(g, F)) / 75 / math.sqrt(K), torch.exp(normal(g, F)) / 75 / math.sqrt(K)
    H = binding.onnx_gated_int8(A, sa, Wg, sg, Wu, su, activation=kind, dtype=t)
    done()
    assert ref.worst(H, ref.gated_int8(A, sa, Wg, sg, Wu, su, kind, t)) <= 1


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("form", range(2))
def test_gated_backward(size, form):
    M, K, F = size
    g = gen(8)
    t, kind = HALVES[form], ref.KINDS[(form + M) % 4]
    dH, X, Wg, Wu = normal(g, M, F).to(t), normal(g, M, K).to(t), (normal(g, F, K) / math.sqrt(K)).to(t), (normal(g, F, K) / math.sqrt(K)).to(t)
    G, U = (2 * normal(g, M, F)).to(t), normal(g, M, F).to(t)
    want = ref.gated_backward(dH, X, Wg, Wu, G, U, kind)
    if form:
        X, Wg, Wu, dH, G, U = pitched(X, -K % 8), pitched(Wg, -K % 8 + 8), pitched(Wu, -K % 8), pitched(dH, 3), pitched(G, -F % 8), pitched(U, 5, 1)
    got = binding.onnx_gated_backward(dH, X, Wg, Wu, G, U, activation=kind)
    done()
    for y, pair in zip(got, want):
        assert ref.worst(y, pair) <= 1


@pytest.mark.parametrize("kind", ref.KINDS)
def test_gated_backward_slopes_over_their_range(kind):
    """Gates from the type's lowest to its largest value: slopes 0 and 1 there, and no NaN."""
    t = torch.bfloat16
    G = torch.cat([torch.linspace(-60, 60, 480, device="cuda"), torch.tensor([-3e38, -1e20, -1e19, -1e10, 0.0, -0.0, 1e10, 1e19, 1e20, 3e38], device="cuda")])
    G = G[:, None].to(t)
    U = torch.full_like(G, 2.0)
    U[480:] = 1e-38
    dH = torch.ones_like(G)
    eye = torch.ones(1, 1, device="cuda", dtype=t)
    dX = binding.onnx_gated_backward(dH, None, eye, eye * 0, G, U, activation=kind, wanted=(True, False, False))[0]
    done()
    value, slope = ref.act(kind, G.double())
    slope = torch.where(G.double().abs() > 1e9, (G > 0).double(), slope)
    dg = U.double() * slope
    off = ref.SLOPE * U.double().abs() + 2.0 ** -7 * dg.abs() + 1e-40
    assert ref.worst(dX, (dg, off)) <= 1


# --------------------------------------------------------------------- strides, places, sizes
@pytest.mark.parametrize("M", [1, 5, 90, 260])
@pytest.mark.parametrize("extra,offset", [(1, 0), (0, 1), (7, 3), (8, 8)])
def test_strides_and_places(M, extra, offset):
    """Rows that begin anywhere, of inputs and outputs; outputs leave what lies between and behind them as it was."""
    g = gen(9)
    K, F, t = 150, 77, torch.bfloat16

    def out(rows, cols, dtype):
        store = torch.full((offset + rows * (cols + extra) + 16,), 44, dtype=dtype, device="cuda")
        view = store[offset:offset + rows * (cols + extra)].view(rows, cols + extra)
        return store, view[:, :cols], view[:, cols:]

    def kept(store, between):
        return bool((store[:offset] == 44).all()) and bool((store[-16:] == 44).all()) and bool((between == 44).all())

    X, Wg, Wu = normal(g, M, K).to(t), (normal(g, F, K) / 12).to(t), (normal(g, F, K) / 12).to(t)
    outs = [out(M, F, t) for _ in range(3)]
    binding.onnx_gated(pitched(X, extra, offset), pitched(Wg, extra, offset), pitched(Wu, extra, offset), H=outs[0][1], G=outs[1][1], U=outs[2][1])
    done()
    for (store, y, between), pair in zip(outs, ref.gated(X, Wg, Wu, "silu")):
        assert ref.worst(y, pair) <= 1 and kept(store, between)

    A, B, Bu = codes(g, M, K), codes(g, F, K), codes(g, F, K)
    sa, sb, su = torch.rand(M, device="cuda", generator=g) / 500, torch.rand(F, device="cuda", generator=g) / 500, torch.rand(F, device="cuda", generator=g)
    for y_type in FLOATS:
        store, y, between = out(M, F, y_type)
        binding.onnx_gemm_int8(pitched(A, extra, offset), sa, pitched(B, extra, offset), sb, Y=y)
        done()
        assert ref.worst(y, ref.gemm_int8(A, sa, B, sb, None, False, y_type)) <= 1 and kept(store, between)
        store, y, between = out(M, F, y_type)
        binding.onnx_gated_int8(pitched(A, extra, offset), sa, pitched(B, extra, offset), sb, pitched(Bu, extra, offset), su, activation="gelu", H=y)
        done()
        assert ref.worst(y, ref.gated_int8(A, sa, B, sb, Bu, su, "gelu", y_type)) <= 1 and kept(store, between)

    dH, G, U = normal(g, M, F).to(t), normal(g, M, F).to(t), normal(g, M, F).to(t)
    outs = [out(M, K, t), out(F, K, t), out(F, K, t)]
    binding.onnx_gated_backward(*(pitched(v, extra, offset) for v in (dH, X, Wg, Wu, G, U)), activation="gelu", dX=outs[0][1], dWg=outs[1][1], dWu=outs[2][1])
    done()
    for (store, y, between), pair in zip(outs, ref.gated_backward(dH, X, Wg, Wu, G, U, "gelu")):
        assert ref.worst(y, pair) <= 1 and kept(store, between)


@pytest.mark.parametrize("M", [3, 200])
def test_weights_and_projections_in_one_tensor(M):
    """Both weights as halves of one tensor, both projections as halves of one: rows of one lie between those of the other."""
    g = gen(10)
    K, F, t = 128, 192, torch.bfloat16
    X, W = normal(g, M, K).to(t), (normal(g, 2 * F, K) / 11).to(t)
    GU = torch.empty(M, 2 * F, dtype=t, device="cuda")
    H, G, U = binding.onnx_gated(X, W[:F], W[F:], G=GU[:, :F], U=GU[:, F:])
    done()
    for y, pair in zip((H, GU[:, :F], GU[:, F:]), ref.gated(X, W[:F], W[F:], "silu")):
        assert ref.worst(y, pair) <= 1
    dH, dW = normal(g, M, F).to(t), torch.empty(2 * F, K, dtype=t, device="cuda")
    dX = binding.onnx_gated_backward(dH, X, W[:F], W[F:], G, U, dWg=dW[:F], dWu=dW[F:])[0]
    done()
    for y, pair in zip((dX, dW[:F], dW[F:]), ref.gated_backward(dH, X, W[:F], W[F:], G, U, "silu")):
        assert ref.worst(y, pair) <= 1


def test_no_tokens():
    t, e = torch.bfloat16, lambda *s: torch.empty(*s, device="cuda")
    Q, scale = binding.onnx_quantize_rows(e(0, 40))
    assert Q.shape == (0, 40) and scale.shape == (0,)
    W, s = torch.ones(24, 40, dtype=torch.int8, device="cuda"), torch.ones(24, device="cuda")
    assert binding.onnx_gemm_int8(Q, scale, W, s).shape == (0, 24)
    assert binding.onnx_gated_int8(Q, scale, W, s, W.clone(), s).shape == (0, 24)
    X, Wg, Wu = e(0, 40).to(t), e(24, 40).to(t), e(24, 40).to(t)
    H, G, U = binding.onnx_gated(X, Wg, Wu, save=True)
    assert H.shape == G.shape == U.shape == (0, 24)
    dW = torch.full((24, 45), 7.0, dtype=t, device="cuda")
    dX, dWg, dWu = binding.onnx_gated_backward(H, X, Wg, Wu, G, U, dWu=dW[:, :40])
    done()
    assert dX.shape == (0, 40) and bool((dWg == 0).all()) and bool((dWu == 0).all()) and bool((dW[:, 40:] == 7).all())


@pytest.mark.parametrize("wanted", [(True, False, False), (False, True, False), (False, False, True), (True, False, True), (False, True, True)], ids=str)
def test_gradients_one_by_one(wanted):
    """What is not wanted is not computed, its inputs may be left out, and the others are the same bit by bit."""
    g = gen(11)
    t, M, K, F = torch.float16, 70, 96, 130
    dH, X, Wg, Wu, G, U = normal(g, M, F).to(t), normal(g, M, K).to(t), normal(g, F, K).to(t), normal(g, F, K).to(t), normal(g, M, F).to(t), normal(g, M, F).to(t)
    every = binding.onnx_gated_backward(dH, X, Wg, Wu, G, U)
    some = binding.onnx_gated_backward(dH, X if wanted[1] or wanted[2] else None, Wg if wanted[0] else None, Wu if wanted[0] else None, G, U, wanted=wanted)
    done()
    for w, a, b in zip(wanted, some, every):
        assert (a is None) == (not w) and (a is None or torch.equal(a, b))


def test_elements_past_32_bits():
    """Views whose last elements lie more than 2^31 elements, and 2^32 bytes, behind their first."""
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("too little memory")
    g = gen(12)
    M, K, ld = 70000, 64, 35000
    store = torch.zeros(M * ld, dtype=torch.bfloat16, device="cuda")         # 2.45e9 elements
    X = store.view(M, ld)[:, :K]
    X.copy_(normal(g, M, K))
    Wg, Wu = (normal(g, 40, K) / 8).bfloat16(), (normal(g, 40, K) / 8).bfloat16()
    H = store.view(M, ld)[:, 1000:1040]
    binding.onnx_gated(X, Wg, Wu, H=H)
    Q = torch.empty(M, ld, dtype=torch.int8, device="cuda")[:, :K]
    Q, scale = binding.onnx_quantize_rows(X, Q=Q)
    dWg = binding.onnx_gated_backward(H, X, None, None, H, H, wanted=(False, True, False))[1]
    done()
    q, s = ref.quantize_rows(X)
    assert torch.equal(Q, q) and torch.equal(scale, s)
    assert ref.worst(H, ref.gated(X, Wg, Wu, "silu")[0]) <= 1
    assert ref.worst(dWg, ref.gated_backward(H, X, Wg, Wu, H, H, "silu")[1]) <= 1
    Y = binding.onnx_gemm_int8(Q, scale, Q[-60:], scale[-60:])
    done()
    assert ref.worst(Y, ref.gemm_int8(Q, scale, Q[-60:], scale[-60:], None, False, torch.float32)) <= 1


# --------------------------------------------------------------------- as they are used
@pytest.mark.parametrize("M", [1, 6, 31, 200])
def test_feed_forward_in_8_bits(M):
    """Weights quantised once; activations quantised, gated block, quantised again, down projection: each step on what the one before
    gave, and the whole against the layer in 64 bits."""
    g = gen(13)
    K, F, t = 264, 520, torch.bfloat16
    X = normal(g, M, K).to(t)
    weights = [normal(g, F, K) / math.sqrt(K), normal(g, F, K) / math.sqrt(K), normal(g, K, F) / math.sqrt(F)]
    (Wg, sg), (Wu, su), (Wd, sd) = (binding.onnx_quantize_rows(w) for w in weights)
    A, sa = binding.onnx_quantize_rows(X)
    H = binding.onnx_gated_int8(A, sa, Wg, sg, Wu, su, dtype=t)
    B, sb = binding.onnx_quantize_rows(H)
    Y = binding.onnx_gemm_int8(B, sb, Wd, sd, dtype=t)
    done()
    for x, (q, s) in ((X, (A, sa)), (H, (B, sb)), (weights[2], (Wd, sd))):
        want = ref.quantize_rows(x)
        assert torch.equal(q, want[0]) and torch.equal(s, want[1])
    assert ref.worst(H, ref.gated_int8(A, sa, Wg, sg, Wu, su, "silu", t)) <= 1
    assert ref.worst(Y, ref.gemm_int8(B, sb, Wd, sd, None, False, t)) <= 1
    g64, u64 = X.double() @ weights[0].double().T, X.double() @ weights[1].double().T
    whole = (ref.act("silu", g64)[0] * u64) @ weights[2].double().T
    # a step of 1/127 of a row's largest value, about 3.5 of its spread, is off by 0.3 of that step on average: 0.8 % of each factor,
    # and five factors are rounded so between X and Y
    assert float((Y.double() - whole).norm() / whole.norm()) < 0.03


@pytest.mark.parametrize("t", HALVES, ids=str)
def test_gated_forward_then_backward(t):
    """The gradients of a training step: G and U as the forward call leaves them."""
    g = gen(14)
    M, K, F = 150, 136, 200
    X, Wg, Wu, dH = normal(g, M, K).to(t), (normal(g, F, K) / 12).to(t), (normal(g, F, K) / 12).to(t), normal(g, M, F).to(t)
    H, G, U = binding.onnx_gated(X, Wg, Wu, activation="gelu", save=True)
    got = binding.onnx_gated_backward(dH, X, Wg, Wu, G, U, activation="gelu")
    done()
    for y, pair in zip(got, ref.gated_backward(dH, X, Wg, Wu, G, U, "gelu")):
        assert ref.worst(y, pair) <= 1


def _calls(M, seed):
    """Every operator on inputs of its own, as (function, outputs' references)."""
    g = gen(seed)
    K, F, t = 200, 144, torch.bfloat16
    X, Wg, Wu, dH = normal(g, M, K).to(t), (normal(g, F, K) / 14).to(t), (normal(g, F, K) / 14).to(t), normal(g, M, F).to(t)
    A, B = codes(g, M, K + 3)[:, :K], codes(g, F, K)
    sa, sb = torch.rand(M, device="cuda", generator=g) / 99, torch.rand(F, device="cuda", generator=g) / 99
    G, U = normal(g, M, F).to(t), normal(g, M, F).to(t)
    return [lambda **k: binding.onnx_quantize_rows(X, **k), lambda **k: binding.onnx_gemm_int8(A, sa, B, sb, **k),
            lambda **k: binding.onnx_gated(X, Wg, Wu, save=True, **k), lambda **k: binding.onnx_gated_int8(A, sa, B, sb, B, sa[:1].expand(F).contiguous(), **k),
            lambda **k: binding.onnx_gated_backward(dH, X, Wg, Wu, G, U, **k)]


def _flat(outs):
    return [o for o in (outs if isinstance(outs, tuple) else (outs,))]


@pytest.mark.parametrize("M", [1, 12, 40, 300])
def test_another_stream_and_a_graph(M):
    """On a stream that is not the current one, and captured and replayed on inputs that have changed: the same results bit by bit."""
    for call in _calls(M, 15):
        want = _flat(call())
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = _flat(call(stream=side))
        torch.cuda.current_stream().wait_stream(side)
        done()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            kept = _flat(call())
        for o in kept:
            o.fill_(3)
        graph.replay()
        done()
        assert all(torch.equal(a, b) for a, b in zip(kept, want))


def test_two_graphs_side_by_side():
    """Two captured graphs, replayed on two streams at once: neither's workspace is the other's."""
    jobs = []
    for seed in (16, 17):
        calls = _calls(257, seed)
        want = [_flat(c()) for c in calls]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            kept = [_flat(c()) for c in calls]
        jobs.append((graph, kept, want, torch.cuda.Stream(), calls))           # (the calls hold their inputs)
    torch.cuda.synchronize()
    for _ in range(5):
        for graph, _, _, stream, _ in jobs:
            with torch.cuda.stream(stream):
                graph.replay()
    done()
    for _, kept, want, _, _ in jobs:
        assert all(torch.equal(a, b) for x, y in zip(kept, want) for a, b in zip(x, y))


def test_back_to_back_without_waiting():
    """A chain of calls that read what the one before wrote, against the same chain with a wait after each."""
    g = gen(18)
    t = torch.bfloat16
    W = [(normal(g, 256, 256) / 16).to(t) for _ in range(4)]
    QW = [binding.onnx_quantize_rows(w) for w in W]

    def chain(M, wait):
        x, out = normal(gen(19), M, 256).to(t), []
        for i in range(6):
            h = binding.onnx_gated(x, W[i % 4], W[(i + 1) % 4])
            wait()
            q, s = binding.onnx_quantize_rows(h)
            wait()
            y = binding.onnx_gemm_int8(q, s, *QW[i % 4], dtype=t)
            wait()
            q, s = binding.onnx_quantize_rows(y)
            wait()
            x = binding.onnx_gated_int8(q, s, *QW[i % 4], *QW[(i + 2) % 4], dtype=t)
            wait()
            dx, dw, _ = binding.onnx_gated_backward(x, y, W[0], W[1], h, y)
            wait()
            x = (x + dx) + dw[:1]
            x = (x / x.float().abs().amax().clamp(min=1e-3)).to(t)
            out += [h, y, x, dx, dw]
        return out

    for M in (1, 10, 300):
        for a, b in zip(chain(M, lambda: None), chain(M, torch.cuda.synchronize)):
            assert torch.equal(a, b)
    done()
