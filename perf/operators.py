"""The operators of a language model's feed-forward layers, as measurable cases: 8-bit integer products for serving, and the gated
block (two projections, an activation and a product) in 16 bits, forward and backward, and in 8.

  quantize_rows   q[i,k] = nearest integer to x[i,k] / s[i], s[i] = max_k |x[i,k]| / 127 (kept as a 32-bit float)
  gemm_int8       y[i,j] = relu?( a_s[i] * b_s[j] * sum_k a[i,k] * b[j,k] + c[j] ), a and b 8-bit integers
  gated           g = X Wg^T, u = X Wu^T, h = act(g) * u; with "save" g and u are outputs too, for the backward pass
  gated_int8      the same of 8-bit integers with scales as in gemm_int8
  gated_backward  dg = dh * u * act'(g), du = dh * act(g); dX = dg Wg + du Wu, dWg = dg^T X, dWu = du^T X

A case is a dict of plain values.  tokens: rows of the activations; width: the reduction of the first product; channels: rows of
the weights (of each of the two, where there are two); type: of the activations and results (8-bit operands have their own);
padded: the rows of 8-bit operands begin at multiples of 16 bytes (as quantising leaves them) and not one right behind the other.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "fp16": 2, "bf16": 2}


def _case(name, op, tokens, width, channels=0, **kw):
    c = {"name": name, "op": op, "tokens": tokens, "width": width, "channels": channels, "type": "bf16"}
    if op in ("gemm_int8", "gated_int8"):
        c["padded"] = True
    if op == "gemm_int8":
        c.update(bias=False, relu=False)
    if op.startswith("gated"):
        c["activation"] = "silu"
    if op == "gated":
        c["save"] = False
    c.update(kw)
    return c


def listed():
    return [
        # One token's activations on the way into an 8-bit layer: the smallest call, where latency is all.
        _case("quantize_token", "quantize_rows", 1, 4096),
        # A long prompt's activations in 32 bits.
        _case("quantize_prompt_fp32", "quantize_rows", 8192, 4096, type="fp32"),
        # The down projection while answering: one token against all the weights, which have to be read.
        _case("gemm_int8_token", "gemm_int8", 1, 10240, 4096),
        # A dense layer whose sizes are no multiples of anything, rows right behind one another.
        _case("gemm_int8_ragged", "gemm_int8", 1001, 777, 1530, type="fp32", padded=False, bias=True, relu=True),
        # The down projection of a prompt.
        _case("gemm_int8_prompt", "gemm_int8", 4096, 10240, 4096),
        # The gated block while answering: one token.
        _case("gated_token", "gated", 1, 4096, 10240),
        # A short prompt through a small model of odd sizes.
        _case("gated_ragged_fp16", "gated", 333, 1000, 2741, type="fp16", activation="gelu_tanh"),
        # A training step's forward half: the two projections are kept.
        _case("gated_train", "gated", 4096, 4096, 10240, save=True),
        # Eight sequences answered together, in 8 bits.
        _case("gated_int8_batch", "gated_int8", 8, 4096, 10240),
        # A prompt in 8 bits.
        _case("gated_int8_prompt", "gated_int8", 4096, 4096, 10240),
        # A small model's training step, backward half.
        _case("gated_backward_small", "gated_backward", 512, 1024, 2816, type="fp16", activation="gelu"),
        # A large model's training step, backward half (the largest case).
        _case("gated_backward_train", "gated_backward", 4096, 4096, 10240),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _wide(rng, lo, hi):
    """Widths as models have them: mostly multiples of 64, sometimes any number."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.3 else max(64, (n + 32) // 64 * 64)


def draw(rng):
    """One more case of the ranges the listed ones stand for."""
    most = max(work(c)["flops"] for c in listed())
    while True:
        op = rng.choice(("quantize_rows", "gemm_int8", "gemm_int8", "gated", "gated", "gated_int8", "gated_backward"))
        tokens = rng.choice((1, rng.randint(2, 32), _log_int(rng, 1, 8192), _log_int(rng, 64, 8192)))
        c = _case("", op, tokens, _wide(rng, 32, 12288), 0 if op == "quantize_rows" else _wide(rng, 32, 12288))
        c["type"] = rng.choice(("bf16", "bf16", "fp16") if op in ("gated", "gated_backward") else ("bf16", "bf16", "fp16", "fp32"))
        if "padded" in c:
            c["padded"] = rng.random() < 0.7
        if "bias" in c:
            c["bias"], c["relu"] = rng.random() < 0.5, rng.random() < 0.3
        if "activation" in c:
            c["activation"] = rng.choice(("silu", "silu", "gelu", "gelu_tanh", "relu"))
        if "save" in c:
            c["save"] = rng.random() < 0.5
        need = work(c)
        if need["flops"] <= most and need["bytes"] >= 20000:
            del c["name"]
            return c


def work(case):
    M, K, N, b, op = case["tokens"], case["width"], case["channels"], BYTES[case["type"]], case["op"]
    if op == "quantize_rows":
        return {"bytes": M * K * (b + 1) + 4 * M, "flops": 3 * M * K}
    if op == "gemm_int8":
        return {"bytes": M * K + N * K + 4 * (M + N) + (4 * N if case["bias"] else 0) + M * N * b, "flops": 2 * M * N * K}
    if op == "gated":
        return {"bytes": b * (M * K + 2 * N * K + M * N * (3 if case["save"] else 1)), "flops": 4 * M * N * K}
    if op == "gated_int8":
        return {"bytes": M * K + 2 * N * K + 4 * (M + 2 * N) + M * N * b, "flops": 4 * M * N * K}
    # dh, g, u, X and both weights are read; dX and both weights' gradients are written
    return {"bytes": b * (3 * M * N + 2 * M * K + 4 * N * K), "flops": 8 * M * N * K}


# --------------------------------------------------------------------- inputs
def _device():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def _codes(x, padded):
    """8-bit integers and scales of the rows of x; padded: rows begin at multiples of 16 bytes, with other values in between."""
    rows, width = x.shape
    scale = x.abs().amax(1) / 127
    q = torch.clamp(torch.round(x / scale[:, None]), -127, 127).to(torch.int8)
    if padded and width % 16:
        store = torch.full((rows, (width + 15) // 16 * 16), 77, dtype=torch.int8, device=x.device)
        store[:, :width] = q
        q = store[:, :width]
    return q, scale


def _inputs(case, seed):
    dev, t = _device(), TYPES[case["type"]]
    gen = torch.Generator(device=dev).manual_seed(seed)
    M, K, N, op = case["tokens"], case["width"], case["channels"], case["op"]

    def normal(*size):
        return torch.randn(*size, generator=gen, device=dev, dtype=torch.float32)

    # activations: some channels are several times as large as others
    x = normal(M, K) * torch.exp(0.5 * normal(K))
    if op == "quantize_rows":
        return {"X": x.to(t)}
    if op in ("gemm_int8", "gated_int8"):
        s = {}
        s["A"], s["a_scale"] = _codes(x, case["padded"])
        for name in ("B",) if op == "gemm_int8" else ("Wg", "Wu"):
            s[name], s[name + "_scale"] = _codes(normal(N, K) / math.sqrt(K), case["padded"])
        if op == "gemm_int8":
            s["C"] = normal(N) if case["bias"] else None
        return s
    s = {"X": x.to(t), "Wg": (normal(N, K) / math.sqrt(K)).to(t), "Wu": (normal(N, K) / math.sqrt(K)).to(t)}
    if op == "gated_backward":
        s["dH"] = normal(M, N).to(t)
        s["G"] = (s["X"].float() @ s["Wg"].float().T).to(t)
        s["U"] = (s["X"].float() @ s["Wu"].float().T).to(t)
    return s


def prepare(case, seed):
    return {"case": dict(case), **_inputs(case, seed)}


# --------------------------------------------------------------------- one pass
def _activate(g, kind):
    if kind == "silu":
        return g / (1 + torch.exp(-g))
    if kind == "gelu":
        return 0.5 * g * (1 + torch.erf(g * math.sqrt(0.5)))
    if kind == "gelu_tanh":
        return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g * g * g)))
    return torch.where(g > 0, g, torch.zeros_like(g))


def _slope(g, kind):
    if kind == "silu":
        p = 1 / (1 + torch.exp(-g))
        return p * (1 + g * (1 - p))
    if kind == "gelu":
        return 0.5 * (1 + torch.erf(g * math.sqrt(0.5))) + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        th = torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g * g * g))
        return 0.5 * (1 + th) + 0.5 * g * (1 - th * th) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g * g)
    return (g > 0).to(g.dtype)


def run(state):
    return _own(state) if own else _plain(state)


def _plain(s):
    c, t = s["case"], TYPES[s["case"]["type"]]
    op = c["op"]
    if op == "quantize_rows":
        x = s["X"].float()
        # (64 bits: a quotient next to a half must not be rounded onto it, and a product with 1/127 is not always the quotient)
        scale = (x.abs().amax(1).double() / 127).float()
        q = torch.where(scale[:, None] > 0, torch.round(x.double() / scale.double()[:, None]), 0.0).clamp(-127, 127)
        return {"values": q.float() * scale[:, None], "scale": scale}
    if op in ("gemm_int8", "gated_int8"):
        a = s["A"].float()

        def product(name):
            return (a @ s[name].float().T) * s["a_scale"][:, None] * s[name + "_scale"][None, :]

        if op == "gated_int8":
            return (_activate(product("Wg"), c["activation"]) * product("Wu")).to(t)
        y = product("B")
        y = y + s["C"] if c["bias"] else y
        return (torch.where(y > 0, y, torch.zeros_like(y)) if c["relu"] else y).to(t)
    X, Wg, Wu = s["X"].float(), s["Wg"].float(), s["Wu"].float()
    if op == "gated":
        g, u = X @ Wg.T, X @ Wu.T
        h = (_activate(g, c["activation"]) * u).to(t)
        return {"H": h, "G": g.to(t), "U": u.to(t)} if c["save"] else {"H": h}
    dh, g, u = s["dH"].float(), s["G"].float(), s["U"].float()
    dg, du = dh * u * _slope(g, c["activation"]), dh * _activate(g, c["activation"])
    return {"dX": (dg @ Wg + du @ Wu).to(t), "dWg": (dg.T @ X).to(t), "dWu": (du.T @ X).to(t)}


def _own(s):
    from paper_2008_08272_b200 import binding
    c, t = s["case"], TYPES[s["case"]["type"]]
    op = c["op"]
    if op == "quantize_rows":
        q, scale = binding.onnx_quantize_rows(s["X"])
        return {"values": q * scale[:, None], "scale": scale}
    if op == "gemm_int8":
        return binding.onnx_gemm_int8(s["A"], s["a_scale"], s["B"], s["B_scale"], s["C"], fuse_relu=c["relu"], dtype=t)
    if op == "gated_int8":
        return binding.onnx_gated_int8(s["A"], s["a_scale"], s["Wg"], s["Wg_scale"], s["Wu"], s["Wu_scale"],
                                       activation=c["activation"], dtype=t)
    if op == "gated":
        if not c["save"]:
            return {"H": binding.onnx_gated(s["X"], s["Wg"], s["Wu"], activation=c["activation"])}
        h, g, u = binding.onnx_gated(s["X"], s["Wg"], s["Wu"], activation=c["activation"], save=True)
        return {"H": h, "G": g, "U": u}
    dx, dwg, dwu = binding.onnx_gated_backward(s["dH"], s["X"], s["Wg"], s["Wu"], s["G"], s["U"], activation=c["activation"])
    return {"dX": dx, "dWg": dwg, "dWu": dwu}


# --------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s, op, kind = _inputs(case, seed), case["op"], case.get("activation")

    def phi(z):             # the normal distribution's value at z
        return torch.special.erfc(-z / math.sqrt(2)) / 2

    def logistic(z):
        return torch.sigmoid(z)

    def share(z):           # what the activation lets through of z: act(z) = z * share(z)
        if kind == "silu":
            return logistic(z)
        if kind == "gelu":
            return phi(z)
        if kind == "gelu_tanh":
            return logistic(math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3))
        return (z > 0).double()

    if op == "quantize_rows":
        x = s["X"].double()
        scale = (x.abs().max(dim=1).values / 127).float().double()
        q = torch.round(x / torch.where(scale > 0, scale, torch.ones_like(scale)).unsqueeze(1)).clamp(-127, 127)
        return {"values": q * scale.unsqueeze(1), "scale": scale}
    if op in ("gemm_int8", "gated_int8"):
        a = s["A"].double() * s["a_scale"].double().unsqueeze(1)
        w = {n: s[n].double() * s[n + "_scale"].double().unsqueeze(1) for n in (("B",) if op == "gemm_int8" else ("Wg", "Wu"))}
        if op == "gated_int8":
            g = torch.einsum("ik,jk->ij", a, w["Wg"])
            return g * share(g) * torch.einsum("ik,jk->ij", a, w["Wu"])
        y = torch.einsum("ik,jk->ij", a, w["B"])
        if case["bias"]:
            y = y + s["C"].double().unsqueeze(0)
        return y.clamp(min=0) if case["relu"] else y
    X, Wg, Wu = s["X"].double(), s["Wg"].double(), s["Wu"].double()
    if op == "gated":
        g, u = torch.einsum("ik,jk->ij", X, Wg), torch.einsum("ik,jk->ij", X, Wu)
        h = g * share(g) * u
        return {"H": h, "G": g, "U": u} if case["save"] else {"H": h}
    g, u, dh = s["G"].double(), s["U"].double(), s["dH"].double()
    p = share(g)
    if kind == "silu":
        slope = p + g * p * (1 - p)
    elif kind == "gelu":
        slope = p + g * torch.exp(-g.square() / 2) / math.sqrt(2 * math.pi)
    elif kind == "gelu_tanh":
        slope = p + g * p * (1 - p) * math.sqrt(8 / math.pi) * (1 + 3 * 0.044715 * g.square())
    else:
        slope = p
    dg, du = dh * u * slope, dh * (g * p)
    return {"dX": torch.einsum("ij,jk->ik", dg, Wg) + torch.einsum("ij,jk->ik", du, Wu),
            "dWg": torch.einsum("ij,ik->jk", dg, X), "dWu": torch.einsum("ij,ik->jk", du, X)}
