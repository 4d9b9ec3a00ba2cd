"""A layer of experts in a language model and the norm in front of it, as measurable cases: layer normalisation and products whose
weights go by the expert that a row belongs to, forward and backward.

  norm             y = (x - mean) * inv_std * scale + bias, mean and inv_std = 1 / sqrt(variance + epsilon) of each row; "save": these two
                   are outputs too, for the backward pass
  norm_backward    with n = (x - mean) * inv_std and d = dy * scale: dX = inv_std * (d - mean(d) - n * mean(d * n)) of each row,
                   dScale = sum over the rows of dy * n, dBias = sum of dy
  gemm             y[i] = W[e] x[i] for the rows i of expert e, which are offsets[e] to offsets[e + 1] - 1
  gated            g[i] = Wg[e] x[i], u[i] = Wu[e] x[i], h = act(g) * u; with "save" g and u are outputs too, for the backward pass
  gemm_backward    dX[i] = dy[i] W[e], dW[e] = sum over the expert's rows of dy[i]^T x[i]
  gated_backward   dg = dh * u * act'(g), du = dh * act(g); dX[i] = dg[i] Wg[e] + du[i] Wu[e], dWg[e] = sum of dg[i]^T x[i], dWu[e] of du[i]^T x[i]

A case is a dict of plain values.  rows: of the activations (of experts' layers: each token as often as it has experts, by expert);
width: the activations' columns; channels: the results' columns; experts; top: how many of them, all different, a token has; skew: how
much more often some are chosen than others; type: of all tensors but mean and inv_std (32 bits) and, where "wide" is true, the norm's
weights (32 bits as well).
"""
import math
import statistics

import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "fp16": 2, "bf16": 2}
NORMS = ("norm", "norm_backward")


def _case(name, op, rows, width, channels=0, experts=0, **kw):
    c = {"name": name, "op": op, "rows": rows, "width": width, "type": "bf16"}
    if op in NORMS:
        c["wide"] = False
    else:
        c.update(channels=channels, experts=experts, top=1, skew=0.5)
    if op == "norm":
        c.update(save=False, epsilon=1e-5)
    if op.startswith("gated"):
        c["activation"] = "silu"
    if op == "gated":
        c["save"] = False
    c.update(kw)
    return c


def listed():
    return [
        # One token's activations on the way into a layer: the smallest call, where latency is all.
        _case("norm_token", "norm", 1, 4096),
        # A training step's forward half, the norm's weights kept in 32 bits.
        _case("norm_train", "norm", 8192, 4096, save=True, wide=True),
        # A small model in 32 bits whose sizes are no multiples of anything.
        _case("norm_backward_ragged", "norm_backward", 1001, 777, type="fp32"),
        # A training step's backward half.
        _case("norm_backward_train", "norm_backward", 16384, 4096, wide=True),
        # The down projections while eight sequences are answered together, four experts each: weights that have to be read.
        _case("gemm_batch", "gemm", 32, 1408, 2048, 64, top=4),
        # The down projections of a prompt.
        _case("gemm_prompt", "gemm", 16384, 2816, 4096, 16, top=2),
        # One token in two of eight large experts.
        _case("gated_token", "gated", 2, 4096, 10240, 8, top=2),
        # A training step's forward half through many small experts: the two projections are kept.
        _case("gated_train", "gated", 16384, 2048, 1408, 64, top=4, save=True),
        # A few experts whose sizes are no multiples of anything.
        _case("gemm_backward_ragged", "gemm_backward", 1001, 777, 1530, 7, type="fp16"),
        # The down projections in a training step's backward half.
        _case("gemm_backward_train", "gemm_backward", 8192, 2048, 4096, 8, top=2),
        # A small model's experts in a training step's backward half, some of them chosen by hardly a token.
        _case("gated_backward_small", "gated_backward", 512, 1024, 2816, 16, top=2, type="fp16", activation="gelu", skew=1.0),
        # A large model's (the largest case).
        _case("gated_backward_train", "gated_backward", 16384, 4096, 2816, 16, top=2),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _wide(rng, lo, hi):
    """Widths as models have them: mostly multiples of 64, sometimes any number."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.3 else max(64, (n + 32) // 64 * 64)


def draw(rng):
    """One more case of the ranges the listed ones stand for."""
    need = [work(c) for c in listed()]
    most = {k: max(n[k] for n in need) for k in ("bytes", "flops")}
    while True:
        op = rng.choice(("norm", "norm_backward", "gemm", "gated", "gemm_backward", "gated_backward"))
        rows = rng.choice((rng.randint(1, 64), _log_int(rng, 1, 16384), _log_int(rng, 64, 16384)))
        if op in NORMS:
            c = _case("", op, rows, _wide(rng, 32, 16384))
            c["type"] = rng.choice(("bf16", "bf16", "fp16", "fp32"))
            c["wide"] = rng.random() < 0.5
        else:
            c = _case("", op, rows, _wide(rng, 32, 10240), _wide(rng, 32, 10240), _log_int(rng, 1, 128))
            c["type"] = rng.choice(("bf16", "bf16", "fp16"))
            c["top"] = min(c["experts"], rng.choice((1, 2, 4, 8)))
            c["skew"] = rng.choice((0.0, 0.5, 1.0))
        if "save" in c:
            c["save"] = rng.random() < 0.5
        if "activation" in c:
            c["activation"] = rng.choice(("silu", "silu", "gelu", "gelu_tanh", "relu"))
        w = work(c)
        # (all the experts' weights have to fit beside their gradients and 32-bit copies, whether or not a row needs them)
        weights = 2 * c.get("channels", 0) * c["width"] * c.get("experts", 0)
        if w["flops"] <= most["flops"] and w["bytes"] <= most["bytes"] and weights <= 2e9 and w["bytes"] >= 20000:
            del c["name"]
            return c


def _touched(case):
    """How many experts have a row, about: their likings lie as evenly as the normal distribution has them."""
    E, top = case["experts"], case["top"]
    liking = [math.exp(case["skew"] * statistics.NormalDist().inv_cdf((e + 0.5) / E)) for e in range(E)]
    tokens, all_of_them = case["rows"] / top, sum(liking)
    return max(1, round(sum(1 - (1 - min(1.0, top * v / all_of_them)) ** tokens for v in liking)))


def work(case):
    M, K, b, op = case["rows"], case["width"], BYTES[case["type"]], case["op"]
    if op in NORMS:
        w = 4 if case["wide"] else b
        if op == "norm":
            return {"bytes": 2 * b * M * K + 2 * w * K + (8 * M if case["save"] else 0), "flops": 8 * M * K}
        return {"bytes": 3 * b * M * K + 3 * w * K + 8 * M, "flops": 14 * M * K}
    # (all the weights' gradients are written, but only the chosen experts' weights are read)
    N, E, touched = case["channels"], case["experts"], _touched(case)
    if op == "gemm":
        return {"bytes": b * (M * K + M * N + touched * N * K) + 4 * (E + 1), "flops": 2 * M * N * K}
    if op == "gated":
        return {"bytes": b * (M * K + M * N * (3 if case["save"] else 1) + 2 * touched * N * K) + 4 * (E + 1), "flops": 4 * M * N * K}
    if op == "gemm_backward":
        return {"bytes": b * (M * N + 2 * M * K + (touched + E) * N * K) + 4 * (E + 1), "flops": 4 * M * N * K}
    return {"bytes": b * (3 * M * N + 2 * M * K + 2 * (touched + E) * N * K) + 4 * (E + 1), "flops": 8 * M * N * K}


# --------------------------------------------------------------------- inputs
def _device():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def _sizes(case, seed):
    """How many rows each expert has: every token's experts are drawn, some experts more likely than others."""
    gen = torch.Generator().manual_seed(seed)
    liking = torch.exp(case["skew"] * torch.randn(case["experts"], generator=gen))
    tokens = -(-case["rows"] // case["top"])
    chosen = torch.multinomial(liking.expand(tokens, -1), case["top"], replacement=False, generator=gen)
    return torch.bincount(chosen.flatten()[:case["rows"]], minlength=case["experts"]).tolist()


def _parts(t, sizes):
    return torch.split(t, sizes)


def _inputs(case, seed):
    dev, t = _device(), TYPES[case["type"]]
    gen = torch.Generator(device=dev).manual_seed(seed)
    M, K, op = case["rows"], case["width"], case["op"]

    def normal(*size):
        return torch.randn(*size, generator=gen, device=dev, dtype=torch.float32)

    # activations: some channels are several times as large as others
    x = normal(M, K) * torch.exp(0.5 * normal(K))
    if op in NORMS:
        w = torch.float32 if case["wide"] else t
        s = {"X": (x + 0.2 * normal(K)).to(t), "scale": (1 + 0.2 * normal(K)).to(w)}
        if op == "norm":
            s["bias"] = (0.1 * normal(K)).to(w)
            return s
        s["dY"] = normal(M, K).to(t)
        wide = s["X"].double()
        s["mean"] = wide.mean(1).float()
        s["inv_std"] = (1 / torch.sqrt(wide.var(1, unbiased=False) + 1e-5)).float()
        return s
    N, E = case["channels"], case["experts"]
    sizes = _sizes(case, seed)
    s = {"X": x.to(t), "sizes": sizes}
    s["offsets"] = torch.tensor([0] + sizes).cumsum(0).to(torch.int32).to(dev)

    def weights():
        w = torch.empty(E, N, K, dtype=t, device=dev)
        for e in range(E):
            w[e] = normal(N, K) / math.sqrt(K)
        return w

    if op in ("gemm", "gemm_backward"):
        s["W"] = weights()
        if op == "gemm_backward":
            s["dY"] = normal(M, N).to(t)
        return s
    s["Wg"], s["Wu"] = weights(), weights()
    if op == "gated_backward":
        s["dH"] = normal(M, N).to(t)
        for name, w in (("G", s["Wg"]), ("U", s["Wu"])):
            s[name] = torch.cat([a.float() @ b.float().T for a, b in zip(_parts(s["X"], sizes), w)]).to(t)
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
    if op == "norm":
        x = s["X"].float()
        mean = x.mean(1, keepdim=True)
        away = x - mean
        inv_std = 1 / torch.sqrt((away * away).mean(1, keepdim=True) + c["epsilon"])
        y = (away * inv_std * s["scale"].float() + s["bias"].float()).to(t)
        return {"Y": y, "mean": mean[:, 0], "inv_std": inv_std[:, 0]} if c["save"] else {"Y": y}
    if op == "norm_backward":
        dy, inv_std = s["dY"].float(), s["inv_std"][:, None]
        n = (s["X"].float() - s["mean"][:, None]) * inv_std
        d = dy * s["scale"].float()
        dx = inv_std * (d - d.mean(1, keepdim=True) - n * (d * n).mean(1, keepdim=True))
        w = s["scale"].dtype
        return {"dX": dx.to(t), "dScale": (dy * n).sum(0).to(w), "dBias": dy.sum(0).to(w)}
    sizes, X = s["sizes"], s["X"]
    if op == "gemm":
        return torch.cat([(x.float() @ w.float().T).to(t) for x, w in zip(_parts(X, sizes), s["W"])])
    if op == "gated":
        out = {"H": torch.empty(c["rows"], c["channels"], dtype=t, device=X.device)}
        if c["save"]:
            out["G"], out["U"] = torch.empty_like(out["H"]), torch.empty_like(out["H"])
        first = 0
        for x, wg, wu in zip(_parts(X, sizes), s["Wg"], s["Wu"]):
            x, last = x.float(), first + len(x)
            g, u = x @ wg.float().T, x @ wu.float().T
            out["H"][first:last] = _activate(g, c["activation"]) * u
            if c["save"]:
                out["G"][first:last], out["U"][first:last] = g, u
            first = last
        return out
    names = ("W",) if op == "gemm_backward" else ("Wg", "Wu")
    dx, dw = [], {"d" + n: torch.empty_like(s[n]) for n in names}
    first = 0
    for e, size in enumerate(sizes):
        rows = slice(first, first + size)
        first += size
        x = X[rows].float()
        if op == "gemm_backward":
            ds = (s["dY"][rows].float(),)
        else:
            dh, g, u = s["dH"][rows].float(), s["G"][rows].float(), s["U"][rows].float()
            ds = (dh * u * _slope(g, c["activation"]), dh * _activate(g, c["activation"]))
        dx.append(sum(d @ s[n][e].float() for d, n in zip(ds, names)).to(t))
        for d, n in zip(ds, names):
            dw["d" + n][e] = d.T @ x
    return {"dX": torch.cat(dx), **dw}


def _own(s):
    from paper_2008_08272_b200 import binding
    c, op = s["case"], s["case"]["op"]
    if op == "norm":
        if not c["save"]:
            return {"Y": binding.onnx_layer_normalization(s["X"], s["scale"], s["bias"], epsilon=c["epsilon"])}
        y, mean, inv_std = binding.onnx_layer_normalization(s["X"], s["scale"], s["bias"], epsilon=c["epsilon"], save=True)
        return {"Y": y, "mean": mean, "inv_std": inv_std}
    if op == "norm_backward":
        dx, dscale, dbias = binding.onnx_layer_normalization_backward(s["dY"], s["X"], s["scale"], s["mean"], s["inv_std"])
        return {"dX": dx, "dScale": dscale, "dBias": dbias}
    if op == "gemm":
        return binding.onnx_grouped_gemm(s["X"], s["W"], s["offsets"])
    if op == "gated":
        if not c["save"]:
            return {"H": binding.onnx_grouped_gated(s["X"], s["Wg"], s["Wu"], s["offsets"], activation=c["activation"])}
        h, g, u = binding.onnx_grouped_gated(s["X"], s["Wg"], s["Wu"], s["offsets"], activation=c["activation"], save=True)
        return {"H": h, "G": g, "U": u}
    if op == "gemm_backward":
        dx, dw = binding.onnx_grouped_gemm_backward(s["dY"], s["X"], s["W"], s["offsets"])
        return {"dX": dx, "dW": dw}
    dx, dwg, dwu = binding.onnx_grouped_gated_backward(s["dH"], s["X"], s["Wg"], s["Wu"], s["G"], s["U"], s["offsets"],
                                                       activation=c["activation"])
    return {"dX": dx, "dWg": dwg, "dWu": dwu}


# --------------------------------------------------------------------- the definition in 64 bits
def _share(z, kind):
    """What the activation lets through of z, act(z) = z * share(z), and its derivative."""
    if kind == "silu":
        p = torch.sigmoid(z)
        return p, p * (1 - p)
    if kind == "gelu":
        return torch.special.erfc(-z / math.sqrt(2)) / 2, torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        p = torch.sigmoid(math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3))
        return p, p * (1 - p) * math.sqrt(8 / math.pi) * (1 + 3 * 0.044715 * z.square())
    return (z > 0).double(), torch.zeros_like(z)


def exact(case, seed):
    s, op = _inputs(case, seed), case["op"]
    X = s["X"].double()
    if op == "norm":
        variance, mean = torch.var_mean(X, dim=1, correction=0)
        inv_std = (variance + case["epsilon"]).rsqrt()
        y = torch.addcmul(s["bias"].double(), (X - mean.unsqueeze(1)) * inv_std.unsqueeze(1), s["scale"].double())
        return {"Y": y, "mean": mean, "inv_std": inv_std} if case["save"] else {"Y": y}
    if op == "norm_backward":
        # of the mean and inv_std that the call is given
        dy, r, scale = s["dY"].double(), s["inv_std"].double(), s["scale"].double()
        n = (X - s["mean"].double().unsqueeze(1)) * r.unsqueeze(1)
        K = case["width"]
        along = torch.einsum("ij,j,ij->i", dy, scale, n) / K
        level = torch.einsum("ij,j->i", dy, scale) / K
        dx = torch.einsum("i,ij->ij", r, dy * scale - level.unsqueeze(1) - n * along.unsqueeze(1))
        return {"dX": dx, "dScale": torch.einsum("ij,ij->j", dy, n), "dBias": torch.einsum("ij->j", dy)}
    M, N, K, E = case["rows"], case["channels"], case["width"], case["experts"]
    ends = s["offsets"].tolist()

    def by_row(a, name, form, cols):          # a product of each expert's rows with its weights
        out = torch.zeros(M, cols, dtype=torch.float64, device=X.device)
        for e in range(E):
            out[ends[e]:ends[e + 1]] = torch.einsum(form, a[ends[e]:ends[e + 1]], s[name][e].double())
        return out

    def by_expert(a):                         # the sum over each expert's rows of a^T x
        return torch.stack([torch.einsum("ij,ik->jk", a[ends[e]:ends[e + 1]], X[ends[e]:ends[e + 1]]) for e in range(E)])

    if op == "gemm":
        return by_row(X, "W", "ik,jk->ij", N)
    if op == "gated":
        g, u = (by_row(X, n, "ik,jk->ij", N) for n in ("Wg", "Wu"))
        h = g * _share(g, case["activation"])[0] * u
        return {"H": h, "G": g, "U": u} if case["save"] else {"H": h}
    if op == "gemm_backward":
        dy = s["dY"].double()
        return {"dX": by_row(dy, "W", "ij,jk->ik", K), "dW": by_expert(dy)}
    g, u, dh = s["G"].double(), s["U"].double(), s["dH"].double()
    p, dp = _share(g, case["activation"])
    dg, du = dh * u * (p + g * dp), dh * (g * p)
    return {"dX": by_row(dg, "Wg", "ij,jk->ik", K) + by_row(du, "Wu", "ij,jk->ik", K), "dWg": by_expert(dg), "dWu": by_expert(du)}
