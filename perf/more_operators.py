"""The work whose speed counts in the 8-bit projections of a video transformer block: the norm in
front of a projection, the projection's product in 8-bit floating point, and both in training.

Operators
  RMS norm    h = x + residual (where there is one), y = h rstd * weight, rstd = 1 / sqrt(mean h^2 + eps),
              with one weight or one for every group of rows; y in the rows' type, or in 8 bits
              with scales, as the product reads it
  8-bit form  q = e4m3(x / s), s the least power of two with max |x| <= 448 s over a block: 1 x 128
              (a row's channels), 128 x 1 (a channel's rows) or 128 x 128
  product     C = A B^T of two matrices in that form, whose scales follow the contraction in
              blocks of 128
  linear      y = x W^T with all three products of training in that form:
              y = [x]_1x128 [W]_128x128^T, dx = [dy]_1x128 [W]_128x128, dW = [dy]_128x1^T [x]_128x1

Kinds of case
  mm       the product alone: activations and weights in 8 bits already
  out      activations put into 8 bits, then the product (an attention's output projection)
  project  RMS norm with the residual's addition and output in 8 bits, then the product
  linear   forward and backward of the linear layer through the autograd function
  norm     RMS norm with the residual's addition, forward and backward through autograd

Sizes are the model table's widths (B 768, 0.5B 1152, 1B 1536, 3B 2560), their projections of one, three
and four times that, the windows of 880-token chunks, and single tokens.
"""
import math

import torch

BF16, F32, F64, E4M3 = torch.bfloat16, torch.float32, torch.float64, torch.float8_e4m3fn
EPS = 1e-6

own = False
mw = None


def _mw():
    global mw
    if mw is None:
        import paper_2608_01127_gb300
        mw = paper_2608_01127_gb300
    return mw


def listed():
    return [
        # serving, the smallest call: one token through the B layout's QKV projection
        dict(name="mm_token_b", kind="mm", M=1, K=768, N=2304),
        # serving: a token of each of eight streams through the 3B layout's second MLP product
        dict(name="mm_tokens_3b", kind="mm", M=8, K=10240, N=2560),
        # validation of the 1B layout: a window of 32 chunks of 600, the first MLP product
        dict(name="mm_eval_1b", kind="mm", M=19200, K=1536, N=6144),
        # streaming: one chunk at an odd latent size (7 x 43) through the 0.5B layout's output projection
        dict(name="out_step_odd", kind="out", M=301, K=1152, N=1152, x="bf16"),
        # the output projection of the 3B layout, a window of 16 chunks
        dict(name="out_3b", kind="out", M=14080, K=2560, N=2560, x="bf16"),
        # serving: norm and QKV projection of two tokens of the 1B layout
        dict(name="project_tokens_1b", kind="project", M=2, K=1536, N=4608, G=1, x="bf16"),
        # norm and QKV projection of the 3B layout, a weight for each of 32 frames
        dict(name="project_3b", kind="project", M=14080, K=2560, N=7680, G=32, x="bf16"),
        # training of the B layout's QKV projection
        dict(name="linear_b", kind="linear", M=14080, K=768, N=2304, w="f32"),
        # training of the 0.5B layout's output projection on ragged clips: an odd number of tokens
        dict(name="linear_odd", kind="linear", M=4403, K=1152, N=1152, w="bf16"),
        # training of the 3B layout's first MLP product
        dict(name="linear_3b", kind="linear", M=14080, K=2560, N=10240, w="f32"),
        # training: the norm in front of the B layout's sublayers, two windows
        dict(name="norm_b", kind="norm", R=28160, C=768, G=1, x="bf16", residual=True),
        # training: the 3B layout's, a weight for each frame of 440 tokens
        dict(name="norm_3b_frames", kind="norm", R=14080, C=2560, G=32, x="bf16", residual=True),
    ]


# ------------------------------------------------------------------ sizes and work

def _blocks(n):
    return (n + 127) // 128


def _size(t):
    return 4 if t == "f32" else 2


def work(case):
    c = case
    if c["kind"] == "norm":
        n, xs, params = c["R"] * c["C"], _size(c["x"]), c["G"] * c["C"] * 4
        # forward: x (and the residual) in, y (and h) out; backward: dy (and dh) and h in, one gradient out
        return {"bytes": n * xs * (8 if c["residual"] else 5) + 3 * params, "flops": 14 * n}
    M, K, N = c["M"], c["K"], c["N"]
    flops = 2 * M * K * N
    weights = N * K + _blocks(N) * _blocks(K)
    if c["kind"] == "mm":
        return {"bytes": M * K + M * _blocks(K) + weights + 2 * M * N, "flops": flops}
    if c["kind"] == "out":
        return {"bytes": M * K * _size(c["x"]) + weights + 2 * M * N, "flops": flops}
    if c["kind"] == "project":
        return {"bytes": 3 * M * K * _size(c["x"]) + 4 * c["G"] * K + weights + 2 * M * N, "flops": flops}
    # x, W, dy in; y, dx, dW out
    return {"bytes": 2 * 2 * M * (K + N) + 2 * N * K * _size(c["w"]), "flops": 3 * flops}


# ------------------------------------------------------------------ drawn cases

def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(work(c)["flops"] for c in listed())
    while True:
        kind = rng.choice(["mm", "mm", "out", "project", "project", "linear", "linear", "norm", "norm"])
        if kind == "norm":
            G = rng.choice([1, 1, rng.randint(2, 40)])
            c = dict(kind=kind, R=G * _log_int(rng, 1, max(1, 40000 // G)),
                     C=rng.choice([768, 1024, 1152, 1536, 2560, _log_int(rng, 33, 8192)]), G=G,
                     x=rng.choice(["bf16", "bf16", "f32"]), residual=rng.random() < 0.7)
            if c["R"] * c["C"] <= 14080 * 2560:
                return c
            continue
        width = [768, 1024, 1152, 1536, 2560]
        K = rng.choice(width + [16 * _log_int(rng, 4, 700)] * 2)
        c = dict(kind=kind, K=K if kind != "project" else min(K, 8192), N=rng.choice([K, 16 * _log_int(rng, 4, 700), 16 * _log_int(rng, 4, 700)]))
        if kind == "linear":
            c.update(M=_log_int(rng, 64, 30000), w=rng.choice(["f32", "bf16"]))
        else:
            c.update(M=rng.choice([1, rng.randint(1, 16), rng.randint(17, 200), _log_int(rng, 200, 30000)]))
        if kind == "project":
            c["G"] = rng.choice([1, 1, rng.randint(1, 8)])
            c["M"] = c["G"] * max(1, c["M"] // c["G"])
        if kind in ("out", "project"):
            c["x"] = rng.choice(["bf16", "bf16", "f32"])
        if work(c)["flops"] <= most and max(c["N"] * c["K"], c["M"] * max(c["N"], c["K"])) <= 14080 * 10240:
            return c


# ------------------------------------------------------------------ inputs

def _type(t):
    return F32 if t == "f32" else BF16


def _inputs(c, seed):
    """The tensors a program has before the call, on the GPU."""
    g = torch.Generator("cuda").manual_seed(int(seed))

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=F32)

    def activations(rows, channels):
        # channels of unequal size, some of them far larger than the rest
        size = (0.3 + randn(channels).abs()) * torch.where(randn(channels) > 2.3, 12.0, 1.0)
        return randn(rows, channels) * size

    if c["kind"] == "norm":
        t = _type(c["x"])
        x = {"x": activations(c["R"], c["C"]).to(t), "dy": randn(c["R"], c["C"]).to(t)}
        x["residual"] = (activations(c["R"], c["C"]) * 2).to(t) if c["residual"] else None
        x["dh"] = randn(c["R"], c["C"]).to(t) if c["residual"] else None
        x["weight"] = 1.0 + 0.2 * randn(*((c["C"],) if c["G"] == 1 else (c["G"], c["C"])))
        return x
    M, K, N = c["M"], c["K"], c["N"]
    x = {"x": activations(M, K).to(_type(c.get("x", "bf16")))}
    x["w"] = (randn(N, K) * (0.5 + randn(N, 1).abs()) / math.sqrt(K)).to(_type(c.get("w", "bf16")))
    if c["kind"] == "project":
        x["residual"] = (activations(M, K) * 2).to(_type(c["x"]))
        x["weight"] = 1.0 + 0.2 * randn(*((K,) if c["G"] == 1 else (c["G"], K)))
    if c["kind"] == "linear":
        # a gradient: far smaller than 1, rows of unequal size
        x["dy"] = (randn(M, N) * (1e-4 * (0.1 + randn(M, 1).abs()))).to(BF16)
    return x


def prepare(case, seed):
    s = dict(case)
    s.update(_inputs(case, seed))
    if case["kind"] == "norm":
        for n in ("x", "residual", "weight"):
            if s[n] is not None:
                s[n].requires_grad_(True)
    elif case["kind"] == "linear":
        s["x"].requires_grad_(True)
        s["w"].requires_grad_(True)
    else:  # serving keeps its weights in 8 bits, and here and there gets activations so
        s["wq"], s["ws"] = _put(s.pop("w"), 128, 128)
        if case["kind"] == "mm":
            s["xq"], s["xs"] = _put(s.pop("x"), 1, 128)
    return s


# ------------------------------------------------------------------ one pass, plain

def _put(x, rows, columns):
    """The 8-bit form of x with a scale for each block of rows x columns: (q, scale)."""
    R, C = x.shape
    r, c = -R % rows, -C % columns
    t = torch.nn.functional.pad(x.float(), (0, c, 0, r)).view((R + r) // rows, rows, (C + c) // columns, columns)
    top = t.abs().amax((1, 3), keepdim=True)
    mantissa, exponent = torch.frexp(top.double() / 448.0)  # top / 448 = mantissa 2^exponent, mantissa in [1/2, 1)
    exponent = torch.where(top == 0, -127, exponent - (mantissa == 0.5).int()).clamp(-127, 127)
    scale = (exponent + 127).to(torch.uint8).view(torch.float8_e8m0fnu)
    q = (t / scale.float()).to(E4M3).view(R + r, C + c)[:R, :C].contiguous()
    return q, scale[:, 0, :, 0].contiguous()


def _values(q, scale, rows, columns):
    """What the 8-bit form stands for, in 32 bits."""
    R, C = q.shape
    s = scale.float().repeat_interleave(rows, 0)[:R].repeat_interleave(columns, 1)[:, :C]
    return q.float() * s


def _rounded(x, rows, columns):
    return _values(*_put(x, rows, columns), rows, columns)


def _plain_norm(s, h):
    """(normalised rows, weights for every row, rstd) in 32 bits."""
    R, C = h.shape
    rstd = 1.0 / torch.sqrt((h * h).sum(-1, keepdim=True) / C + EPS)
    w = s["weight"].detach().view(s["G"], 1, C).expand(s["G"], R // s["G"], C).reshape(R, C)
    return h * rstd, w, rstd


def _sum(s):
    x, r = s["x"].detach(), s["residual"]
    return x if r is None else (x.float() + r.detach().float()).to(x.dtype)


def _plain(s):
    kind = s["kind"]
    if kind == "norm":
        h = _sum(s)
        xh, w, rstd = _plain_norm(s, h.float())
        C, dy = s["C"], s["dy"].float()
        g = dy * w
        d = rstd * (g - xh * ((g * xh).sum(-1, keepdim=True) / C))
        if s["dh"] is not None:
            d = d + s["dh"].float()
        dw = (dy * xh).view(s["G"], -1, C).sum(1).view(s["weight"].shape)
        d = d.to(h.dtype)
        out = {"y": (xh * w).to(h.dtype), "dx": d, "dweight": dw}
        if s["dh"] is not None:
            out.update(h=h, dresidual=d)
        return out
    if kind == "linear":
        x, w, dy = s["x"].detach(), s["w"].detach(), s["dy"]
        wr = _rounded(w, 128, 128)
        y = torch.matmul(_rounded(x, 1, 128), wr.T).to(BF16)
        dx = torch.matmul(_rounded(dy, 1, 128), wr).to(BF16)
        dw = torch.matmul(_rounded(dy, 128, 1).T, _rounded(x, 128, 1)).to(w.dtype)
        return {"y": y, "dx": dx, "dw": dw}
    out = {}
    if kind == "mm":
        x = _values(s["xq"], s["xs"], 1, 128)
    elif kind == "out":
        x = _rounded(s["x"], 1, 128)
    else:
        out["h"] = _sum(s)
        xh, w, _ = _plain_norm(s, out["h"].float())
        x = _rounded(xh * w, 1, 128)
    out["y"] = torch.matmul(x, _values(s["wq"], s["ws"], 128, 128).T).to(BF16)
    return out


# ------------------------------------------------------------------ one pass

def run(state):
    s = state
    if not own:
        return _plain(s)
    lib = _mw()
    kind = s["kind"]
    if kind == "norm":
        if s["residual"] is None:
            y = lib.RMSNorm.apply(s["x"], s["weight"], None, EPS)
            dx, dw = torch.autograd.grad(y, (s["x"], s["weight"]), s["dy"])
            return {"y": y.detach(), "dx": dx, "dweight": dw}
        y, h = lib.RMSNorm.apply(s["x"], s["weight"], s["residual"], EPS)
        dx, dr, dw = torch.autograd.grad((y, h), (s["x"], s["residual"], s["weight"]), (s["dy"], s["dh"]))
        return {"y": y.detach(), "h": h.detach(), "dx": dx, "dresidual": dr, "dweight": dw}
    if kind == "linear":
        y = lib.Fp8Linear.apply(s["x"], s["w"])
        dx, dw = torch.autograd.grad(y, (s["x"], s["w"]), s["dy"])
        return {"y": y.detach(), "dx": dx, "dw": dw}
    if kind == "mm":
        return {"y": lib.mw_scaled_matmul(s["xq"], s["xs"], s["wq"], s["ws"])}
    if kind == "out":
        q, scale = lib.mw_quantize(s["x"], (1, 128))
        return {"y": lib.mw_scaled_matmul(q, scale, s["wq"], s["ws"])}
    q, scale, h, _ = lib.mw_rmsnorm_quantize(s["x"], s["weight"], s["residual"], EPS, need_stats=False)
    return {"h": h, "y": lib.mw_scaled_matmul(q, scale, s["wq"], s["ws"])}


# ------------------------------------------------------------------ the same in 64 bits

def _nearest(v):
    """The e4m3 values next to v, |v| <= 448, ties to even: steps of 2^-3 of the power of two below
    |v|, of 2^-9 below 2^-6."""
    a = v.abs()
    step = torch.exp2(torch.floor(torch.log2(torch.clamp(a, min=2.0 ** -6))) - 3)
    return torch.round(v / step) * step


def _form(x, block):
    """What the 8-bit form of x stands for, a block one of "row", "column", "tile"."""
    x = x.to(F64)
    out = torch.empty_like(x)
    R, C = x.shape
    if block == "column":
        return _form(x.T.contiguous(), "row").T
    tall = 1 if block == "row" else 128
    for j in range(0, C, 128):
        part = x[:, j:j + 128]
        top = part.abs().amax(1, keepdim=True)
        if tall > 1:
            groups = [top[i:i + tall].amax().expand(len(top[i:i + tall]), 1) for i in range(0, R, tall)]
            top = torch.cat(groups)
        ratio = top / 448.0
        power = torch.exp2(torch.ceil(torch.log2(torch.where(ratio > 0, ratio, 1.0))))
        # (the logarithm of a value next to a power of two may come out as a whole number)
        power = torch.where(ratio > power, power * 2, torch.where(ratio <= power / 2, power / 2, power))
        power = torch.clamp(power, min=2.0 ** -127)
        out[:, j:j + 128] = _nearest(part / power) * power
    return out


def exact(case, seed):
    c, x = case, _inputs(case, seed)
    kind = c["kind"]

    def normed():
        h = x["x"] if x["residual"] is None else (x["x"].to(F64) + x["residual"].to(F64)).to(x["x"].dtype)
        h3 = h.to(F64).view(c["G"], -1, h.shape[1])
        norm = h3.square().mean(-1, keepdim=True).add(EPS).sqrt()
        return h, h3 / norm, norm

    if kind == "norm":
        h, xh, norm = normed()
        w, dy = x["weight"].to(F64).view(c["G"], 1, c["C"]), x["dy"].to(F64).view(c["G"], -1, c["C"])
        g = dy * w
        d = (g - xh * (g * xh).mean(-1, keepdim=True)) / norm
        out = {"y": (xh * w).view(c["R"], c["C"]), "dweight": (dy * xh).sum(1).view(x["weight"].shape)}
        d = d.view(c["R"], c["C"])
        if c["residual"]:
            d = d + x["dh"].to(F64)
            out.update(h=h.to(F64), dresidual=d)
        out["dx"] = d
        return out
    if kind == "linear":
        w = _form(x["w"], "tile")
        return {"y": _form(x["x"], "row") @ w.T, "dx": _form(x["dy"], "row") @ w,
                "dw": _form(x["dy"], "column").T @ _form(x["x"], "column")}
    out = {}
    if kind == "project":
        h, xh, _ = normed()
        out["h"] = h.to(F64)
        a = (xh * x["weight"].to(F64).view(c["G"], 1, c["K"])).view(c["M"], c["K"])
    else:
        a = x["x"]
    out["y"] = _form(a, "row") @ _form(x["w"], "tile").T
    return out
