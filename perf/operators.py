"""The work whose speed counts in the conditioning path of a video transformer block: a
pre-norm cross attention sublayer, as training, evaluation and streaming programs call it.

Operators
  cross attention   softmax(scale Q K^T) V over an encoder's states of another length, with
                    heads of K and V shared by groups of query heads and a number of valid
                    states per sample (padded prompts; 0 where the condition is dropped)
  layer norm        y = (x - mean) rstd * weight + bias over the channels, with one weight and
                    bias, or one of each for every group of rows (a sample, a frame) as adaptive
                    modulation needs

Kinds of case
  train    cross attention forward and backward through the autograd function
  eval     cross attention forward only, with or without LSE
  token    cross attention of a single new token (or a few), as serving steps call it
  norm     layer norm forward and backward through the autograd function
  norm_fwd layer norm forward only

Sizes are the model table's head layouts and widths (B and L: 64 channels per head, 0.5B: 72,
1B and 3B: 128), its windows of 880-token chunks, and generic lengths of encoder states.
"""
import math

import torch

BF16 = torch.bfloat16
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
        # serving, the smallest call: one new token of the B layout against a short prompt
        dict(name="token_tiny_d64", kind="token", B=1, H=12, Hkv=12, d=64, M=1, S=77, lens="full", lse=False, gain=1.0),
        # serving: eight streams of the 3B layout, five query heads to a head of K and V, each
        # token against the states of a long document, of which a stream holds some
        dict(name="token_3b_8k", kind="token", B=8, H=20, Hkv=4, d=128, M=1, S=8192, lens="ragged", lse=False, gain=1.5),
        # streaming: one chunk of the L layout against a padded prompt of an odd length
        dict(name="eval_step_odd", kind="eval", B=1, H=16, Hkv=16, d=64, M=880, S=301, lens="ragged", lse=True, gain=1.0),
        # validation of the 1B layout: a window of 32 chunks of 600 against 512 states
        dict(name="eval_1b_512", kind="eval", B=1, H=12, Hkv=12, d=128, M=19200, S=512, lens="full", lse=False, gain=1.5),
        # training of the B layout on padded prompts, one sample's condition dropped
        dict(name="train_b_text", kind="train", B=4, H=12, Hkv=12, d=64, M=14080, S=256, lens="dropped", gain=1.0),
        # training of the 0.5B layout (72 channels) on images' patch states
        dict(name="train_05b_d72", kind="train", B=1, H=16, Hkv=16, d=72, M=14080, S=1025, lens="full", gain=1.0),
        # training of the 3B layout with shared heads on a short clip, ragged states
        dict(name="train_3b_shared", kind="train", B=2, H=20, Hkv=4, d=128, M=4400, S=1500, lens="ragged", gain=1.5),
        # 16 heads of 128, a window against the states of eight chunks of a reference video
        dict(name="train_h16_video", kind="train", B=1, H=16, Hkv=16, d=128, M=14080, S=7040, lens="full", gain=2.0),
        # the norm in front of it: B layout, two windows of 16 chunks, one weight
        dict(name="norm_b_768", kind="norm", R=28160, C=768, G=1, x="bf16", y="bf16"),
        # the same for the 3B layout with a weight and bias for each frame of 440 tokens
        dict(name="norm_3b_frames", kind="norm", R=14080, C=2560, G=32, x="bf16", y="bf16"),
        # a residual stream kept in 32 bits, odd width
        dict(name="norm_odd_f32", kind="norm", R=5003, C=1155, G=1, x="f32", y="bf16"),
        # streaming: one chunk of the 0.5B layout, forward only
        dict(name="norm_fwd_step", kind="norm_fwd", R=880, C=1152, G=2, x="bf16", y="bf16"),
    ]


# ------------------------------------------------------------------ sizes and work

def _attends(c):
    return c["kind"] in ("train", "eval", "token")


def _size(t):
    return 4 if t == "f32" else 2


def _lens(c, seed):
    """Valid states of each sample, on the host."""
    B, S = c["B"], c["S"]
    if c["lens"] == "full":
        return [S] * B
    g = torch.Generator().manual_seed(int(seed) * 7 + 1)
    lens = torch.randint((S + 3) // 4, S + 1, (B,), generator=g).tolist()
    lens[int(torch.randint(0, B, (1,), generator=g))] = S  # padded to the longest
    if c["lens"] == "dropped" and B > 1:
        lens[int(torch.randint(0, B, (1,), generator=g))] = 0
    return lens


def _states(c):
    """Valid states over the samples of a batch: its expectation, where it is drawn."""
    B, S = c["B"], c["S"]
    if c["lens"] == "full":
        return B * S
    some = S + (B - 1) * 0.625 * S
    return some * (B - 1) / B if c["lens"] == "dropped" and B > 1 else some


def work(case):
    c = case
    if _attends(c):
        rows, pairs = c["B"] * c["H"] * c["M"], c["H"] * c["M"] * _states(c)
        keys = c["Hkv"] * _states(c)  # padded states need not be read
        if c["kind"] == "train":
            # Q, dO in, O, dQ out, K, V in; dK, dV out whole, zeros in padded places
            return {"bytes": int(4 * rows * c["d"] * 2 + 2 * keys * c["d"] * 2 + 2 * c["B"] * c["Hkv"] * c["S"] * c["d"] * 2),
                    "flops": int(14 * c["d"] * pairs)}
        return {"bytes": int(2 * rows * c["d"] * 2 + 2 * keys * c["d"] * 2 + (4 * rows if c["lse"] else 0)),
                "flops": int(4 * c["d"] * pairs)}
    n, xs, ys, params = c["R"] * c["C"], _size(c["x"]), _size(c["y"]), c["G"] * c["C"] * 4
    if c["kind"] == "norm":
        # x read and y written; x and dy read again for the gradient (dy comes after y), dx written
        return {"bytes": n * (3 * xs + 2 * ys) + 4 * params, "flops": 20 * n}
    return {"bytes": n * (xs + ys) + 2 * params, "flops": 8 * n}


# ------------------------------------------------------------------ drawn cases

def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(work(c)["flops"] for c in listed())
    while True:
        kind = rng.choice(["train", "train", "eval", "token", "token", "norm", "norm", "norm_fwd"])
        if kind in ("norm", "norm_fwd"):
            G = rng.choice([1, 1, rng.randint(2, 40)])
            c = dict(kind=kind, R=G * _log_int(rng, 1, max(1, 40000 // G)),
                     C=rng.choice([768, 1024, 1152, 1536, 2560, _log_int(rng, 33, 8192)]), G=G,
                     x=rng.choice(["bf16", "bf16", "f32"]), y="bf16")
            if c["x"] == "f32":
                c["y"] = rng.choice(["bf16", "f32"])
            if c["R"] * c["C"] > 14080 * 2560 or 3072 in (c["R"], c["C"]):
                continue
            return c
        Hkv = rng.choice([1, 2, 4, 8, 12, 16, rng.randint(1, 20)])
        c = dict(kind=kind, B=rng.choice([1, 1, 2, 4, rng.randint(1, 8)]), H=Hkv * rng.choice([1, 1, 1, 2, 4, 5]), Hkv=Hkv,
                 d=rng.choice([64, 64, 72, 128, 128, rng.choice([80, 88, 96, 112])]),
                 M=rng.choice([1, 1, rng.randint(1, 16)]) if kind == "token" else _log_int(rng, 17, 20000),
                 S=_log_int(rng, 1, 32768 if kind == "token" else 8192),
                 lens=rng.choice(["full", "ragged", "dropped"]), gain=rng.choice([1.0, 1.5, 2.0]))
        if kind != "train":
            c["lse"] = rng.random() < 0.5
        if c["H"] > 24 or 3072 in (c["M"], c["S"]):
            continue
        # a pass costs no more than the largest listed one, with all states valid
        pairs = c["B"] * c["H"] * c["M"] * c["S"]
        if 14 * c["d"] * pairs <= most and c["B"] * c["Hkv"] * c["S"] <= 8 * 4 * 32768:
            return c


# ------------------------------------------------------------------ inputs

def _inputs(c, seed):
    """The tensors a program has before the call, on the GPU."""
    g = torch.Generator("cuda").manual_seed(int(seed))

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    if _attends(c):
        x = {"q": randn(c["B"], c["H"], c["M"], c["d"]) * c["gain"]}
        x["k"] = randn(c["B"], c["Hkv"], c["S"], c["d"]) * c["gain"]
        x["v"] = randn(c["B"], c["Hkv"], c["S"], c["d"])
        if c["kind"] == "train":
            x["do"] = randn(c["B"], c["H"], c["M"], c["d"])
        x = {n: t.to(BF16) for n, t in x.items()}
        x["kv_len"] = None
        if c["lens"] != "full":
            x["kv_len"] = torch.tensor(_lens(c, seed), dtype=torch.int32, device="cuda")
        return x
    R, C, G = c["R"], c["C"], c["G"]
    # a residual stream: channels of unequal size about a mean of their own
    x = {"x": randn(R, C) * (0.5 + randn(C).abs()) + 0.5 * randn(C)}
    x["x"] = x["x"].to(torch.float32 if c["x"] == "f32" else BF16)
    shape = (C,) if G == 1 else (G, C)
    x["weight"], x["bias"] = 1.0 + 0.2 * randn(*shape), 0.2 * randn(*shape)
    if c["kind"] == "norm":
        x["dy"] = randn(R, C).to(torch.float32 if c["y"] == "f32" else BF16)
    return x


def prepare(case, seed):
    s = dict(case)
    s.update(_inputs(case, seed))
    if case["kind"] == "train":
        for n in ("q", "k", "v"):
            s[n].requires_grad_(True)
    if case["kind"] == "norm":
        for n in ("x", "weight", "bias"):
            s[n].requires_grad_(True)
    if not _attends(case):
        s["out_dtype"] = torch.float32 if case["y"] == "f32" else BF16
    return s


# ------------------------------------------------------------------ one pass, plain

def _plain_attention(s):
    """Cross attention in elementary operations, 32 bits, rounded once at the end."""
    B, H, M, d = s["q"].shape
    Hkv, S = s["k"].shape[1], s["k"].shape[2]
    scale = 1.0 / math.sqrt(d)
    # the query heads that share a head of K and V, one after another
    q = s["q"].detach().float().reshape(B, Hkv, H // Hkv * M, d)
    k, v = s["k"].detach().float(), s["v"].detach().float()
    if s["kv_len"] is None:
        seen = torch.ones(B, 1, 1, S, dtype=torch.bool, device=q.device)
    else:
        seen = (torch.arange(S, device=q.device) < s["kv_len"][:, None]).view(B, 1, 1, S)
    k = torch.where(seen.view(B, 1, S, 1), k, 0.0)  # what lies in padded places does not count
    v = torch.where(seen.view(B, 1, S, 1), v, 0.0)
    x = torch.matmul(q, k.transpose(-1, -2)).mul_(scale)
    x.masked_fill_(~seen, -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = x.sum(-1, keepdim=True)
    p = x.mul_(torch.where(total > 0, 1.0 / total, 0.0))
    o = torch.matmul(p, v)
    out = {"o": o.reshape(B, H, M, d).to(BF16)}
    if s["kind"] != "train":
        out["lse"] = (top + total.log()).reshape(B, H, M) if s["lse"] else None
        return out
    g = s["do"].float().reshape(B, Hkv, H // Hkv * M, d)
    dv = torch.matmul(p.transpose(-1, -2), g)
    ds = torch.matmul(g, v.transpose(-1, -2))
    ds.sub_((g * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(-1, -2), q)
    out.update(dq=dq.reshape(B, H, M, d).to(BF16), dk=dk.to(BF16), dv=dv.to(BF16))
    return out


def _plain_norm(s):
    """Layer norm in elementary operations, 32 bits, rounded once at the end."""
    x = s["x"].detach().float()
    R, C = x.shape
    G = s["G"]
    w, b = s["weight"].detach().view(G, 1, C), s["bias"].detach().view(G, 1, C)
    mean = x.sum(-1, keepdim=True) / C
    xc = x - mean
    rstd = 1.0 / torch.sqrt((xc * xc).sum(-1, keepdim=True) / C + EPS)
    xh = xc * rstd
    out = {"y": (xh.view(G, R // G, C) * w + b).view(R, C).to(s["out_dtype"])}
    if s["kind"] == "norm":
        dy = s["dy"].float()
        g = (dy.view(G, R // G, C) * w).view(R, C)
        dx = rstd * (g - g.sum(-1, keepdim=True) / C - xh * ((g * xh).sum(-1, keepdim=True) / C))
        out["dx"] = dx.to(s["x"].dtype)
        out["dweight"] = (dy * xh).view(G, R // G, C).sum(1).view(s["weight"].shape)
        out["dbias"] = dy.view(G, R // G, C).sum(1).view(s["bias"].shape)
    return out


# ------------------------------------------------------------------ one pass

def run(state):
    s = state
    if not own:
        return _plain_attention(s) if _attends(s) else _plain_norm(s)
    lib = _mw()
    if s["kind"] == "train":
        o = lib.CrossAttention.apply(s["q"], s["k"], s["v"], s["kv_len"])
        dq, dk, dv = torch.autograd.grad(o, (s["q"], s["k"], s["v"]), s["do"])
        return {"o": o.detach(), "dq": dq, "dk": dk, "dv": dv}
    if _attends(s):
        o, lse = lib.mw_xattn_fwd(s["q"], s["k"], s["v"], s["kv_len"], need_lse=s["lse"])
        return {"o": o, "lse": lse}
    if s["kind"] == "norm":
        y = lib.LayerNorm.apply(s["x"], s["weight"], s["bias"], EPS, s["out_dtype"])
        dx, dw, db = torch.autograd.grad(y, (s["x"], s["weight"], s["bias"]), s["dy"])
        return {"y": y.detach(), "dx": dx, "dweight": dw, "dbias": db}
    y, _, _ = lib.mw_layernorm_fwd(s["x"], s["weight"], s["bias"], EPS, out_dtype=s["out_dtype"], need_stats=False)
    return {"y": y}


# ------------------------------------------------------------------ the same in 64 bits

def exact(case, seed):
    c, x = case, _inputs(case, seed)
    if not _attends(c):
        x = {n: t.to(torch.float64) for n, t in x.items()}
        G, C = c["G"], c["C"]
        x3 = x["x"].view(G, -1, C)
        w, b = x["weight"].view(G, 1, C), x["bias"].view(G, 1, C)
        var, mean = torch.var_mean(x3, dim=-1, correction=0, keepdim=True)
        sd = (var + EPS).sqrt()
        xh = (x3 - mean) / sd
        out = {"y": torch.addcmul(b, xh, w).view(c["R"], C)}
        if c["kind"] == "norm":
            dy = x["dy"].view(G, -1, C)
            out["dweight"] = torch.einsum("grc,grc->gc", dy, xh).view(x["weight"].shape)
            out["dbias"] = dy.sum(1).view(x["bias"].shape)
            dxh = dy * w
            out["dx"] = ((dxh - dxh.mean(-1, keepdim=True) - xh * (dxh * xh).mean(-1, keepdim=True)) / sd).view(c["R"], C)
            out = {n: out[n] for n in ("y", "dx", "dweight", "dbias")}
        return out
    B, H, M, d = x["q"].shape
    share = H // c["Hkv"]
    lens = _lens(c, seed)
    train = c["kind"] == "train"

    def zeros(t):
        return torch.zeros(t.shape, dtype=torch.float64, device="cuda")

    o, lse = zeros(x["q"]), torch.full((B, H, M), -math.inf, dtype=torch.float64, device="cuda")
    if train:
        dq, dk, dv = zeros(x["q"]), zeros(x["k"]), zeros(x["v"])
    for b in range(B):
        n = lens[b]
        if n == 0:
            continue
        for h in range(H):
            q = x["q"][b, h].double()
            k, v = (x[t][b, h // share, :n].double() for t in ("k", "v"))
            s = q @ k.T / math.sqrt(d)
            lse[b, h] = torch.logsumexp(s, -1)
            p = s.sub_(lse[b, h][:, None]).exp_()
            o[b, h] = p @ v
            if train:
                g = x["do"][b, h].double()
                dv[b, h // share, :n] += p.T @ g
                ds = g @ v.T
                ds -= torch.einsum("md,md->m", g, o[b, h])[:, None]
                ds *= p
                dq[b, h] = ds @ k / math.sqrt(d)
                dk[b, h // share, :n] += ds.T @ q / math.sqrt(d)
    if train:
        return {"o": o, "dq": dq, "dk": dk, "dv": dv}
    return {"o": o, "lse": lse if c["lse"] else None}
