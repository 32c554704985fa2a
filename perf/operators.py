"""Cases of the text encoder's entry and of its 8-bit serving path: what is measured, and the same operators in plain form.

Kinds of case
  embedding   embedding(tokens, weight, scale): rows of a table, scaled; in training also the table's gradient
  norm        add_rms_norm(x, residual, weight): h = x + residual and the root-mean-square norm of h; in training
              also the gradients of x, of the residual stream and of the gains
  norm_fp8    add_rms_norm_fp8 / rms_norm_fp8: the norm's rows in 8 bits (e4m3) with one scale a row
  quantize    quantize_rows(x): a tensor's rows in that form (an attention's output, a weight when it is laid out)
  linear      linear_fp8(x8, x_scale, w8, w_scale, bias): the product that reads two such tensors

With residual "f32" the residual stream is held in 32 bits, with "same" in the format of x.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-6
F8 = torch.float8_e4m3fn
F8_MAX = 448.0
LEAST = 2.0 ** -96  # a row's largest magnitude counts as at least this


# ------------------------------------------------------------------------------------------------ cases
def _embedding(captions, length, V, D, table="bf16", out="bf16", ignored=False, train=True):
    return {"kind": "embedding", "captions": captions, "length": length, "V": V, "D": D, "table": table, "out": out,
            "ignored": ignored, "train": train}


def _norm(M, D, dtype="bf16", residual="same", train=True):
    return {"kind": "norm", "M": M, "D": D, "dtype": dtype, "residual": residual, "train": train}


def _norm_fp8(M, D, dtype="bf16", residual="same"):
    return {"kind": "norm_fp8", "M": M, "D": D, "dtype": dtype, "residual": residual}


def _quantize(M, D, dtype="bf16"):
    return {"kind": "quantize", "M": M, "D": D, "dtype": dtype}


def _linear(M, N, K, dtype="bf16", bias=True):
    return {"kind": "linear", "M": M, "N": N, "K": K, "dtype": dtype, "bias": bias}


def listed():
    return [
        # one token of a prompt that is being written: launch and latency
        dict(_embedding(1, 1, 50000, 512, train=False), name="embed_one"),
        # the captions of a contrastive batch: 2048 of 77 tokens, most of them the padding after a short sentence
        dict(_embedding(2048, 77, 50000, 512), name="embed_captions_train"),
        # a small ragged batch under mixed precision: table and gradient in 32 bits, rows in fp16, slots without a token
        dict(_embedding(37, 61, 10007, 776, table="f32", out="f16", ignored=True), name="embed_ragged_train"),
        # one token in a wide layer: latency again
        dict(_norm(1, 4096, train=False), name="norm_one"),
        # the same captions in front of a text encoder's attention
        dict(_norm(2048 * 77, 512), name="norm_captions_train"),
        # an odd number of tokens of ViT-H's width and one chunk more, the residual stream in 32 bits
        dict(_norm(4999, 1288, dtype="f16", residual="f32"), name="norm_ragged_f32_train"),
        # a few tokens that are answered at once
        dict(_norm_fp8(7, 4096), name="norm_fp8_few"),
        # the tokens of 32 video clips (1568 each) on their way into an 8-bit joint projection
        dict(_norm_fp8(32 * 1568, 768), name="norm_fp8_video"),
        # the output of the attention over 8 clips, on its way into an 8-bit output projection
        dict(_quantize(8 * 1568, 1024, dtype="f16"), name="quantize_attention"),
        # one token through a wide projection: the weight's bytes
        dict(_linear(1, 6144, 4096, bias=False), name="linear_one"),
        # two clips of 784 tokens and a class token each, through a projection of odd width
        dict(_linear(2 * 785, 1000, 1280, dtype="f16"), name="linear_ragged"),
        # the joint query/key/value projection of 32 clips
        dict(_linear(32 * 1568, 3 * 768, 768), name="linear_video_qkv"),
    ]


MOST_BYTES = 6.0e8      # no drawn case costs more than the largest listed ones
MOST_FLOPS = 1.7e11


def _log_int(rng, lo, hi, step=1):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step
    return max(-(-lo // step) * step, min(hi // step * step, n))


def draw(rng):
    kind = rng.choice(("embedding", "embedding", "norm", "norm", "norm_fp8", "quantize", "linear", "linear"))
    while True:
        if kind == "embedding":
            out = rng.choice(("bf16", "f16"))
            c = _embedding(_log_int(rng, 1, 4096), rng.randint(1, 128), _log_int(rng, 8, 130000), _log_int(rng, 64, 4096, 8),
                           table=rng.choice((out, out, "f32")), out=out, ignored=rng.random() < 0.3, train=rng.random() < 0.75)
        elif kind == "norm":
            c = _norm(_log_int(rng, 1, 160000), _log_int(rng, 64, 8192, 8), dtype=rng.choice(("bf16", "f16")),
                      residual=rng.choice(("same", "same", "f32")), train=rng.random() < 0.75)
        elif kind == "norm_fp8":
            c = _norm_fp8(_log_int(rng, 1, 160000), _log_int(rng, 64, 8192, 16), dtype=rng.choice(("bf16", "f16")),
                          residual=rng.choice(("same", "same", "f32", "none")))
        elif kind == "quantize":
            c = _quantize(_log_int(rng, 1, 160000), _log_int(rng, 64, 8192, 16), dtype=rng.choice(("bf16", "f16")))
        else:
            c = _linear(_log_int(rng, 1, 50176), _log_int(rng, 64, 8192, 8), _log_int(rng, 64, 8192, 16),
                        dtype=rng.choice(("bf16", "f16")), bias=rng.random() < 0.5)
        w = work(c)
        if w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS:
            return c


# ----------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _sentence_lengths(captions, length):
    """How many of a caption's slots hold words: spoken descriptions are short, the rest is padding."""
    return max(1, length // 10), max(1, (length * 2) // 5)


def _tokens(g, c):
    """Captions: words by rank (each octave of the ranks as likely as the next), an end mark, then padding (token 0) or,
    where slots are `ignored`, -1."""
    B, L, V = c["captions"], c["length"], c["V"]
    u = torch.rand((B, L), generator=g, device="cuda", dtype=torch.float64)
    words = (torch.exp(u * math.log(V)).long() - 1).clamp_(0, V - 1)
    lo, hi = _sentence_lengths(B, L)
    n = torch.randint(lo, hi + 1, (B, 1), generator=g, device="cuda")
    at = torch.arange(L, device="cuda")[None]
    t = torch.where(at < n, words, torch.full_like(words, -1 if c["ignored"] else 0))
    return torch.where(at == n, torch.full_like(t, V - 1), t)


def _rows8(g, rows, K, scale):
    """Rows in 8 bits with their scales, as quantised activations or weights are: each row fills the format's range."""
    x = torch.randn((rows, K), generator=g, device="cuda") * scale
    s = x.abs().amax(1).clamp_min(LEAST) / F8_MAX
    return (x / s[:, None]).to(F8), s


def prepare(case, seed):
    g, c, k = _generator(seed), case, case["kind"]
    if k == "embedding":
        s = {"tokens": _tokens(g, c), "weight": _normal(g, (c["V"], c["D"]), DTYPES[c["table"]], 0.02),
             "scale": math.sqrt(c["D"])}
        if c["train"]:
            s["dy"] = _normal(g, (c["captions"], c["length"], c["D"]), DTYPES[c["out"]])
            s["weight"].requires_grad_(True)
    elif k in ("norm", "norm_fp8"):
        dt = DTYPES[c["dtype"]]
        rt = torch.float32 if c["residual"] == "f32" else dt
        s = {"x": _normal(g, (c["M"], c["D"]), dt), "weight": 1 + _normal(g, (c["D"],), torch.float32, 0.1)}
        if c["residual"] != "none":
            s["residual"] = _normal(g, (c["M"], c["D"]), rt, 2.0)
        if c.get("train"):
            s["dy"], s["dh"] = _normal(g, (c["M"], c["D"]), dt), _normal(g, (c["M"], c["D"]), rt)
            for n in ("x", "residual", "weight"):
                s[n].requires_grad_(True)
    elif k == "quantize":
        s = {"x": _normal(g, (c["M"], c["D"]), DTYPES[c["dtype"]])}
    else:
        x8, xs = _rows8(g, c["M"], c["K"], 1.0)
        w8, ws = _rows8(g, c["N"], c["K"], c["K"] ** -0.5)
        s = {"x8": x8, "x_scale": xs, "w8": w8, "w_scale": ws,
             "bias": _normal(g, (c["N"],), torch.float32, 0.1) if c["bias"] else None}
    return dict(s, case=c)


# ------------------------------------------------------------------------------------------------- work
def _distinct(c):
    """Expected number of different rows that the captions' tokens name."""
    V, L = c["V"], c["length"]
    lo, hi = _sentence_lengths(c["captions"], L)
    words = c["captions"] * min(L, (lo + hi) / 2)
    rank = np.arange(V, dtype=np.float64)
    p = np.log((rank + 2) / (rank + 1)) / math.log(max(V, 2))
    return max(1.0, min(float(V), float(-np.expm1(words * np.log1p(-np.minimum(p, 1 - 1e-12))).sum())))


def work(case):
    c, k = case, case["kind"]
    if k == "embedding":
        n, D, t = c["captions"] * c["length"], c["D"], BYTES[c["table"]]
        b, f = n * 8 + _distinct(c) * D * t + n * D * 2, n * D
        if c["train"]:  # the gradient of the rows, and a gradient for every row of the table
            b, f = b + n * D * 2 + c["V"] * D * t, f + 2 * n * D
    elif k in ("norm", "norm_fp8"):
        n, D = c["M"], c["D"]
        r = {"same": 2, "f32": 4, "none": 0}[c["residual"]]
        b, f = n * D * (2 + r + r + (2 if k == "norm" else 1)) + 4 * D + (0 if k == "norm" else 4 * n), 6 * n * D
        if c.get("train"):  # the gradients of both outputs in, those of both inputs and of the gains out
            b, f = b + n * D * (2 + r + 2 + (4 if r == 4 else 0)) + 4 * D, f + 12 * n * D
    elif k == "quantize":
        b, f = c["M"] * (c["D"] * 3 + 4), 3 * c["M"] * c["D"]
    else:
        M, N, K = c["M"], c["N"], c["K"]
        b, f = (M + N) * (K + 4) + M * N * 2 + (4 * N if c["bias"] else 0), 2.0 * M * N * K
    return {"bytes": float(b), "flops": float(f)}


# ------------------------------------------------------------------------------------------------- runs
_ops = None


def _entry_points():
    global _ops
    if _ops is None:
        from paper_2309_16669_amd import autograd
        _ops = autograd
    return _ops


def _run_own(s):
    c, ag = s["case"], _ops or _entry_points()
    k = c["kind"]
    if k == "embedding":
        y = ag.embedding(s["tokens"], s["weight"], s["scale"], DTYPES[c["out"]])
        if not c["train"]:
            return {"y": y}
        (dw,) = torch.autograd.grad(y, (s["weight"],), s["dy"])
        return {"y": y, "dweight": dw}
    if k == "norm":
        y, h = ag.add_rms_norm(s["x"], s["residual"], s["weight"], EPS)
        if not c["train"]:
            return {"y": y, "h": h}
        dx, dr, dw = torch.autograd.grad((y, h), (s["x"], s["residual"], s["weight"]), (s["dy"], s["dh"]))
        return {"y": y, "h": h, "dx": dx, "dresidual": dr, "dweight": dw}
    if k == "norm_fp8":
        if c["residual"] == "none":
            y8, scale = ag.rms_norm_fp8(s["x"], s["weight"], EPS)
            return {"y8": y8, "scale": scale}
        y8, scale, h = ag.add_rms_norm_fp8(s["x"], s["residual"], s["weight"], EPS)
        return {"y8": y8, "scale": scale, "h": h}
    if k == "quantize":
        x8, scale = ag.quantize_rows(s["x"])
        return {"x8": x8, "scale": scale}
    return {"y": ag.linear_fp8(s["x8"], s["x_scale"], s["w8"], s["w_scale"], s["bias"], DTYPES[c["dtype"]])}


def _plain_rows8(y):
    scale = y.abs().amax(1).clamp_min(LEAST) / F8_MAX
    return (y / scale[:, None]).to(F8), scale


@torch.no_grad()
def _run_plain(s):
    c = s["case"]
    k = c["kind"]
    if k == "embedding":
        t, w = s["tokens"].reshape(-1), s["weight"]
        V, D = w.shape
        real = (t >= 0) & (t < V)
        at = torch.where(real, t, torch.zeros_like(t))
        y = torch.where(real[:, None], w[at].float() * s["scale"], torch.zeros((), device=w.device))
        out = {"y": y.to(DTYPES[c["out"]]).reshape(*s["tokens"].shape, D)}
        if c["train"]:
            # by sorted tokens, as differences of running sums in 64 bits: a row's sum may be long (the padding's)
            name, order = torch.sort(torch.where(real, t, V))
            sums = torch.cumsum(s["dy"].reshape(-1, D)[order].double().t().contiguous(), 1)
            ends = torch.searchsorted(name, torch.arange(V, device=w.device), right=True)
            upto = torch.where(ends > 0, sums[:, (ends - 1).clamp_min(0)], torch.zeros((), dtype=sums.dtype, device=w.device))
            dw = torch.diff(upto, dim=1, prepend=torch.zeros_like(upto[:, :1])).t().contiguous()
            out["dweight"] = (dw * s["scale"]).to(w.dtype)
        return out
    if k in ("norm", "norm_fp8"):
        x, r, w = s["x"], s.get("residual"), s["weight"]
        h = x if r is None else (x.float() + r.float()).to(r.dtype)  # the stream's format: the norm is of what it holds
        hf = h.float()
        rstd = 1.0 / torch.sqrt((hf * hf).mean(1, keepdim=True) + EPS)
        xhat = hf * rstd
        if k == "norm_fp8":
            y8, scale = _plain_rows8(xhat * w)
            return {"y8": y8, "scale": scale} if r is None else {"y8": y8, "scale": scale, "h": h}
        out = {"y": (xhat * w).to(x.dtype), "h": h}
        if c["train"]:
            dy = s["dy"].float()
            g = dy * w
            d = rstd * (g - xhat * (g * xhat).mean(1, keepdim=True)) + s["dh"].float()
            out |= {"dx": d.to(x.dtype), "dresidual": d.to(r.dtype), "dweight": (dy * xhat).sum(0)}
        return out
    if k == "quantize":
        x8, scale = _plain_rows8(s["x"].float())
        return {"x8": x8, "scale": scale}
    y = s["x8"].float() @ s["w8"].float().t() * s["x_scale"][:, None] * s["w_scale"]
    return {"y": (y if s["bias"] is None else y + s["bias"]).to(DTYPES[c["dtype"]])}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------ exact
def _to_e4m3(v):
    """The nearest e4m3 value of each number (ties to the even one), in 64 bits: steps of an eighth of the number's power of
    two, of 2^-9 below 2^-6, up to 448."""
    a = v.abs()
    _, e = torch.frexp(a)
    step = torch.ldexp(torch.ones_like(a), torch.clamp(e - 4, min=-9))
    return torch.sign(v) * torch.clamp(torch.round(a / step) * step, max=F8_MAX)


def _exact_rows8(y):
    big = torch.clamp(torch.max(torch.abs(y), dim=-1).values, min=LEAST)
    return _to_e4m3(y * (F8_MAX / big).unsqueeze(-1)), big / F8_MAX


@torch.no_grad()
def exact(case, seed):
    c, s = case, prepare(case, seed)
    k = c["kind"]
    if k == "embedding":
        flat, V, D = s["tokens"].flatten(), c["V"], c["D"]
        table = torch.cat([s["weight"].detach().double() * s["scale"], torch.zeros((1, D), dtype=torch.float64, device="cuda")])
        row = torch.where((flat < 0) | (flat >= V), V, flat)
        out = {"y": table.index_select(0, row).view(c["captions"], c["length"], D)}
        if c["train"]:
            total = torch.zeros((V + 1, D), dtype=torch.float64, device="cuda")
            total.index_add_(0, row, s["dy"].view(-1, D).double())
            out["dweight"] = total[:V] * s["scale"]
        return out
    if k in ("norm", "norm_fp8"):
        h = s["x"].detach().double()
        if "residual" in s:
            h = (h + s["residual"].detach().double()).to(s["residual"].dtype).double()
        w, D = s["weight"].detach().double(), c["D"]
        r = torch.rsqrt(torch.einsum("md,md->m", h, h) / D + EPS)[:, None]
        y = h * w * r
        if k == "norm_fp8":
            y8, scale = _exact_rows8(y)
            return {"y8": y8, "scale": scale} if c["residual"] == "none" else {"y8": y8, "scale": scale, "h": h}
        out = {"y": y, "h": h}
        if c["train"]:
            dy = s["dy"].double()
            # y_d = w_d h_d r and dr/dh_e = -r^3 h_e / D
            along = torch.einsum("md,d,md->m", dy, w, h)[:, None]
            d = dy * w * r - h * along * r ** 3 / D + s["dh"].double()
            out |= {"dx": d, "dresidual": d, "dweight": torch.einsum("md,md->d", dy, h * r)}
        return out
    if k == "quantize":
        x8, scale = _exact_rows8(s["x"].double())
        return {"x8": x8, "scale": scale}
    a = s["x8"].double() * s["x_scale"].double().unsqueeze(1)
    b = s["w8"].double() * s["w_scale"].double().unsqueeze(1)
    y = torch.mm(a, b.t().contiguous())
    return {"y": y + s["bias"].double() if c["bias"] else y}
