"""Cases of rotary positions, of attention over sequences of different lengths and of the loss over a vocabulary: what is
measured, and the same operators in plain form.

Kinds of case
  rotary     rotary(q, k, positions, freqs, sections): queries and keys turned by the angles of their positions, one to
             three axes (time, height, width); in training also the gradients of both
  attention  attention_ragged(q, k, v, offsets, offsets_k, causal): sequences of different lengths one after the other,
             query heads that share key heads, the last query beside the last key under `causal`; in training also the
             gradients of all three
  loss       linear_cross_entropy(x, weight, targets): softmax cross entropy of the logits scale * x weight^T, which are
             not kept; in training the mean and the gradients of x and weight, else one loss a row
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


# ------------------------------------------------------------------------------------------------ cases
def _rotary(clips, frames, height, width, Hq, Hk, d, dtype="bf16", turned=1.0, interleaved=False, start=0, train=True):
    """clips of frames x height x width tokens that share their positions; height 0: text, one axis.  `turned`: the share of
    a head's channels that turn; `start`: the first position."""
    return {"kind": "rotary", "clips": clips, "frames": frames, "height": height, "width": width, "Hq": Hq, "Hk": Hk, "d": d,
            "dtype": dtype, "turned": turned, "interleaved": interleaved, "start": start, "train": train}


def _attention(S, lo, hi, Hq, Hk, d, dtype="bf16", causal=True, before=0, single=False, empty=False, lengths=1, train=True):
    """S sequences of lo to hi queries (their logarithm spread evenly), behind up to `before` earlier keys each; `single`: one
    query each, and lo to hi keys; `empty`: some sequences have no token, and some fewer keys than queries."""
    return {"kind": "attention", "S": S, "lo": lo, "hi": hi, "Hq": Hq, "Hk": Hk, "d": d, "dtype": dtype, "causal": causal,
            "before": before, "single": single, "empty": empty, "lengths": lengths, "train": train}


def _loss(T, V, D, dtype="bf16", pairs=False, ignored=0.0, scale=1.0, train=True):
    """T rows against V rows of width D; `pairs`: row i belongs to row i (a contrastive batch), else targets are words, a
    share `ignored` of them none."""
    return {"kind": "loss", "T": T, "V": V, "D": D, "dtype": dtype, "pairs": pairs, "ignored": ignored, "scale": scale,
            "train": train}


def listed():
    return [
        # the next token of a sentence that is being written: launch and latency
        dict(_rotary(1, 1, 0, 0, 16, 4, 64, start=20000, train=False), name="rotary_one"),
        # the tokens of 32 video clips, 8 x 14 x 14 each, on three axes
        dict(_rotary(32, 8, 14, 14, 12, 12, 64), name="rotary_video_train"),
        # odd numbers of frames and patches, heads of 80 channels of which 48 turn, neighbouring pairs, fp16
        dict(_rotary(3, 7, 13, 17, 16, 8, 80, dtype="f16", turned=0.6, interleaved=True), name="rotary_odd_train"),
        # 24 sentences that each get their next token, up to 9000 tokens behind it: the cache's bytes
        dict(_attention(24, 100, 9000, 32, 8, 128, single=True, lengths=3, train=False), name="attn_tokens"),
        # a text-encoder layer on the 2048 captions of a contrastive batch, without their padding
        dict(_attention(2048, 6, 77, 8, 8, 64, lengths=5), name="attn_captions_train"),
        # 16 videos of different lengths, from one frame to 16, every token sees its whole video
        dict(_attention(16, 196, 3136, 12, 12, 64, causal=False, lengths=7), name="attn_videos_train"),
        # prompts of a text decoder, four query heads for a key head, answered at once
        dict(_attention(6, 500, 8000, 32, 8, 128, dtype="f16", lengths=9, train=False), name="attn_prompts"),
        # text behind the tokens of a video, odd lengths, some empty, eight query heads for a key head
        dict(_attention(37, 3, 700, 16, 2, 80, before=400, empty=True, lengths=11), name="attn_shared_train"),
        # five words of a sentence scored
        dict(_loss(5, 50000, 512, train=False), name="loss_few"),
        # a contrastive batch of 2048 pairs
        dict(_loss(2048, 2048, 512, pairs=True, scale=14.3), name="loss_pairs_train"),
        # odd sizes in fp16, a third of the slots without a word
        dict(_loss(997, 10007, 776, dtype="f16", ignored=0.33), name="loss_odd_train"),
        # the words of a captioning batch over the text encoder's vocabulary
        dict(_loss(16384, 50000, 768, ignored=0.05), name="loss_vocab_train"),
    ]


MOST_BYTES = 4.0e8      # no drawn case costs more than the largest listed ones
MOST_FLOPS = {"rotary": 1.0e12, "attention": 4.5e11, "loss": 3.7e12}


def _log_int(rng, lo, hi, step=1):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step
    return max(-(-lo // step) * step, min(hi // step * step, n))


def _draw_attention(rng):
    dtype, lengths = rng.choice(("bf16", "bf16", "f16")), rng.randint(1, 10 ** 6)
    d = rng.choice((64, 64, 80, 128))
    Hk = rng.choice((1, 2, 4, 8, 12))
    Hq = Hk * rng.choice((1, 2, 4, 8) if Hk < 8 else (1, 2))
    pick = rng.random()
    if pick < 0.25:     # single tokens
        hi = _log_int(rng, 64, 60000)
        return _attention(_log_int(rng, 1, 256), max(1, hi // 40), hi, Hq, Hk, d, dtype, rng.random() < 0.5, single=True,
                          lengths=lengths, train=False)
    if pick < 0.5:      # captions
        hi = rng.randint(8, 128)
        return _attention(_log_int(rng, 1, 4096), max(1, hi // 12), hi, Hq, Hk, d, dtype, True, empty=rng.random() < 0.3,
                          lengths=lengths, train=rng.random() < 0.75)
    hi = _log_int(rng, 100, 9000)   # prompts, videos, text behind other tokens
    return _attention(_log_int(rng, 1, 64), max(1, hi // rng.choice((2, 16))), hi, Hq, Hk, d, dtype, rng.random() < 0.6,
                      before=rng.choice((0, 0, 600)), empty=rng.random() < 0.3, lengths=lengths, train=rng.random() < 0.7)


def draw(rng):
    kind = rng.choice(("rotary", "attention", "attention", "loss"))
    while True:
        if kind == "rotary":
            text = rng.random() < 0.4
            Hk = rng.choice((1, 2, 4, 8, 12, 16))
            d = rng.choice((64, 64, 80, 128))
            c = _rotary(_log_int(rng, 1, 256), _log_int(rng, 1, 20000) if text else rng.randint(1, 32),
                        0 if text else rng.randint(1, 24), 0 if text else rng.randint(1, 24), Hk * rng.choice((1, 1, 2, 4)), Hk, d,
                        rng.choice(("bf16", "f16")), turned=rng.choice((1.0, 1.0, 0.6)), interleaved=rng.random() < 0.4,
                        start=rng.choice((0, 0, 1000000)), train=rng.random() < 0.7)
        elif kind == "attention":
            c = _draw_attention(rng)
        else:
            pairs = rng.random() < 0.25
            T = _log_int(rng, 1, 8192 if pairs else 16384)
            c = _loss(T, T if pairs else _log_int(rng, 2, 130000), _log_int(rng, 64, 2048, 8), rng.choice(("bf16", "bf16", "f16")),
                      pairs=pairs, ignored=0.0 if pairs else rng.choice((0.0, 0.3)), scale=rng.choice((1.0, 14.3)) if pairs else 1.0,
                      train=rng.random() < 0.75)
        w = work(c)
        if w["bytes"] <= MOST_BYTES and 0 < w["flops"] <= MOST_FLOPS[kind]:
            return c


# ---------------------------------------------------------------------------------------------- lengths
def _lengths(c):
    """Queries and keys of each sequence."""
    rng, nq, nk = random.Random(c["lengths"]), [], []
    for _ in range(c["S"]):
        n = _log_int(rng, c["lo"], c["hi"])
        if c["single"]:
            nq.append(1)
            nk.append(n)
            continue
        earlier = rng.randint(0, c["before"])
        if c["empty"] and rng.random() < 0.15:
            nq.append(rng.choice((0, n)))
            nk.append(rng.choice((0, n // 2)))
        else:
            nq.append(n)
            nk.append(n + earlier)
    return nq, nk


def _seen(nq, nk, causal):
    """How many (query, key) pairs a sequence has: query i sees the keys up to i + nk - nq."""
    if not causal:
        return nq * nk
    first = max(0, nq - nk)     # queries before it see nothing
    rows = nq - first
    return rows * (nk - nq + first + 1) + rows * (rows - 1) // 2


# ----------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _turned_pairs(c):
    return int(c["d"] * c["turned"]) // 16 * 8


def _sections(c):
    """Pairs of each axis: time, height, width; text has one axis."""
    n = _turned_pairs(c)
    if c["height"] == 0:
        return (n,)
    a = n // 3
    return (n - 2 * a, a, a)


def _offsets(lengths):
    total, out = 0, [0]
    for n in lengths:
        total += n
        out.append(total)
    return out


def prepare(case, seed):
    g, c, k = _generator(seed), case, case["kind"]
    dt = DTYPES[c["dtype"]]
    if k == "rotary":
        n = c["frames"] * max(1, c["height"]) * max(1, c["width"])
        s = {"q": _normal(g, (c["clips"], n, c["Hq"], c["d"]), dt), "k": _normal(g, (c["clips"], n, c["Hk"], c["d"]), dt)}
        freqs = []
        for m in _sections(c):  # each axis its own spectrum, slowest last
            freqs += [10000.0 ** (-j / m) for j in range(m)]
        s["freqs"] = torch.tensor(freqs, dtype=torch.float32, device="cuda")
        begin = c["start"] + seed % 7
        if c["height"] == 0:
            s["sections"], s["positions"] = None, torch.arange(begin, begin + n, device="cuda", dtype=torch.int32)
        else:
            s["sections"] = _sections(c)
            grid = torch.meshgrid(*(torch.arange(m, device="cuda", dtype=torch.int32) for m in
                                    (c["frames"], c["height"], c["width"])), indexing="ij")
            s["positions"] = torch.stack([x.reshape(-1) for x in grid]) + begin
        if c["train"]:
            s["dq"], s["dk"] = _normal(g, tuple(s["q"].shape), dt), _normal(g, tuple(s["k"].shape), dt)
            s["q"].requires_grad_(True)
            s["k"].requires_grad_(True)
    elif k == "attention":
        nq, nk = _lengths(c)
        same = nq == nk
        s = {"q": _normal(g, (sum(nq), c["Hq"], c["d"]), dt), "k": _normal(g, (sum(nk), c["Hk"], c["d"]), dt),
             "v": _normal(g, (sum(nk), c["Hk"], c["d"]), dt)}
        s["offsets"] = torch.tensor(_offsets(nq), dtype=torch.int32, device="cuda")
        s["offsets_k"] = None if same else torch.tensor(_offsets(nk), dtype=torch.int32, device="cuda")
        if c["train"]:
            s["do"] = _normal(g, tuple(s["q"].shape), dt)
            for n in ("q", "k", "v"):
                s[n].requires_grad_(True)
    else:
        T, V, D = c["T"], c["V"], c["D"]
        if c["pairs"]:      # two embeddings of unit length, the right one nearer than the others
            a, b = (torch.nn.functional.normalize(torch.randn((n, D), generator=g, device="cuda")) for n in (T, V))
            s = {"x": torch.nn.functional.normalize(a + 0.6 * b).to(dt), "weight": b.to(dt),
                 "targets": torch.arange(T, device="cuda")}
        else:
            s = {"x": _normal(g, (T, D), dt), "weight": _normal(g, (V, D), dt, 2.0 * D ** -0.5)}
            u = torch.rand((T,), generator=g, device="cuda", dtype=torch.float64)
            t = (torch.exp(u * math.log(V)).long() - 1).clamp_(0, V - 1)
            out = torch.rand((T,), generator=g, device="cuda") < c["ignored"]
            s["targets"] = torch.where(out, -100, t)
        if c["train"]:
            s["x"].requires_grad_(True)
            s["weight"].requires_grad_(True)
    return dict(s, case=c)


# ------------------------------------------------------------------------------------------------- work
def work(case):
    c, k = case, case["kind"]
    if k == "rotary":
        tokens = c["frames"] * max(1, c["height"]) * max(1, c["width"])
        n = c["clips"] * tokens * (c["Hq"] + c["Hk"]) * c["d"]
        b, f = 4 * n + 4 * tokens * (3 if c["height"] else 1), 3 * n
        return {"bytes": float(b if not c["train"] else 2 * b), "flops": float(f if not c["train"] else 2 * f)}
    if k == "attention":
        nq, nk = _lengths(c)
        pairs = sum(_seen(a, b, c["causal"]) for a, b in zip(nq, nk))
        q, kv = 2 * sum(nq) * c["Hq"] * c["d"], 2 * sum(nk) * c["Hk"] * c["d"]
        b, f = 2 * q + 2 * kv, 4.0 * pairs * c["Hq"] * c["d"]
        if c["train"]:      # backward: the outputs' gradient in, three out; scores, dP, dQ, dK, dV
            b, f = b + 2 * q + 2 * kv, f + 10.0 * pairs * c["Hq"] * c["d"]
        return {"bytes": float(b), "flops": float(f)}
    T, V, D = c["T"], c["V"], c["D"]
    b, f = 2 * (T + V) * D + 8 * T, 2.0 * T * V * D
    return {"bytes": float(b + (4 * T if not c["train"] else 2 * (T + V) * D)), "flops": f if not c["train"] else 3 * f}


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
    if k == "rotary":
        q, kk = ag.rotary(s["q"], s["k"], s["positions"], s["freqs"], s["sections"], c["interleaved"])
        if not c["train"]:
            return {"q": q, "k": kk}
        dq, dk = torch.autograd.grad((q, kk), (s["q"], s["k"]), (s["dq"], s["dk"]))
        return {"q": q, "k": kk, "dq": dq, "dk": dk}
    if k == "attention":
        o = ag.attention_ragged(s["q"], s["k"], s["v"], s["offsets"], s["offsets_k"], causal=c["causal"])
        if not c["train"]:
            return {"o": o}
        dq, dk, dv = torch.autograd.grad(o, (s["q"], s["k"], s["v"]), s["do"])
        return {"o": o, "dq": dq, "dk": dk, "dv": dv}
    if not c["train"]:
        return {"loss": ag.linear_cross_entropy(s["x"], s["weight"], s["targets"], scale=c["scale"], reduction="none")}
    loss = ag.linear_cross_entropy(s["x"], s["weight"], s["targets"], scale=c["scale"])
    dx, dw = torch.autograd.grad(loss, (s["x"], s["weight"]))
    return {"loss": loss, "dx": dx, "dweight": dw}


def _plain_turn(x, cos, sin, interleaved, dtype):
    """Pairs of x turned: cos and sin [tokens, pairs]."""
    m = cos.shape[-1]
    xf, cos, sin = x.float(), cos[:, None], sin[:, None]
    turned, rest = xf[..., :2 * m], xf[..., 2 * m:]
    if interleaved:
        a, b = turned[..., 0::2], turned[..., 1::2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
    else:
        a, b = turned[..., :m], turned[..., m:]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    return torch.cat((y, rest), dim=-1).to(dtype)


MOST_SCORES = 1 << 28   # scores that the plain form holds at a time


def _plain_attention(s):
    """Sequences padded to the longest of as many neighbours as fit, in 32 bits."""
    c, q, k, v = s["case"], s["q"], s["k"], s["v"]
    (Hq, d), Hk = q.shape[1:], k.shape[1]
    G, scale = Hq // Hk, 1.0 / math.sqrt(d)
    nq, nk = _lengths(c)
    oq, ok = _offsets(nq), _offsets(nk)
    out = {"o": torch.zeros_like(q)}
    if c["train"]:
        out |= {"dq": torch.zeros_like(q), "dk": torch.zeros_like(k), "dv": torch.zeros_like(v)}
    begin = 0
    while begin < len(nq):
        end, mq, mk = begin, 0, 0
        while end < len(nq):
            a, b = max(mq, nq[end]), max(mk, nk[end])
            if end > begin and (end - begin + 1) * Hq * a * b > MOST_SCORES:
                break
            end, mq, mk = end + 1, a, b
        n = end - begin
        if mq and mk:
            def rows(offsets, lengths, width):
                at = torch.arange(width)[None]
                live = at < torch.tensor(lengths[begin:end])[:, None]
                index = torch.where(live, at + torch.tensor(offsets[begin:end])[:, None], 0)
                return live.cuda(), index.cuda()

            live_q, index_q = rows(oq, nq, mq)
            live_k, index_k = rows(ok, nk, mk)
            late = (torch.tensor(nk[begin:end]) - torch.tensor(nq[begin:end])).cuda()
            see = live_q[:, :, None] & live_k[:, None, :]
            if c["causal"]:
                i, j = torch.arange(mq, device="cuda")[None, :, None], torch.arange(mk, device="cuda")[None, None]
                see = see & (j <= i + late[:, None, None])

            def heads_q(t):     # [n Hk, G mq, d]
                t = t[index_q].float() * live_q[..., None, None]
                return t.view(n, mq, Hk, G, d).permute(0, 2, 3, 1, 4).reshape(n * Hk, G * mq, d)

            def heads_k(t):     # [n Hk, mk, d]
                t = t[index_k].float() * live_k[..., None, None]
                return t.permute(0, 2, 1, 3).reshape(n * Hk, mk, d)

            def back_q(t, into):
                t = t.view(n, Hk, G, mq, d).permute(0, 3, 1, 2, 4).reshape(n, mq, Hq, d)
                into[index_q[live_q]] = t[live_q].to(into.dtype)

            def back_k(t, into):
                t = t.view(n, Hk, mk, d).permute(0, 2, 1, 3)
                into[index_k[live_k]] = t[live_k].to(into.dtype)

            qh, kh, vh = heads_q(q), heads_k(k), heads_k(v)
            p = torch.matmul(qh, kh.transpose(1, 2).contiguous()).view(n, Hk, G, mq, mk)
            p = torch.where(see[:, None, None], p * scale, -math.inf)
            top = p.amax(-1, keepdim=True)
            p = torch.exp(p - torch.where(top == -math.inf, torch.zeros_like(top), top))
            total = p.sum(-1, keepdim=True)
            p = (p / torch.where(total == 0, torch.ones_like(total), total)).view(n * Hk, G * mq, mk)
            o = torch.matmul(p, vh)
            back_q(o, out["o"])
            if c["train"]:
                do = heads_q(s["do"])
                back_k(torch.matmul(p.transpose(1, 2).contiguous(), do), out["dv"])
                dp = torch.matmul(do, vh.transpose(1, 2).contiguous())
                ds = p * (dp - (do * o).sum(-1, keepdim=True)) * scale
                back_q(torch.matmul(ds, kh), out["dq"])
                back_k(torch.matmul(ds.transpose(1, 2).contiguous(), qh), out["dk"])
        begin = end
    return out


@torch.no_grad()
def _run_plain(s):
    c = s["case"]
    k = c["kind"]
    if k == "rotary":
        pos = s["positions"].view(1, -1) if s["sections"] is None else s["positions"]
        axis = [a for a, m in enumerate(_sections(c)) for _ in range(m)]
        # far positions: angles in 64 bits
        angle = pos.double().t()[:, axis] * s["freqs"].double()
        cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
        dt, il = DTYPES[c["dtype"]], c["interleaved"]
        out = {"q": _plain_turn(s["q"], cos, sin, il, dt), "k": _plain_turn(s["k"], cos, sin, il, dt)}
        if c["train"]:
            out |= {"dq": _plain_turn(s["dq"], cos, -sin, il, dt), "dk": _plain_turn(s["dk"], cos, -sin, il, dt)}
        return out
    if k == "attention":
        return _plain_attention(s)
    x, w, t = s["x"].float(), s["weight"].float(), s["targets"]
    real = (t >= 0) & (t < c["V"])
    at = torch.where(real, t, torch.zeros_like(t))[:, None]
    z = torch.matmul(x, w.t()) * c["scale"]
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    loss = torch.where(real, (torch.log(total) + top - torch.gather(z, 1, at))[:, 0], torch.zeros_like(total[:, 0]))
    if not c["train"]:
        return {"loss": loss}
    n = real.sum().clamp_min(1)
    g = e / total
    g.scatter_add_(1, at, torch.full_like(total, -1.0))
    g = g * (real[:, None] * c["scale"]) / n
    return {"loss": (loss.double().sum() / n).float(), "dx": torch.matmul(g, w).to(s["x"].dtype),
            "dweight": torch.matmul(g.t(), x).to(s["weight"].dtype)}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------ exact
def _exact_rotary(c, s):
    pos = s["positions"].double().reshape(len(_sections(c)), -1)
    parts, at = [], 0
    for a, m in enumerate(_sections(c)):
        parts.append(torch.outer(pos[a], s["freqs"][at:at + m].double()))
        at += m
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.cat(parts, 1))[None, :, None]

    def turned(x, by):
        x, m = x.detach().double(), by.shape[-1]
        head = x[..., :2 * m]
        if c["interleaved"]:
            y = torch.view_as_real(torch.view_as_complex(head.reshape(*head.shape[:-1], m, 2).contiguous()) * by).flatten(-2)
        else:
            z = torch.complex(head[..., :m].contiguous(), head[..., m:].contiguous()) * by
            y = torch.cat([z.real, z.imag], -1)
        return torch.cat([y, x[..., 2 * m:]], -1)

    out = {"q": turned(s["q"], turn), "k": turned(s["k"], turn)}
    if c["train"]:
        out |= {"dq": turned(s["dq"], turn.conj()), "dk": turned(s["dk"], turn.conj())}
    return out


def _exact_attention(c, s):
    nq, nk = _lengths(c)
    Hq, Hk, d = c["Hq"], c["Hk"], c["d"]
    f64 = {n: s[n].detach().double() for n in ("q", "k", "v", "do") if n in s}
    out = {"o": torch.zeros_like(f64["q"])}
    if c["train"]:
        out |= {"dq": torch.zeros_like(f64["q"]), "dk": torch.zeros_like(f64["k"]), "dv": torch.zeros_like(f64["v"])}
    a = b = 0
    for m, n in zip(nq, nk):
        if m and n:
            hidden = torch.ones((m, n), dtype=torch.bool, device="cuda").triu(n - m + 1) if c["causal"] else None
            some = torch.ones(m, dtype=torch.float64, device="cuda")
            if c["causal"] and m > n:
                some[:m - n] = 0
            step = max(1, min(Hk, (1 << 27) // (m * n * (Hq // Hk))))
            for h in range(0, Hk, step):
                hk = slice(h, min(Hk, h + step))
                hq = slice(hk.start * (Hq // Hk), hk.stop * (Hq // Hk))
                q, k, v = f64["q"][a:a + m, hq].transpose(0, 1), f64["k"][b:b + n, hk], f64["v"][b:b + n, hk]
                k, v = (t.transpose(0, 1).repeat_interleave(Hq // Hk, 0) for t in (k, v))
                z = torch.bmm(q, k.transpose(1, 2)) / math.sqrt(d)
                if hidden is not None:
                    z.masked_fill_(hidden, -math.inf)
                p = torch.nan_to_num(torch.softmax(z, -1), nan=0.0) * some[:, None]
                o = torch.bmm(p, v)
                out["o"][a:a + m, hq] = o.transpose(0, 1)
                if c["train"]:
                    do = f64["do"][a:a + m, hq].transpose(0, 1)
                    dp = torch.bmm(do, v.transpose(1, 2))
                    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) / math.sqrt(d)
                    out["dq"][a:a + m, hq] = torch.bmm(ds, k).transpose(0, 1)
                    for name, left, right in (("dk", ds, q), ("dv", p, do)):
                        t = torch.bmm(left.transpose(1, 2), right)
                        out[name][b:b + n, hk] = t.view(-1, Hq // Hk, n, d).sum(1).transpose(0, 1)
        a, b = a + m, b + n
    return out


@torch.no_grad()
def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "rotary":
        return _exact_rotary(c, s)
    if c["kind"] == "attention":
        return _exact_attention(c, s)
    x, w, t = s["x"].detach().double(), s["weight"].detach().double(), s["targets"]
    real = ((t >= 0) & (t < c["V"])).nonzero().flatten()
    lost = torch.zeros(c["T"], dtype=torch.float64, device="cuda")
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    step = max(1, (1 << 28) // c["V"])
    for i in range(0, len(real), step):
        rows = real[i:i + step]
        log_p = torch.log_softmax(torch.mm(x[rows], w.t()) * c["scale"], 1)
        hit = t[rows]
        lost[rows] = -log_p[torch.arange(len(rows), device="cuda"), hit]
        if c["train"]:
            p = log_p.exp_()
            p[torch.arange(len(rows), device="cuda"), hit] -= 1
            p *= c["scale"] / max(1, len(real))
            dx[rows] = torch.mm(p, w)
            dw += torch.mm(p.t(), x[rows])
    if not c["train"]:
        return {"loss": lost}
    return {"loss": lost.sum() / max(1, len(real)), "dx": dx, "dweight": dw}
