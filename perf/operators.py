"""The operators around the ragged-cache path, as cases that can be timed and compared: the normalisation and rotation that
queries and keys get before any attention, and the attention of packed prompts, alone or behind a prefix that all share.

Kinds:

  rows    q and k of ``tokens`` tokens, RMS-normalised per head and rotated by their positions (one axis: text or frames; three: frame,
          row, column of a picture grid)
  attn    attention of ``seqs`` packed sequences, causal by blocks of ``block`` tokens (0: no mask), ``heads`` query heads in groups over
          ``kv_heads``; ``prefix`` > 0: keys and values that stand in front of every sequence and are stored once

Tensors are held as the model holds them, [tokens][heads][head_dim], in bfloat16.  ``own`` False: the plain form in torch; True: the
library's entry points.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6


def listed():
    return [
        # ---- rows ----
        # single tokens of four sequences, far out, positions stretched for a long context: the step of a decoder with grouped heads
        dict(name="rows_step", kind="rows", tokens=4, heads=32, kv_heads=8, head_dim=128, rot=128, interleaved=False, axes=1, first=120000,
             grid_h=1, grid_w=1, norm=True, stretch=8.0),
        # the chunk of three frames of 30 x 52 tokens that every denoising pass works on (the benchmark's layer)
        dict(name="rows_chunk", kind="rows", tokens=4680, heads=12, kv_heads=12, head_dim=128, rot=128, interleaved=True, axes=3, first=57,
             grid_h=30, grid_w=52, norm=True, stretch=1.0),
        # a small picture, head_dim 64, half of the channels rotated, no norm
        dict(name="rows_odd", kind="rows", tokens=999, heads=5, kv_heads=5, head_dim=64, rot=32, interleaved=False, axes=1, first=0,
             grid_h=1, grid_w=1, norm=False, stretch=1.0),
        # a video of 57 frames, taken in at once to be continued
        dict(name="rows_video", kind="rows", tokens=88920, heads=12, kv_heads=12, head_dim=128, rot=128, interleaved=True, axes=3, first=0,
             grid_h=30, grid_w=52, norm=True, stretch=1.0),
        # ---- prompts ----
        # the tiny configuration: two videos of up to 12 frames of 16 tokens, generated three frames at a time
        dict(name="prompt_tiny", kind="attn", seqs=2, q_max=192, k_max=192, heads=4, kv_heads=4, head_dim=64, block=48, prefix=0, spread=1.0, lengths=3),
        # text prompts of different lengths, grouped heads, plainly causal
        dict(name="prompt_text", kind="attn", seqs=7, q_max=4001, k_max=4001, heads=32, kv_heads=8, head_dim=128, block=1, prefix=0, spread=8.0, lengths=5),
        # an existing video of nine frames, generated three frames at a time, at the benchmark's layer shape
        dict(name="prompt_video", kind="attn", seqs=1, q_max=14040, k_max=14040, heads=12, kv_heads=12, head_dim=128, block=4680, prefix=0, spread=1.0, lengths=0),
        # the other head size: three videos of one-frame chunks
        dict(name="prompt_d64", kind="attn", seqs=3, q_max=6240, k_max=6240, heads=16, kv_heads=16, head_dim=64, block=1560, prefix=0, spread=2.0, lengths=1),
        # ---- behind a shared prefix ----
        # single tokens of a few answers to one short prompt
        dict(name="shared_step", kind="attn", seqs=8, q_max=1, k_max=300, heads=12, kv_heads=12, head_dim=128, block=1, prefix=2048, spread=16.0, lengths=2),
        # single tokens of many answers to one long prompt
        dict(name="shared_wide", kind="attn", seqs=64, q_max=1, k_max=1024, heads=32, kv_heads=8, head_dim=128, block=1, prefix=16384, spread=16.0, lengths=4),
        # four ways to continue a video of six frames by one frame each
        dict(name="shared_video", kind="attn", seqs=4, q_max=1560, k_max=1560, heads=12, kv_heads=12, head_dim=128, block=1560, prefix=9360, spread=1.0, lengths=0),
        # short questions of different lengths about one document, head_dim 64
        dict(name="shared_d64", kind="attn", seqs=13, q_max=97, k_max=131, heads=10, kv_heads=2, head_dim=64, block=1, prefix=5003, spread=6.0, lengths=7),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, no dearer than the dearest listed one of its kind."""
    while True:
        if rng.random() < 0.3:
            three = rng.random() < 0.5
            h, w = (rng.randint(4, 30), rng.randint(4, 52)) if three else (1, 1)
            D = rng.choice([64, 128, 128])
            kv = rng.choice([1, 2, 4, 5, 8, 12])
            c = dict(kind="rows", tokens=_log_int(rng, 1, 88920), heads=kv * rng.choice([1, 1, 2, 4]), kv_heads=kv, head_dim=D,
                     rot=D if three else rng.choice([D, D, D // 2, 16]), interleaved=rng.random() < 0.5, axes=3 if three else 1,
                     first=_log_int(rng, 1, 100) if three else _log_int(rng, 1, 200000), grid_h=h, grid_w=w, norm=rng.random() < 0.8,
                     stretch=rng.choice([1.0, 4.0, 8.0]))
        else:
            kv = rng.choice([1, 2, 4, 8, 12])
            step = rng.random() < 0.35
            q = rng.randint(1, 4) if step else _log_int(rng, 8, 14040)
            c = dict(kind="attn", seqs=_log_int(rng, 1, 64), q_max=q, k_max=_log_int(rng, max(q, 16), 4 * q + 2000) if step or rng.random() < 0.3 else q,
                     heads=kv * rng.choice([1, 1, 2, 4]), kv_heads=kv, head_dim=rng.choice([64, 128, 128]),
                     block=rng.choice([0, 1, 1, 48, 1560, 4680]), prefix=_log_int(rng, 64, 16384) if rng.random() < 0.5 else 0,
                     spread=rng.choice([1.0, 2.0, 8.0]), lengths=rng.randint(0, 9999))
        if _cost(c) <= max(_cost(x) for x in listed() if x["kind"] == c["kind"]) and _dense(c) <= max(_dense(x) for x in listed()):
            return c


def _lengths(c):
    """(queries, keys) of every sequence: the longest first, the others down to 1 / spread of it, all from the case alone."""
    rng = random.Random(c["lengths"])
    part = [1.0] + [math.exp(-rng.random() * math.log(c["spread"])) for _ in range(c["seqs"] - 1)]
    ks = [max(1, int(c["k_max"] * p)) for p in part]
    qs = ks if c["q_max"] == c["k_max"] else [min(k, max(1, int(c["q_max"] * p))) for k, p in zip(ks, part)]
    return list(qs), ks


def _cu(lengths):
    cu = [0]
    for n in lengths:
        cu.append(cu[-1] + n)
    return cu


def _dense(c):
    """Scores that the plain form holds at once."""
    if c["kind"] == "rows":
        return 0
    qs, ks = _lengths(c)
    return c["heads"] * (c["seqs"] * max(qs) * max(ks) + sum(qs) * (c["prefix"] + (max(ks) if c["prefix"] else 0)))


def _pairs(c):
    """Visible (query, key) pairs of one head, the prefix's included."""
    qs, ks = _lengths(c)
    n = 0
    for lq, lk in zip(qs, ks):
        if c["block"] == 0:
            n += lq * lk
        else:
            b = c["block"]
            n += sum(min(lk, (p // b + 1) * b) * (min(p // b * b + b, lk) - p) for p in _block_starts(lk - lq, lk, b))
    return n + sum(qs) * c["prefix"]


def _block_starts(p0, p1, b):
    return [p0] + list(range(p0 // b * b + b, p1, b)) if p1 > p0 else []


def work(case):
    c = case
    if c["kind"] == "rows":
        values = c["tokens"] * (c["heads"] + c["kv_heads"]) * c["head_dim"]
        return {"bytes": 4.0 * values + 4.0 * c["axes"] * c["tokens"], "flops": 8.0 * values}
    qs, ks = _lengths(c)
    row = 2.0 * c["head_dim"]
    return {"bytes": 2 * row * c["heads"] * sum(qs) + 2 * row * c["kv_heads"] * (sum(ks) + c["prefix"]),
            "flops": 4.0 * c["head_dim"] * c["heads"] * _pairs(c)}


def _cost(c):
    w = work(c)
    return w["bytes"] / 4e12 + w["flops"] / 0.8e15


def _randn(shape, seed, scale=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * scale).to(torch.bfloat16)


def _axis_pairs(c):
    """Channel pairs of each axis: the spatial axes a third each (rounded down), the frame axis the rest."""
    n = c["rot"] // 2
    return [n] if c["axes"] == 1 else [n - 2 * (n // 3), n // 3, n // 3]


def prepare(case, seed):
    c, base = dict(case), 1000003 * (int(seed) % (1 << 31))
    H, KV, D = c["heads"], c["kv_heads"], c["head_dim"]
    s = {"case": c}
    if c["kind"] == "rows":
        n = c["tokens"]
        s["q"], s["k"] = _randn((n, H, D), base, 1.7), _randn((n, KV, D), base + 1, 0.6)
        s["qw"], s["kw"] = (1.0 + 0.3 * _randn((D,), base + 2 + i).float() for i in (0, 1))
        s["qw"], s["kw"] = s["qw"].to(torch.bfloat16), s["kw"].to(torch.bfloat16)
        t = torch.arange(n, device=DEV, dtype=torch.int32)
        if c["axes"] == 1:
            s["positions"] = (c["first"] + t)[None].contiguous()
        else:
            per = c["grid_h"] * c["grid_w"]
            s["positions"] = torch.stack([c["first"] + t // per, t % per // c["grid_w"], t % c["grid_w"]]).to(torch.int32).contiguous()
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        return s
    qs, ks = _lengths(c)
    tq, tk = sum(qs), sum(ks)
    s["q"], s["k"], s["v"] = _randn((tq, H, D), base), _randn((tk, KV, D), base + 1), _randn((tk, KV, D), base + 2)
    if c["prefix"]:
        s["k_prefix"], s["v_prefix"] = (_randn((c["prefix"], KV, D), base + 3 + i) for i in (0, 1))
    s["cu_q"], s["cu_k"] = _cu(qs), _cu(ks)
    s["out"] = torch.empty_like(s["q"])
    return s


def run(state):
    rows = state["case"]["kind"] == "rows"
    if own:
        return _own_rows(state) if rows else _own_attn(state)
    return _plain_rows(state) if rows else _plain_attn(state)


# ---- the library's calls ---------------------------------------------------------------------------------------------

def _heads_first(t):
    return t.transpose(0, 1)


def _own_rows(s):
    from paper_2605_13111_amd import binding as B
    c = s["case"]
    if "rope" not in s:        # a model's frequencies: made once, on the host
        s["rope"] = B.make_rope(c["head_dim"], c["rot"], interleaved=c["interleaved"], axis_pairs=_axis_pairs(c), scaling="linear" if c["stretch"] != 1.0 else "none",
                                factor=c["stretch"])
    B.pf_qk_norm_rope(s["rope"], s["positions"], _heads_first(s["q"]), _heads_first(s["q_out"]), _heads_first(s["k"]), _heads_first(s["k_out"]),
                      q_weight=s["qw"] if c["norm"] else None, k_weight=s["kw"] if c["norm"] else None, eps=EPS if c["norm"] else 0.0)
    return [s["q_out"], s["k_out"]]


def _own_attn(s):
    from paper_2605_13111_amd import binding as B
    c = s["case"]
    if "packed" not in s:      # the batch's plan and workspace: made once for all layers of a model, whose lengths are the same
        s["packed"] = B.Packed(s["cu_q"], s["cu_k"], c["heads"], c["kv_heads"], c["head_dim"], block=c["block"], prefix_tokens=c["prefix"], device=DEV)
        B.pf_packed_plan(s["packed"])
        s["workspace"] = torch.empty(B.pf_packed_workspace_bytes(s["packed"]), dtype=torch.uint8, device=DEV)
    prefix = (_heads_first(s["k_prefix"]), _heads_first(s["v_prefix"])) if c["prefix"] else (None, None)
    B.pf_packed_attn_fwd(s["packed"], _heads_first(s["q"]), _heads_first(s["k"]), _heads_first(s["v"]), _heads_first(s["out"]), s["workspace"],
                         k_prefix=prefix[0], v_prefix=prefix[1])
    return [s["out"]]


# ---- the plain form --------------------------------------------------------------------------------------------------

def _plain_rotate(x, w, s):
    """x [tokens, heads, D] in 32 bits: normalised, rotated, rounded once."""
    c = s["case"]
    if c["norm"]:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    pairs = _axis_pairs(c)
    axis = torch.repeat_interleave(torch.arange(c["axes"], device=DEV), torch.tensor(pairs, device=DEV))
    at = torch.cat([torch.arange(n, device=DEV, dtype=torch.float64) / n for n in pairs])
    # angles of far positions in 64 bits
    angle = s["positions"].double()[axis].T * (10000.0 ** -at / c["stretch"])
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    r, half = c["rot"], c["rot"] // 2
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if c["interleaved"] else (x[..., :half], x[..., half:r])
    a, b = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., r:]], -1).to(torch.bfloat16)


def _plain_rows(s):
    return [_plain_rotate(s["q"].float(), s["qw"], s), _plain_rotate(s["k"].float(), s["kw"], s)]


def _padded(x, cu, longest):
    """Packed rows [tokens, ...] as [seqs, longest, ...]; places behind a sequence's end repeat some row."""
    start, end = torch.tensor(cu[:-1], device=DEV), torch.tensor(cu[1:], device=DEV)
    at = start[:, None] + torch.arange(longest, device=DEV)
    return x[torch.minimum(at, (end - 1)[:, None]).clamp_min(0)]


def _plain_attn(s):
    """Every sequence padded to the longest; scores of the own keys and of the prefix side by side, one softmax over both."""
    c = s["case"]
    S, H, KV, D, P = c["seqs"], c["heads"], c["kv_heads"], c["head_dim"], c["prefix"]
    G, cu_q, cu_k = H // KV, s["cu_q"], s["cu_k"]
    lq, lk = torch.tensor(cu_q, device=DEV).diff(), torch.tensor(cu_k, device=DEV).diff()
    mq, mk, tq = int(max(b - a for a, b in zip(cu_q, cu_q[1:]))), int(max(b - a for a, b in zip(cu_k, cu_k[1:]))), cu_q[-1]
    q = s["q"].float() * D ** -0.5
    qp = _padded(q, cu_q, mq).view(S, mq, KV, G, D).permute(0, 2, 3, 1, 4).reshape(S * KV, G * mq, D)
    kp, vp = (_padded(t, cu_k, mk).float().permute(0, 2, 1, 3).reshape(S * KV, mk, D) for t in (s["k"], s["v"]))
    scores = torch.bmm(qp, kp.transpose(1, 2).contiguous()).view(S, KV, G, mq, mk)
    j, p = torch.arange(mk, device=DEV), (lk - lq)[:, None] + torch.arange(mq, device=DEV)
    seen = (j < lk[:, None])[:, None, :]                                         # [S, mq, mk]
    if c["block"]:
        seen = seen & (torch.div(j, c["block"], rounding_mode="floor")[None, None] <= torch.div(p, c["block"], rounding_mode="floor")[..., None])
    scores.masked_fill_(~seen.expand(S, mq, mk)[:, None, None], -math.inf)
    if not P:
        top = scores.amax(-1, keepdim=True).clamp_min(-3e38)
        weights = scores.sub_(top).exp_()
        total = weights.sum(-1).view(S * KV, G * mq, 1)
        o = torch.bmm(weights.view(S * KV, G * mq, mk), vp) / total
        o = o.view(S, KV, G, mq, D).permute(0, 3, 1, 2, 4).reshape(S, mq, H, D)
        row_seq = torch.repeat_interleave(torch.arange(S, device=DEV), lq)
        return [o[row_seq, torch.arange(tq, device=DEV) - torch.tensor(cu_q, device=DEV)[row_seq]].to(torch.bfloat16)]
    # the prefix's scores belong to packed rows; the own ones join them there and go back for their values
    row_seq = torch.repeat_interleave(torch.arange(S, device=DEV), lq)
    row_at = torch.arange(tq, device=DEV) - torch.tensor(cu_q, device=DEV)[row_seq]
    mine = scores.permute(0, 3, 1, 2, 4)[row_seq, row_at]                        # [tq, KV, G, mk]
    kf, vf = (s[n].float().transpose(0, 1).contiguous() for n in ("k_prefix", "v_prefix"))   # [KV, P, D]
    rows = q.view(tq, KV, G, D).transpose(0, 1).reshape(KV, tq * G, D)
    shared = torch.bmm(rows, kf.transpose(1, 2).contiguous()).view(KV, tq, G, P).transpose(0, 1)
    top = torch.maximum(mine.amax(-1, keepdim=True), shared.amax(-1, keepdim=True))
    mine, shared = torch.exp(mine - top), torch.exp(shared - top)
    total = mine.sum(-1, keepdim=True) + shared.sum(-1, keepdim=True)
    back = torch.zeros((S, mq, KV, G, mk), device=DEV)
    back[row_seq, row_at] = mine
    o_own = torch.bmm(back.permute(0, 2, 3, 1, 4).reshape(S * KV, G * mq, mk), vp).view(S, KV, G, mq, D)
    o_own = o_own.permute(0, 3, 1, 2, 4)[row_seq, row_at]
    o_pre = torch.bmm(shared.transpose(0, 1).reshape(KV, tq * G, P), vf).view(KV, tq, G, D).transpose(0, 1)
    return [((o_own + o_pre) / total).reshape(tq, H, D).to(torch.bfloat16)]


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------

def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["kind"] == "rows":
        return [_exact_rows(c, s["q"], s["qw"], s["positions"]), _exact_rows(c, s["k"], s["kw"], s["positions"])]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    G = c["heads"] // c["kv_heads"]
    for n in range(c["seqs"]):
        q0, q1, k0, k1 = s["cu_q"][n], s["cu_q"][n + 1], s["cu_k"][n], s["cu_k"][n + 1]
        for h in range(c["heads"]):
            k, v = s["k"][k0:k1, h // G].double(), s["v"][k0:k1, h // G].double()
            if c["prefix"]:
                k, v = torch.cat([s["k_prefix"][:, h // G].double(), k]), torch.cat([s["v_prefix"][:, h // G].double(), v])
            for r0 in range(q0, q1, 4096):
                r1 = min(r0 + 4096, q1)
                x = s["q"][r0:r1, h].double() @ k.T / math.sqrt(c["head_dim"])
                if c["block"]:
                    place = torch.arange(r0, r1, device=DEV) - q0 + (k1 - k0) - (q1 - q0)
                    last = c["prefix"] + (place // c["block"] + 1) * c["block"]
                    x = torch.where(torch.arange(k.shape[0], device=DEV) < last[:, None], x, -math.inf)
                out[r0:r1, h] = torch.softmax(x, -1) @ v
    return [out]


def _exact_rows(c, x, w, positions):
    """Pairs as complex numbers, turned by exp(i angle)."""
    y = x.double()
    if c["norm"]:
        y = y / torch.sqrt(y.pow(2).sum(-1, keepdim=True) / c["head_dim"] + EPS) * w.double()
    n, r = c["rot"] // 2, c["rot"]
    first = 2 * torch.arange(n, device=DEV) if c["interleaved"] else torch.arange(n, device=DEV)
    second = first + (1 if c["interleaved"] else n)
    out, i = y.clone(), 0
    for axis, pairs in enumerate(_axis_pairs(c)):
        for m in range(pairs):
            angle = positions[axis].double() * math.exp(-math.log(10000.0) * m / pairs) / c["stretch"]
            z = torch.complex(y[..., first[i]], y[..., second[i]]) * torch.polar(torch.ones_like(angle), angle)[:, None]
            out[..., first[i]], out[..., second[i]] = z.real, z.imag
            i += 1
    return out
