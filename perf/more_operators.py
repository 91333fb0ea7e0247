"""What the position rotation and the 4-bit cache behind the pruning are measured on.

A layer behind the pruning takes its projections' queries, keys and values, brings queries and
keys to length head by head where the model has such norms, turns them by the position ids that
the compaction carried along (one axis, or three of images and videos), puts keys and values
into the paged cache and decodes from it; a cache held in 4 bits takes 72 bytes for a head's
128 values and leaves room for three to four times the questions. Five operators do that:

  rotate  provip_rotate           norm (or none) and rotation of packed rows' queries and keys
  append  provip_rotate_append    the same, with keys and values into pages on the way: pages
                                  of the rows' type, or of 4 bits (read back by provip_kv_read4)
  store   provip_kv_append4       rows into 4-bit pages, and out of them again for a prompt's
          provip_kv_read4         attention
  decode  DecodeAttention4        one token per request over 4-bit pages, shared and own ones

The 4-bit form of a row of 128 values: for each 32 of them a bf16 scale d and 32 codes n from 0
to 15 that stand for d (n - 8). d = -e / 8 with e the value of largest magnitude (the positive
one of two), n = round(x (1 / d)) + 8, at most 15. Codes: 16 bits at 16-bit place 4 g + q hold
values 32 q + 4 g .. + 3, the first in the lowest bits. A page of one head: its rows' 64 bytes
of codes, then its rows' four scales.

Each case is a dict of plain values. `run` computes an operator in elementary torch
operations in 32 bits (angles in 64), or, where `own` is true, through the package's entry
points. Lengths are a function of the case alone (`mix` is their seed), values of the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
DH = 128            # head size of every model here
SYS = 35            # system rows in front of the visual ones
EPS = 1e-6
ROW4 = 72           # bytes of a head's row in 4 bits: 64 of codes, 8 of scales
SECTIONS = (16, 24, 24)  # pairs that turn with the time, the height and the width of a position
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # norm and rotation ------------------------------------------------------------
        # the follow-up question of one user: 48 rows of a 7B model without norms
        dict(name="rotate_follow_up", op="rotate", dtype="bf16", T=48, H_q=32, H_kv=32, axes=1, norm=False, far=4096,
             base=1e4, mix=1),
        # a 7B fp32 model's prompt after the pre-LLM stage, late in a long conversation
        dict(name="rotate_one_fp32", op="rotate", dtype="f32", T=291, H_q=32, H_kv=32, axes=1, norm=True, far=1000000,
             base=1e6, mix=2),
        # one video before any pruning: 35 + 9216 + 128 rows, three axes, norms of queries and keys
        dict(name="rotate_video", op="rotate", dtype="bf16", T=9379, H_q=28, H_kv=4, axes=3, norm=True, far=32768,
             base=1e6, mix=3),
        # rotation on the way into the cache -------------------------------------------
        # a decode step of 256 requests, 28 heads in 4 groups
        dict(name="append_decode_256", op="append", bits=16, dtype="bf16", T=256, H_q=28, H_kv=4, axes=3, norm=True,
             page=16, far=32768, base=1e6, mix=4),
        # the prompts of an anyres batch after the pre-LLM stage, 32 heads
        dict(name="append_anyres", op="append", bits=16, dtype="bf16", T=8 * 1091 - 3, H_q=32, H_kv=32, axes=1,
             norm=False, page=64, far=4096, base=1e4, mix=5),
        # a pruned video's rows into a 4-bit cache: 35 + 2304 rows
        dict(name="append4_video", op="append", bits=4, dtype="bf16", T=SYS + 2304, H_q=28, H_kv=4, axes=3, norm=True,
             page=64, far=32768, base=1e6, mix=6),
        # rows into 4-bit pages and out again ------------------------------------------
        # one pruned image that several questions will share: 35 + 64 rows
        dict(name="store_image", op="store", dtype="bf16", T=SYS + 64, H_kv=32, page=16, mix=7),
        # a compacted anyres batch, 32 heads
        dict(name="store_anyres", op="store", dtype="bf16", T=8 * 1091 - 3, H_kv=32, page=64, mix=8),
        # decoding from 4 bits ---------------------------------------------------------
        # a single user's token over a pruned image (35 + 64 + 112 rows)
        dict(name="decode_one", op="decode", dtype="bf16", B=1, H_q=32, H_kv=32, lo=211, hi=211, prefix=0, page=16,
             mix=9),
        # 32 users with an image each, no shared rows, fp32 queries
        dict(name="decode_ragged_fp32", op="decode", dtype="f32", B=32, H_q=32, H_kv=32, lo=163, hi=1091, prefix=0,
             page=16, mix=10),
        # 64 questions about one unpruned video
        dict(name="decode_shared_video", op="decode", dtype="bf16", B=64, H_q=28, H_kv=4, lo=1, hi=512,
             prefix=SYS + 9216, page=64, mix=11),
        # 128 users with an image or a video of their own, 32 heads
        dict(name="decode_ragged_128", op="decode", dtype="bf16", B=128, H_q=32, H_kv=32, lo=163, hi=2339, prefix=0,
             page=64, mix=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate", "append", "store", "decode", "decode"])
    mix = rng.randrange(1 << 20)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    H_q, H_kv = rng.choice([(32, 32), (40, 40), (28, 4)])
    page = rng.choice([16, 32, 64, 128])
    most = max(work(x)["bytes"] for x in listed() if x["op"] == op)
    if op == "decode":
        hi = _log(rng, 1, 9379)
        c = dict(op=op, dtype=dtype, B=_log(rng, 1, 256), H_q=H_q, H_kv=H_kv, lo=rng.randint(max(hi // 4, 1), hi), hi=hi,
                 prefix=rng.choice([0, _log(rng, 1, SYS + 9216)]), page=page, mix=mix)
        flops = max(work(x)["flops"] for x in listed() if x["op"] == op)
        while work(c)["bytes"] > most or work(c)["flops"] > flops:
            if c["B"] > 1:
                c["B"] = (c["B"] + 1) // 2
            else:
                c["hi"], c["prefix"] = c["hi"] * 4 // 5, c["prefix"] * 4 // 5
                c["lo"] = min(c["lo"], c["hi"])
        return c
    c = dict(op=op, dtype=dtype, T=_log(rng, 1, 9379), H_kv=H_kv, page=page, mix=mix)
    if op != "store":
        c.update(H_q=H_q, axes=rng.choice([1, 3]), norm=rng.random() < 0.5, far=_log(rng, 1, 1000000),
                 base=rng.choice([1e4, 1e6]))
    if op == "append":
        # (fp32 models rotate first and store the rows then: rounded to no 16-bit type between, a
        # value next to a border of two codes may fall on either side)
        c["bits"] = rng.choice([16, 4]) if dtype == "bf16" else 16
    while work(c)["bytes"] > most:
        c["T"] = c["T"] * 4 // 5
    return c


# ---------------------------------------------------------------------------
# lengths of a case
# ---------------------------------------------------------------------------
def _spread(n, lo, hi, mix):
    """n lengths from lo to hi, evenly apart, in an order drawn from mix."""
    v = [lo + (hi - lo) * i // max(n - 1, 1) for i in range(n)]
    random.Random(mix).shuffle(v)
    return v


def _ceil(a, b):
    return -(-a // b)


def work(case):
    c, op = case, case["op"]
    es = 4 if c["dtype"] == "f32" else 2
    if op == "decode":
        k = sum(_spread(c["B"], c["lo"], c["hi"], c["mix"]))
        n = es * DH * 2 * c["B"] * c["H_q"] + 2 * ROW4 * (k + c["prefix"]) * c["H_kv"] + 4 * c["B"] * (c["H_q"] + 1)
        n += 4 * _ceil(k + c["prefix"], c["page"])
        return {"bytes": n, "flops": 4 * DH * c["H_q"] * (k + c["B"] * c["prefix"])}
    T, H = c["T"], c["H_kv"]
    if op == "store":  # rows in, codes and scales, rows out
        return {"bytes": T * H * (4 * es * DH + 2 * ROW4) + 4 * T, "flops": 0}
    turned = 2 * es * DH * T * (c["H_q"] + H) + 4 * T * c["axes"]
    flops = (3 + 4 * c["norm"]) * DH * T * (c["H_q"] + H)
    if op == "rotate":
        return {"bytes": turned, "flops": flops}
    if c["bits"] == 16:
        return {"bytes": turned + 2 * es * DH * T * H + 4 * T, "flops": flops}
    # 4 bits: queries, keys and values in; queries, codes and scales, keys and values read back out
    return {"bytes": turned + 3 * es * DH * T * H + 2 * ROW4 * T * H + 4 * T, "flops": flops}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _freq(c):
    return [c["base"] ** (-2 * i / DH) for i in range(DH // 2)]


def _axis(c):
    return [0] * (DH // 2) if c["axes"] == 1 else [a for a in range(3) for _ in range(SECTIONS[a])]


def prepare(case, seed):
    if case["op"] == "decode":
        return _prepare_decode(case, seed)
    return _prepare_rows(case, seed)


def _prepare_rows(c, seed):
    """Queries, keys and values are slices of one fused buffer, as a model's projection leaves
    them. Position ids ascend with gaps, as pruning leaves them, up to `far`; height and width
    ids lie in a grid beside them. Slots are spread over the pool; one row in 50 of those that go
    into pages has none (its request got no page)."""
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    T, H = c["T"], c["H_kv"]
    s = dict(case=c)
    H_q = c.get("H_q", 0)
    heads = [H_q, H, H]
    # (a value in 64 of the keys' is far larger, as some channels of real keys are)
    big = 1 + 7 * (torch.rand(sum(heads), DH, device=DEV, generator=g) < 1 / 64)
    fused = torch.randn(T, sum(heads), DH, device=DEV, generator=g) * big
    s["Q"], s["K"], s["V"] = fused.to(dt).split(heads, 1)
    if c["op"] != "store":
        far = c["far"]
        pos = torch.randint(0, max(far, 1), (T,), device=DEV, generator=g).sort().values
        grid = torch.randint(0, 96, (c["axes"] - 1, T), device=DEV, generator=g)
        s["pos"] = torch.cat([pos[None], pos[None] + grid]).to(torch.int32)
        s["w_q"] = s["w_k"] = None
        if c["norm"]:
            s["w_q"], s["w_k"] = (1 + 0.2 * torch.randn(2, DH, device=DEV, generator=g)).to(dt)
        s["freq"] = torch.tensor(_freq(c), dtype=torch.float64, device=DEV)
        s["axis"] = torch.tensor(_axis(c), dtype=torch.long, device=DEV)
    if c["op"] != "rotate":
        p = c["page"]
        pages = _ceil(T, p) + 2
        slot = torch.randperm(pages * p, device=DEV, generator=g)[:T].to(torch.int32)
        slot[torch.rand(T, device=DEV, generator=g) < 0.02] = -1
        s["slot"] = slot
        if c["op"] == "append" and c["bits"] == 16:
            s["k_pages"], s["v_pages"] = torch.zeros(2, pages, p, H, DH, dtype=dt, device=DEV)
        else:
            s["k_pages"], s["v_pages"] = torch.zeros(2, pages, H, p * ROW4, dtype=torch.uint8, device=DEV)
            s["rows"] = torch.zeros(2, T, H, DH, dtype=dt, device=DEV)
    if H_q:
        s["q_out"] = torch.empty(T, H_q, DH, dtype=dt, device=DEV)
        s["k_out"] = torch.empty(T, H, DH, dtype=dt, device=DEV) if c["op"] == "rotate" else None
    if own and c["op"] != "store":
        from paper_2608_25332_gb300 import provip as P
        s["rotary"] = P.Rotary(_freq(c), _axis(c))
    return s


def _prepare_decode(c, seed):
    """Pages in a seeded order; what no request holds, and the slots past each length, have NaN
    scales: whoever reads them shows it."""
    g, dt, p, n = _gen(seed), DTYPES[c["dtype"]], c["page"], c["prefix"]
    B, H_q, H_kv = c["B"], c["H_q"], c["H_kv"]
    lens = _spread(B, c["lo"], c["hi"], c["mix"])
    held, pre = [_ceil(x, p) for x in lens], _ceil(n, p)
    width, pages = max(held), sum(held) + pre + 3
    order = torch.randperm(pages, device=DEV, generator=g).to(torch.int32)
    table = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    kv_len = _i32(lens)
    col = torch.arange(width, device=DEV)
    table[col[None] < _i32(held)[:, None]] = order[pre:pre + sum(held)]
    prefix_table = order[:pre].clone()
    u = torch.randn(H_kv, DH, device=DEV, generator=g)
    u = u / u.norm(dim=1, keepdim=True)
    at = torch.arange(width * p, device=DEV)
    own_slots = (table.long()[:, at // p] * p + at % p)[at[None] < kv_len[:, None]]
    at = torch.arange(n, device=DEV)
    slots = torch.cat([prefix_table.long()[at // p] * p + at % p if n else at, own_slots])
    first = (slots[:1] if n else table[:, 0].long() * p)
    s = dict(case=c, table=table, kv_len=kv_len, prefix_table=prefix_table if n else None)
    for name in ("k_pages", "v_pages"):
        codes = torch.randint(0, 256, (pages, H_kv, p, 64), device=DEV, generator=g, dtype=torch.uint8)
        scales = torch.full((pages, p, H_kv, 4), math.nan, dtype=torch.bfloat16, device=DEV)
        # (a scale for values around 1 as their largest leaves it, of either sign)
        d = (0.2 + 0.25 * torch.rand(len(slots), H_kv, 4, device=DEV, generator=g))
        d *= 1 - 2 * torch.randint(0, 2, d.shape, device=DEV, generator=g)
        scales.view(-1, H_kv, 4)[slots] = d.to(torch.bfloat16)
        codes, scales = codes.view(pages, H_kv, p * 64), scales.permute(0, 2, 1, 3).contiguous()
        if name == "k_pages":
            # the first key is a sink along the direction that the queries of a group share
            c4, d4 = _pack((8 * math.sqrt(DH) * u))
            page, row = first // p, first % p
            codes.view(pages, H_kv, p, 64)[page, :, row] = c4
            scales[page, :, row] = d4
        s[name] = torch.cat([codes, scales.view(torch.uint8).view(pages, H_kv, p * 8)], 2)
    s["Q"] = (torch.randn(B, H_q, DH, device=DEV, generator=g) + u.repeat_interleave(H_q // H_kv, 0)).to(dt)
    if own:
        from paper_2608_25332_gb300 import provip as P
        s["step"] = P.DecodeAttention4(B, H_q, H_kv, max(lens), prefix_len=n, dtype=dt, device=DEV)
    return s


# ---------------------------------------------------------------------------
# the 4-bit form
# ---------------------------------------------------------------------------
def _pack(x):
    """[..., 128] in 32 bits -> codes [..., 64] uint8, scales [..., 4] bf16"""
    v = x.unflatten(-1, (4, 32))
    hi, lo = v.amax(-1, keepdim=True), v.amin(-1, keepdim=True)
    d = (torch.where(hi >= -lo, hi, lo) / -8).to(torch.bfloat16)
    f = d.float()
    r = torch.where(f == 0, 0.0, 1.0 / f)
    n = (torch.round((v * r).clamp(-8, 7)) + 8).to(torch.uint8)  # [..., q, 32]
    n = n.unflatten(-1, (8, 2, 2)).transpose(-4, -3)             # [..., g, q, 2 bytes, 2 values]
    return (n[..., 0] | n[..., 1] << 4).flatten(-3), d.squeeze(-1)


def _unpack(codes, scales):
    """codes [..., 64] uint8, scales [..., 4] -> [..., 128] in 32 bits"""
    n = codes.unflatten(-1, (8, 4, 2)).transpose(-3, -2)         # [..., q, g, 2 bytes]
    n = torch.stack([n & 15, n >> 4], -1).flatten(-3).float() - 8
    return (n * scales.float()[..., None]).flatten(-2)


def _rows4(pages, slot, p):
    """codes and scales of the rows at `slot` (any shape), all heads"""
    H = pages.shape[1]
    page, row, h = slot[..., None] // p, slot[..., None] % p, torch.arange(H, device=DEV)
    codes = pages[..., :p * 64].unflatten(-1, (p, 64))[page, h, row]
    scales = pages[..., p * 64:].unflatten(-1, (p, 8))[page, h, row]
    return codes, scales.contiguous().view(torch.bfloat16)


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(state):
    return {"rotate": _run_rotate, "append": _run_append, "store": _run_store,
            "decode": _run_decode}[state["case"]["op"]](state)


def _turn(x, w, s):
    """norm (with weights w) and rotation of [T, H, 128]"""
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w.float()
    angle = (s["pos"][s["axis"]].T.double() * s["freq"])[:, None]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    a, b = y[..., :DH // 2], y[..., DH // 2:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(x.dtype)


def _run_rotate(s):
    if own:
        from paper_2608_25332_gb300 import provip as P
        return P.provip_rotate(s["Q"], s["K"], s["pos"], s["rotary"], s["w_q"], s["w_k"], EPS, out=(s["q_out"], s["k_out"]))
    return _turn(s["Q"], s["w_q"], s), _turn(s["K"], s["w_k"], s)


def _run_append(s):
    c = s["case"]
    if own:
        from paper_2608_25332_gb300 import provip as P
        q, _ = P.provip_rotate_append(s["Q"], s["K"], s["V"], s["pos"], s["rotary"], s["slot"], s["k_pages"], s["v_pages"],
                                      s["w_q"], s["w_k"], EPS, out=(s["q_out"], None))
        if c["bits"] == 16:
            return q, s["k_pages"], s["v_pages"]
        return (q, *P.provip_kv_read4(s["slot"], s["k_pages"], s["v_pages"], out=(s["rows"][0], s["rows"][1])))
    q, k = _turn(s["Q"], s["w_q"], s), _turn(s["K"], s["w_k"], s)
    if c["bits"] == 4:
        return (q, *_store(s, k, s["V"]))
    keep = s["slot"] >= 0
    at = s["slot"][keep].long()
    s["k_pages"].flatten(0, 1)[at] = k[keep]
    s["v_pages"].flatten(0, 1)[at] = s["V"][keep]
    return q, s["k_pages"], s["v_pages"]


def _store(s, K, V):
    """rows into 4-bit pages, and the rows at those slots out again"""
    p, out = s["case"]["page"], []
    keep = s["slot"] >= 0
    at = s["slot"][keep].long()
    h = torch.arange(s["case"]["H_kv"], device=DEV)
    for rows, pages in ((K, s["k_pages"]), (V, s["v_pages"])):
        codes, d = _pack(rows[keep].float())
        page, row = at[:, None] // p, at[:, None] % p
        pages[..., :p * 64].unflatten(-1, (p, 64))[page, h, row] = codes
        pages[..., p * 64:].unflatten(-1, (p, 8))[page, h, row] = d.view(torch.uint8)
        back = torch.zeros(rows.shape, dtype=rows.dtype, device=DEV)
        back[keep] = _unpack(*_rows4(pages, at, p)).to(rows.dtype)
        out.append(back)
    return tuple(out)


def _run_store(s):
    if own:
        from paper_2608_25332_gb300 import provip as P
        P.provip_kv_append4(s["K"], s["V"], s["slot"], s["k_pages"], s["v_pages"])
        return P.provip_kv_read4(s["slot"], s["k_pages"], s["v_pages"], out=(s["rows"][0], s["rows"][1]))
    return _store(s, s["K"], s["V"])


def _softmax(x):
    """softmax and log-sum-exp over the last axis; a row of -inf gives zeros and -inf"""
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
    t = e.sum(-1, keepdim=True)
    return e / torch.where(t == 0, 1.0, t), (m + torch.log(t)).squeeze(-1)


def _run_decode(s):
    c = s["case"]
    if own:
        r = s["step"](s["Q"], s["k_pages"], s["v_pages"], s["table"], s["kv_len"], s["prefix_table"])
        return r["out"], r["lse"]
    p, n, G = c["page"], c["prefix"], c["H_kv"]
    Q = s["Q"].float().unflatten(1, (G, c["H_q"] // G))
    j = torch.arange(c["hi"], device=DEV)
    seen = j[None] < s["kv_len"][:, None]
    slot = torch.where(seen, s["table"][:, j // p].long() * p + j % p, 0)
    K = _unpack(*_rows4(s["k_pages"], slot, p))
    V = _unpack(*_rows4(s["v_pages"], slot, p)).masked_fill_(~seen[..., None, None], 0.0)
    x = torch.einsum("bgrd,bjgd->bgrj", Q, K) / math.sqrt(DH)
    x.masked_fill_(~seen[:, None, None], -math.inf)
    if n:
        j = torch.arange(n, device=DEV)
        slot = s["prefix_table"][j // p].long() * p + j % p
        Kp, Vp = _unpack(*_rows4(s["k_pages"], slot, p)), _unpack(*_rows4(s["v_pages"], slot, p))
        x = torch.cat([torch.einsum("bgrd,jgd->bgrj", Q, Kp) / math.sqrt(DH), x], -1)
    a, lse = _softmax(x)
    o = torch.einsum("bgrj,bjgd->bgrd", a[..., n:], V)
    if n:
        o = o + torch.einsum("bgrj,jgd->bgrd", a[..., :n], Vp)
    return o.flatten(1, 2).to(s["Q"].dtype), lse.flatten(1)


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "rotate":
        return _exact_turn(case, s, "Q", "w_q"), _exact_turn(case, s, "K", "w_k")
    if op == "store":
        return tuple(_exact_held(s[x], s["slot"]) for x in ("K", "V"))
    if op == "append" and case["bits"] == 4:
        k = _exact_turn(case, s, "K", "w_k").to(DTYPES[case["dtype"]])  # (what the cache takes in)
        return _exact_turn(case, s, "Q", "w_q"), _exact_held(k, s["slot"]), _exact_held(s["V"], s["slot"])
    if op == "append":
        k, v = _exact_turn(case, s, "K", "w_k"), s["V"].double()
        pages, p = s["k_pages"].shape[:2]
        src = torch.full((pages * p + 1,), -1, dtype=torch.long, device=DEV)
        src[s["slot"].long()] = torch.arange(case["T"], device=DEV)  # -1 is the last entry, cut off
        src = src[:-1]
        held = [(x[src.clamp(min=0)] * (src >= 0).double()[:, None, None]).view(pages, p, case["H_kv"], DH) for x in (k, v)]
        return (_exact_turn(case, s, "Q", "w_q"), *held)
    return _exact_decode(case, s)


def _exact_turn(case, s, name, weights):
    """pairs (i, i + 64) as complex numbers, times exp(i angle)"""
    x = s[name].double()
    if case["norm"]:
        x = x / (x.square().sum(-1, keepdim=True) / DH + EPS).sqrt() * s[weights].double()
    at = torch.stack([s["pos"][a].double() for a in _axis(case)], 1)
    turn = torch.polar(torch.ones_like(at), at * torch.tensor(_freq(case), dtype=torch.float64, device=DEV))
    z = torch.complex(x[..., :64].contiguous(), x[..., 64:].contiguous()) * turn[:, None]
    return torch.cat([z.real, z.imag], -1)


def _exact_held(x, slot):
    """what the nearest code stands for, with a scale of 8 bits"""
    v = x.double().view(*x.shape[:2], 4, 32) if x.is_contiguous() else x.double().reshape(*x.shape[:2], 4, 32)
    at = v.abs().argmax(-1, keepdim=True)
    most = v.gather(-1, at).abs()
    e = torch.where((v == most).any(-1, keepdim=True), most, -most)
    d = (-e / 8).float().to(torch.bfloat16).double()
    n = torch.nan_to_num(v / d).round().clamp(-8, 7)
    return (n * d * (slot >= 0).double()[:, None, None, None]).reshape(x.shape)


def _exact_rows(pages, table, n, p):
    """a sequence's n rows [n, H, 128], value by value"""
    H = pages.shape[1]
    j = torch.arange(n, device=DEV)
    block = pages[table[j // p].long()]                       # [n, H, p * 72]
    at = torch.arange(DH, device=DEV)
    q, g, t = at // 32, at % 32 // 4, at % 4
    byte = ((j % p)[:, None] * 64 + 2 * (4 * g + q) + t // 2)[:, None].expand(n, H, DH)
    code = (block.gather(2, byte).long() >> (4 * (t % 2))) & 15
    low = (p * 64 + (j % p)[:, None] * 8 + 2 * q)[:, None].expand(n, H, DH)
    bits = block.gather(2, low).int() << 16 | block.gather(2, low + 1).int() << 24
    return (code - 8).double() * bits.view(torch.float32).double()


def _exact_decode(case, s):
    H_q, H_kv, p = case["H_q"], case["H_kv"], case["page"]
    out = torch.zeros(s["Q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["Q"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    pre = [_exact_rows(s[x], s["prefix_table"], case["prefix"], p) for x in ("k_pages", "v_pages")] if case["prefix"] else None
    for b in range(case["B"]):
        K, V = (_exact_rows(s[x], s["table"][b], int(s["kv_len"][b]), p) for x in ("k_pages", "v_pages"))
        if pre:
            K, V = torch.cat([pre[0], K]), torch.cat([pre[1], V])
        heads = torch.arange(H_q, device=DEV) * H_kv // H_q
        for g in range(H_kv):
            rows = heads == g
            x = (s["Q"][b, rows].double() @ K[:, g].T) * DH ** -0.5
            lse[b, rows] = torch.logsumexp(x, 1)
            out[b, rows] = torch.softmax(x, 1) @ V[:, g]
    return out, lse
