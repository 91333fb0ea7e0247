"""What the attention and cache operators behind the pruning are measured on.

After the in-LLM pruning step a serving program attends over the pruned prompts, puts the
surviving key/value rows and the new tokens' rows into a paged cache, and decodes; several
questions about one image or video share its long prefix. Four operators do that:

  prompt  PromptAttention     attention over whole prompts: packed sequences of different
                              lengths, causal, grouped heads, an optional shared prefix
  tables  PageTables          block tables and slot maps of a paged cache, from the requests'
                              lengths: pages of ended requests go back, new tokens get theirs
  append  provip_kv_append    key/value rows of new tokens into the pages, by slot map
  decode  DecodeAttention     one token per request over shared prefix pages and own pages

Each case is a dict of plain values. `run` computes an operator in elementary torch
operations in 32 bits, or, where `own` is true, through the package's entry points.
Lengths are a function of the case alone (`mix` is their seed), values of the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
DH = 128            # head size of every model here
SYS = 35            # system rows in front of the visual ones
MOST_LOGITS = 2.5e9  # padded logits of a plain pass
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # attention over prompts -------------------------------------------------------
        # the follow-up question of one user: 48 new rows over a pruned image's 211 keys
        dict(name="prompt_follow_up", op="prompt", dtype="bf16", B=1, H_q=32, H_kv=32, lo=211, hi=211, q=48,
             causal=True, prefix=0, mix=1),
        # a 7B fp32 model's prompt after the pre-LLM stage: 35 + 192 + 64 rows
        dict(name="prompt_one_fp32", op="prompt", dtype="f32", B=1, H_q=32, H_kv=32, lo=291, hi=291, q=0,
             causal=True, prefix=0, mix=2),
        # anyres batch of 8 after the pre-LLM stage, text lengths apart: packed, ragged
        dict(name="prompt_packed_anyres", op="prompt", dtype="bf16", B=8, H_q=32, H_kv=32, lo=1000, hi=1091, q=0,
             causal=True, prefix=0, mix=3),
        # one video before any pruning: 35 + 9216 + 128 rows, 28 heads in 4 groups
        dict(name="prompt_video", op="prompt", dtype="bf16", B=1, H_q=28, H_kv=4, lo=9379, hi=9379, q=0,
             causal=True, prefix=0, mix=4),
        # 16 questions about one pruned video: every row sees its 35 + 2304 rows
        dict(name="prompt_shared_video", op="prompt", dtype="bf16", B=16, H_q=28, H_kv=4, lo=9, hi=128, q=0,
             causal=True, prefix=SYS + 2304, mix=5),
        # block tables and slot maps ---------------------------------------------------
        # one decode step of 256 requests, one in 16 of them at its end
        dict(name="tables_decode_256", op="tables", B=256, lo=163, hi=1091, new_lo=1, new_hi=1, ended=16, page=16,
             supply=1.5, mix=6),
        # 64 prompts arrive at once, and the pages do not suffice for the last of them
        dict(name="tables_prompts_64", op="tables", B=64, lo=0, hi=0, new_lo=163, new_hi=1091, ended=0, page=64,
             supply=0.9, mix=7),
        # rows into pages --------------------------------------------------------------
        # the 256 rows of a decode step, 4 key/value heads
        dict(name="append_decode_256", op="append", dtype="bf16", T=256, H_kv=4, page=16, mix=8),
        # the rows of an anyres batch's prompts, 32 key/value heads
        dict(name="append_anyres", op="append", dtype="bf16", T=8 * 1091 - 3, H_kv=32, page=64, mix=9),
        # decoding -------------------------------------------------------------------
        # a single user's token over a pruned image (35 + 64 + 112 rows)
        dict(name="decode_one", op="decode", dtype="bf16", B=1, H_q=32, H_kv=32, lo=211, hi=211, prefix=0, page=16,
             mix=10),
        # 32 users with an image each, no shared rows
        dict(name="decode_ragged_32", op="decode", dtype="bf16", B=32, H_q=32, H_kv=32, lo=163, hi=1091, prefix=0,
             page=16, mix=11),
        # 64 questions about one unpruned video
        dict(name="decode_shared_video", op="decode", dtype="bf16", B=64, H_q=28, H_kv=4, lo=1, hi=512,
             prefix=SYS + 9216, page=64, mix=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "decode", "decode", "tables", "append"])
    mix = rng.randrange(1 << 20)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    H_q, H_kv = rng.choice([(32, 32), (40, 40), (28, 4)])
    page = rng.choice([16, 32, 64, 128])
    if op == "prompt":
        hi = _log(rng, 1, 9379)
        c = dict(op=op, dtype=dtype, B=_log(rng, 1, 32), H_q=H_q, H_kv=H_kv, lo=rng.randint(max(hi // 4, 1), hi), hi=hi,
                 q=rng.choice([0, 0, _log(rng, 1, hi)]), causal=rng.random() < 0.8,
                 prefix=rng.choice([0, 0, _log(rng, 1, SYS + 9216)]), mix=mix)
        most = max(work(x)["flops"] for x in listed() if x["op"] == op)
        while work(c)["flops"] > most or c["B"] * H_q * max(_prompt_lens(c)[0]) * (c["prefix"] + c["hi"]) > MOST_LOGITS:
            if c["B"] > 1:
                c["B"] = (c["B"] + 1) // 2
            else:
                c["hi"], c["prefix"] = c["hi"] * 4 // 5, c["prefix"] * 4 // 5
                c["lo"] = min(c["lo"], c["hi"])
        return c
    if op == "decode":
        hi = _log(rng, 1, 9379)
        c = dict(op=op, dtype=dtype, B=_log(rng, 1, 256), H_q=H_q, H_kv=H_kv, lo=rng.randint(max(hi // 4, 1), hi), hi=hi,
                 prefix=rng.choice([0, _log(rng, 1, SYS + 9216)]), page=page, mix=mix)
        most = max(work(x)["bytes"] for x in listed() if x["op"] == op)
        flops = max(work(x)["flops"] for x in listed() if x["op"] == op)
        while work(c)["bytes"] > most or work(c)["flops"] > flops:
            if c["B"] > 1:
                c["B"] = (c["B"] + 1) // 2
            else:
                c["hi"], c["prefix"] = c["hi"] * 4 // 5, c["prefix"] * 4 // 5
                c["lo"] = min(c["lo"], c["hi"])
        return c
    if op == "tables":
        B = _log(rng, 1, 512)
        hi = rng.choice([0, _log(rng, 1, 4096)])
        new_hi = min(rng.choice([1, 1, _log(rng, 1, 2048)]), 65536 // B)
        return dict(op=op, B=B, lo=rng.randint(0, hi), hi=hi, new_lo=rng.randint(0, new_hi), new_hi=new_hi,
                    ended=rng.choice([0, 4, 16]), page=page, supply=rng.choice([1.5, 1.0, 0.7]), mix=mix)
    T = _log(rng, 1, 8 * 1091 * 32 // H_kv)
    return dict(op=op, dtype="bf16" if T * H_kv > 140000 else dtype, T=T, H_kv=H_kv, page=page, mix=mix)


# ---------------------------------------------------------------------------
# lengths of a case
# ---------------------------------------------------------------------------
def _spread(n, lo, hi, mix):
    """n lengths from lo to hi, evenly apart, in an order drawn from mix."""
    v = [lo + (hi - lo) * i // max(n - 1, 1) for i in range(n)]
    random.Random(mix).shuffle(v)
    return v


def _prompt_lens(c):
    k = _spread(c["B"], c["lo"], c["hi"], c["mix"])
    return [min(x, c["q"]) if c["q"] else x for x in k], k


def _table_lens(c):
    kv = _spread(c["B"], c["lo"], c["hi"], c["mix"])
    new = _spread(c["B"], c["new_lo"], c["new_hi"], c["mix"] + 1)
    return kv, [-1 if c["ended"] and i % c["ended"] == c["ended"] - 1 else x for i, x in enumerate(new)]


def _ceil(a, b):
    return -(-a // b)


def work(case):
    c, op = case, case["op"]
    es = 4 if c.get("dtype") == "f32" else 2
    if op == "prompt":
        q, k = _prompt_lens(c)
        pairs = 0
        for lq, lk in zip(q, k):
            # visible own keys: lk a row, or i + 1 + lk - lq for row i (lq <= lk here)
            pairs += lq * c["prefix"] + (lq * (lk - lq) + lq * (lq + 1) // 2 if c["causal"] else lq * lk)
        n = es * DH * (2 * sum(q) * c["H_q"] + 2 * (sum(k) + c["prefix"]) * c["H_kv"]) + 4 * sum(q) * c["H_q"]
        return {"bytes": n, "flops": 4 * DH * c["H_q"] * pairs}
    if op == "decode":
        k = sum(_spread(c["B"], c["lo"], c["hi"], c["mix"]))
        n = es * DH * (2 * c["B"] * c["H_q"] + 2 * (k + c["prefix"]) * c["H_kv"]) + 4 * c["B"] * (c["H_q"] + 1)
        n += 4 * _ceil(k + c["prefix"], c["page"])
        return {"bytes": n, "flops": 4 * DH * c["H_q"] * (k + c["B"] * c["prefix"])}
    if op == "append":
        return {"bytes": 4 * es * DH * c["T"] * c["H_kv"] + 4 * c["T"], "flops": 0}
    kv, new = _table_lens(c)
    p = c["page"]
    moved = sum(_ceil(a, p) if b < 0 else _ceil(a + b, p) - _ceil(a, p) for a, b in zip(kv, new))
    return {"bytes": 4 * (4 * c["B"] + 2 * moved + sum(max(b, 0) for b in new) + 3), "flops": 0}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _starts(v):
    out = [0]
    for x in v:
        out.append(out[-1] + x)
    return out


def _units(g, H_kv):
    u = torch.randn(H_kv, DH, device=DEV, generator=g)
    return u / u.norm(dim=1, keepdim=True)


def prepare(case, seed):
    return {"prompt": _prepare_prompt, "tables": _prepare_tables, "append": _prepare_append,
            "decode": _prepare_decode}[case["op"]](case, seed)


def _prepare_prompt(c, seed):
    """Queries share a direction within a group, the first key of a sequence (or of the prefix)
    is a sink along it, as in real attention. Whole prompts are slices of one fused
    query/key/value buffer, as a model's projection leaves them."""
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    q, k = _prompt_lens(c)
    H_q, H_kv, Tq, Tk, n = c["H_q"], c["H_kv"], sum(q), sum(k), c["prefix"]
    u = _units(g, H_kv)
    qs = torch.randn(Tq, H_q, DH, device=DEV, generator=g) + u.repeat_interleave(H_q // H_kv, 0)
    ks = torch.randn(Tk, H_kv, DH, device=DEV, generator=g)
    vs = torch.randn(Tk, H_kv, DH, device=DEV, generator=g)
    s = dict(case=c, q_start=_i32(_starts(q)[:-1]), q_len=_i32(q), k_start=_i32(_starts(k)[:-1]), k_len=_i32(k))
    if n:
        kp = torch.randn(n, H_kv, DH, device=DEV, generator=g)
        kp[0] = 8 * math.sqrt(DH) * u
        s["K_prefix"] = kp.to(dt)
        s["V_prefix"] = torch.randn(n, H_kv, DH, device=DEV, generator=g).to(dt)
    else:
        ks[s["k_start"].long()] = 8 * math.sqrt(DH) * u
    if c["q"]:
        s["Q"], s["K"], s["V"] = qs.to(dt), ks.to(dt), vs.to(dt)
    else:
        s["Q"], s["K"], s["V"] = torch.cat([qs, ks, vs], 1).to(dt).split([H_q, H_kv, H_kv], 1)
    if own:
        from paper_2608_25332_gb300 import provip as P
        s["step"] = P.PromptAttention(Tq, c["B"], H_q, H_kv, max(q), max(k), prefix_len=n, causal=c["causal"], dtype=dt,
                                      device=DEV)
    return s


def _prepare_tables(c, seed):
    """A pool whose free pages are in a seeded order; the requests' tables and others' hold the rest."""
    g, p = _gen(seed), c["page"]
    kv, new = _table_lens(c)
    held = [_ceil(x, p) for x in kv]
    width = max([_ceil(a + max(b, 0), p) for a, b in zip(kv, new)] + [1])
    back = sum(h for h, b in zip(held, new) if b < 0)
    need = sum(_ceil(a + b, p) - h for a, b, h in zip(kv, new, held) if b >= 0)
    free = max(int(need * c["supply"]) - back, 0) + 1
    n = sum(held) + free + 512
    order = torch.randperm(n, device=DEV, generator=g).to(torch.int32)
    table = torch.full((c["B"], width), -1, dtype=torch.int32, device=DEV)
    col = torch.arange(width, device=DEV)
    table[col[None] < _i32(held)[:, None]] = order[free:free + sum(held)]
    stack = torch.full((n,), -1, dtype=torch.int32, device=DEV)
    stack[:free] = order[:free]
    rows = sum(max(b, 0) for b in new)
    s = dict(case=c, kv_len=_i32(kv), new_len=_i32(new), table=table, stack=stack, count=_i32([free]), rows=rows)
    if own:
        from paper_2608_25332_gb300 import provip as P
        s["step"] = P.PageTables(c["B"], p, rows, device=DEV)
    return s


def _prepare_append(c, seed):
    """Rows go to slots spread over the pool; one row in 50 has no slot (its request got no page)."""
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    T, H, p = c["T"], c["H_kv"], c["page"]
    pages = _ceil(T, p) + 2
    slot = torch.randperm(pages * p, device=DEV, generator=g)[:T].to(torch.int32)
    slot[torch.rand(T, device=DEV, generator=g) < 0.02] = -1
    kv = torch.randn(T, 2 * H, DH, device=DEV, generator=g).to(dt)
    return dict(case=c, K=kv[:, :H], V=kv[:, H:], slot=slot, k_pages=torch.zeros(pages, p, H, DH, dtype=dt, device=DEV),
                v_pages=torch.zeros(pages, p, H, DH, dtype=dt, device=DEV))


def _prepare_decode(c, seed):
    """Pages in a seeded order; what no request holds, and the slots past each length, are NaN:
    whoever reads them shows it."""
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
    u = _units(g, H_kv)
    pool = torch.full((2, pages * p, H_kv, DH), math.nan, dtype=dt, device=DEV)
    at = torch.arange(width * p, device=DEV)
    own_slots = (table.long()[:, at // p] * p + at % p)[at[None] < kv_len[:, None]]
    at = torch.arange(n, device=DEV)
    slots = torch.cat([prefix_table.long()[at // p] * p + at % p if n else at, own_slots])
    for i in range(2):
        pool[i, slots] = torch.randn(len(slots), H_kv, DH, device=DEV, generator=g).to(dt)
    first = slots[:1] if n else table[:, 0].long() * p
    pool[0, first] = (8 * math.sqrt(DH) * u).to(dt)
    Q = (torch.randn(B, H_q, DH, device=DEV, generator=g) + u.repeat_interleave(H_q // H_kv, 0)).to(dt)
    s = dict(case=c, Q=Q, k_pages=pool[0].view(pages, p, H_kv, DH), v_pages=pool[1].view(pages, p, H_kv, DH), table=table,
             kv_len=kv_len, prefix_table=prefix_table if n else None)
    if own:
        from paper_2608_25332_gb300 import provip as P
        s["step"] = P.DecodeAttention(B, H_q, H_kv, max(lens), prefix_len=n, dtype=dt, device=DEV)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(state):
    return {"prompt": _run_prompt, "tables": _run_tables, "append": _run_append,
            "decode": _run_decode}[state["case"]["op"]](state)


def _softmax(x):
    """softmax and log-sum-exp over the last axis; a row of -inf gives zeros and -inf"""
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
    t = e.sum(-1, keepdim=True)
    return e / torch.where(t == 0, 1.0, t), (m + torch.log(t)).squeeze(-1)


def _run_prompt(s):
    c = s["case"]
    if own:
        r = s["step"](s["Q"], s["K"], s["V"], s["q_start"], s["q_len"], s["k_start"], s["k_len"], s.get("K_prefix"),
                      s.get("V_prefix"))
        return r["out"], r["lse"]
    # sequences padded to the longest: [B, rows, groups, heads of a group, DH]
    (q, k), G, R, n = _prompt_lens(c), c["H_kv"], c["H_q"] // c["H_kv"], c["prefix"]
    i, j = torch.arange(max(q), device=DEV), torch.arange(max(k), device=DEV)
    q_in, k_in = i[None] < s["q_len"][:, None], j[None] < s["k_len"][:, None]
    Q = s["Q"][((s["q_start"][:, None] + i) * q_in).long()].float().unflatten(2, (G, R))
    rows = ((s["k_start"][:, None] + j) * k_in).long()
    K, V = s["K"][rows].float(), s["V"][rows].float()
    x = torch.einsum("bigrd,bjgd->bgrij", Q, K) / math.sqrt(DH)
    seen = k_in[:, None, :]
    if c["causal"]:
        seen = seen & (j[None, None] <= i[None, :, None] + (s["k_len"] - s["q_len"])[:, None, None])
    x.masked_fill_(~seen[:, None, None], -math.inf)
    if n:
        Kp, Vp = s["K_prefix"].float(), s["V_prefix"].float()
        x = torch.cat([torch.einsum("bigrd,jgd->bgrij", Q, Kp) / math.sqrt(DH), x], -1)
    a, lse = _softmax(x)
    o = torch.einsum("bgrij,bjgd->bigrd", a[..., n:], V)
    if n:
        o = o + torch.einsum("bgrij,jgd->bigrd", a[..., :n], Vp)
    return o[q_in].flatten(1, 2).to(s["Q"].dtype), lse.permute(0, 3, 1, 2)[q_in].flatten(1)


def _run_tables(s):
    p = s["case"]["page"]
    if own:
        r = s["step"](s["kv_len"], s["new_len"], s["stack"], s["count"], s["table"])
        return r["kv_len"], r["row_start"], r["slot_map"], r["free_count"], s["table"], s["stack"]
    kv, new, table, stack = s["kv_len"].long(), s["new_len"].long(), s["table"].clone(), s["stack"].clone()
    B, width = table.shape
    col = torch.arange(width, device=DEV)
    held, end = (kv + p - 1) // p, new < 0
    add = new.clamp(min=0)
    # pages of ended requests on top of the stack, in the tables' order
    given = end[:, None] & (col[None] < held[:, None])
    count = s["count"].long()
    back = table[given]
    stack[count + torch.arange(len(back), device=DEV)] = back
    total = count + len(back)
    # pages off the top of it, in the requests' order
    need = torch.where(end, 0, (kv + add + p - 1) // p - held)
    upto = need.cumsum(0)
    ok = ~end & ((need == 0) | (upto <= total))
    take = torch.where(ok, need, 0)
    at = col[None] - held[:, None]
    fresh = (at >= 0) & (at < take[:, None])
    from_top = total - 1 - ((upto - need)[:, None] + at)
    table[fresh] = stack[from_top[fresh]]
    row_start = torch.cat([torch.zeros(1, dtype=torch.long, device=DEV), add.cumsum(0)])
    t = torch.arange(s["rows"], device=DEV)
    b = (t[:, None] >= row_start[None, 1:]).sum(1)
    pos = kv[b] + t - row_start[b]
    slot = torch.where(ok[b], table[b, torch.where(ok[b], pos // p, 0)].long() * p + pos % p, -1)
    kv_out = torch.where(end, 0, torch.where(ok, kv + add, kv))
    return (kv_out.int(), row_start.int(), slot.int(), (total - take.sum()).int(), table, stack)


def _run_append(s):
    if own:
        from paper_2608_25332_gb300 import provip as P
        P.provip_kv_append(s["K"], s["V"], s["slot"], s["k_pages"], s["v_pages"])
    else:
        keep = s["slot"] >= 0
        at = s["slot"][keep].long()
        s["k_pages"].flatten(0, 1)[at] = s["K"][keep]
        s["v_pages"].flatten(0, 1)[at] = s["V"][keep]
    return s["k_pages"], s["v_pages"]


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
    k_rows, v_rows = s["k_pages"].flatten(0, 1), s["v_pages"].flatten(0, 1)
    K, V = k_rows[slot].float(), v_rows[slot].float().masked_fill_(~seen[..., None, None], 0.0)
    x = torch.einsum("bgrd,bjgd->bgrj", Q, K) / math.sqrt(DH)
    x.masked_fill_(~seen[:, None, None], -math.inf)
    if n:
        j = torch.arange(n, device=DEV)
        slot = s["prefix_table"][j // p].long() * p + j % p
        Kp, Vp = k_rows[slot].float(), v_rows[slot].float()
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
    op = case["op"]
    if op == "tables":
        return None  # whole numbers
    s = prepare(case, seed)
    if op == "append":
        return tuple(_exact_append(case, s, x) for x in ("K", "V"))
    H_q, H_kv = case["H_q"], case["H_kv"]
    out = torch.zeros(s["Q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["Q"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    for b in range(case["B"]):
        if op == "prompt":
            q0, lq, k0, lk = (int(s[x][b]) for x in ("q_start", "q_len", "k_start", "k_len"))
            rows, K, V = slice(q0, q0 + lq), s["K"][k0:k0 + lk], s["V"][k0:k0 + lk]
            # own key j is hidden from row i where j - i exceeds the lengths' difference
            hidden = (torch.ones(lq, lk, dtype=torch.bool, device=DEV).triu(lk - lq + 1) if case["causal"]
                      else torch.zeros(lq, lk, dtype=torch.bool, device=DEV))
            pre = (s["K_prefix"], s["V_prefix"]) if case["prefix"] else ()
        else:
            rows, n, p = slice(b, b + 1), int(s["kv_len"][b]), case["page"]
            K, V = (x[s["table"][b, :_ceil(n, p)].long()].reshape(-1, H_kv, DH)[:n] for x in (s["k_pages"], s["v_pages"]))
            hidden = torch.zeros(1, n, dtype=torch.bool, device=DEV)
            pre = tuple(x[s["prefix_table"].long()].reshape(-1, H_kv, DH)[:case["prefix"]]
                        for x in (s["k_pages"], s["v_pages"])) if case["prefix"] else ()
        if pre:
            K, V = torch.cat([pre[0], K]), torch.cat([pre[1], V])
            hidden = torch.nn.functional.pad(hidden, (case["prefix"], 0))
        for h in range(H_q):
            kd, vd = K[:, h * H_kv // H_q].double(), V[:, h * H_kv // H_q].double()
            x = (s["Q"][rows, h].double() @ kd.T) * DH ** -0.5
            x[hidden] = -math.inf
            lse[rows, h] = torch.logsumexp(x, 1)
            out[rows, h] = torch.softmax(x, 1) @ vd
    return out, lse


def _exact_append(case, s, which):
    """For every slot of the pool the row that goes there, or zeros."""
    pages = s["k_pages"].shape[0]
    src = torch.full((pages * case["page"] + 1,), -1, dtype=torch.long, device=DEV)
    src[s["slot"].long()] = torch.arange(case["T"], device=DEV)  # -1 is the last entry, cut off
    src = src[:-1]
    rows = s[which].double()[src.clamp(min=0)] * (src >= 0).double()[:, None, None]
    return rows.view(pages, case["page"], case["H_kv"], DH)
