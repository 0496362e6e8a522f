"""Performance cases of the serving operators: page tables, rotary positions with the store into a paged cache, causal
attention over packed prompts, attention of new tokens over the paged cache.

A program that answers requests with a transformer calls them in this order for every step: the tables (which page and
slot each new token gets), per layer the rotation of queries and keys that also stores keys and values, then the
attention: over the packed prompts themselves where nothing is cached yet, else over the cache.  All lengths live on
the GPU; the host knows upper bounds.  `own` chooses between plain torch operations in 32 bits and the framework's calls.
"""
from __future__ import annotations

import math
import random
from types import SimpleNamespace

import numpy as np
import torch

own = False

_DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_CODE = {"f32": 0, "bf16": 1, "f16": 4}


# ------------------------------------------------------------------------------------------------ cases
def _log(rng, lo, hi):
    """An integer of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, round(lo * (hi / lo) ** rng.random())))


def _text(lengths):
    return " ".join(str(n) for n in lengths)


def listed():
    r = random.Random(176)
    return [
        # one decode step's tables for a batch of conversations: latency
        {"name": "tables, decode of 48", "op": "tables", "page": 16, "past": _text(r.randint(16, 4000) for _ in range(48)),
         "new": _text([1] * 48), "pad": 16},
        # a large ingest: 500 requests of ragged prompts, some of them continued, 400k tokens
        {"name": "tables, ingest of 500", "op": "tables", "page": 32, "past": _text(r.choice([0, 0, r.randint(1, 9000)]) for _ in range(500)),
         "new": _text(_log(r, 1, 4000) for _ in range(500)), "pad": 77},
        # rotary positions and cache store of a decode step
        {"name": "rope store, decode of 64", "op": "rope", "dtype": "bf16", "tokens": 64, "pad": 0, "heads": 32, "kv": 8, "dim": 128, "rot": 128,
         "axes": "64", "local": False, "pairs": False, "theta": 500000.0, "far": 32000, "page": 16},
        # the same for a step of prompts: partial rotation of adjacent pairs at far positions, some padding tokens
        {"name": "rope store, 8191 tokens", "op": "rope", "dtype": "f16", "tokens": 8191, "pad": 65, "heads": 28, "kv": 4, "dim": 96, "rot": 64,
         "axes": "32", "local": False, "pairs": True, "theta": 1000000.0, "far": 1000000, "page": 64},
        # patches of a video: time, height and width each turn a section of the head; no cache
        {"name": "rope, video 16x42x60", "op": "rope", "dtype": "bf16", "tokens": 40320, "pad": 0, "heads": 12, "kv": 12, "dim": 64, "rot": 64,
         "axes": "8 12 12", "local": True, "pairs": False, "theta": 10000.0, "far": 60, "page": 0},
        # one short prompt: latency
        {"name": "prompt, 37 tokens", "op": "prompt", "dtype": "bf16", "lens": "37", "pad": 0, "heads": 12, "kv": 12, "dim": 64, "packed": True},
        # the encoder's ordinary batch sizes, as a causal network with grouped heads
        {"name": "prompt, 8 of 16..512", "op": "prompt", "dtype": "bf16", "lens": _text(r.randint(16, 512) for _ in range(8)), "pad": 0,
         "heads": 12, "kv": 4, "dim": 64, "packed": True},
        # ragged prompts, an empty one and a single token among them, odd group and head sizes
        {"name": "prompt, ragged to 3000", "op": "prompt", "dtype": "f16", "lens": "1 2999 0 777 128 2049 1500 5", "pad": 11, "heads": 15, "kv": 3,
         "dim": 80, "packed": False},
        # a long document beside ordinary prompts: the largest
        {"name": "prompt, 16k and others", "op": "prompt", "dtype": "bf16", "lens": "16384 4096 2000 8191 1025", "pad": 0, "heads": 32, "kv": 8,
         "dim": 128, "packed": False},
        # one conversation, one token
        {"name": "paged, decode of 1", "op": "paged", "dtype": "bf16", "past": "776", "new": "1", "pad": 0, "heads": 12, "kv": 4, "dim": 64, "page": 16},
        # the ordinary decode step: 64 conversations of ragged length
        {"name": "paged, decode of 64", "op": "paged", "dtype": "bf16", "past": _text(_log(r, 100, 8000) for _ in range(64)), "new": _text([1] * 64),
         "pad": 0, "heads": 32, "kv": 8, "dim": 128, "page": 16},
        # a chunk of a long document, the next chunks of short ones and single tokens in one step
        {"name": "paged, mixed chunks", "op": "paged", "dtype": "f16", "past": "98765 0 3000 511 12000 2047 64 9999", "new": "1024 700 1 33 1 5 1 2",
         "pad": 9, "heads": 32, "kv": 8, "dim": 128, "page": 64},
    ]


def draw(rng):
    op = rng.choice(["tables", "rope", "rope", "prompt", "prompt", "prompt", "paged", "paged", "paged", "paged"])
    pad = rng.choice([0, 0, rng.randint(1, 99)])
    if op == "tables":
        n = _log(rng, 1, 500)
        most = _log(rng, 1, 3000)
        return {"op": op, "page": rng.choice([8, 16, 24, 32, 64, 128, 256]), "past": _text(rng.choice([0, _log(rng, 1, 9000)]) for _ in range(n)),
                "new": _text(rng.choice([0, 1, rng.randint(1, most), _log(rng, 1, most)]) for _ in range(n)), "pad": pad}
    dtype, kv = rng.choice(["bf16", "bf16", "f16"]), rng.choice([1, 2, 3, 4, 5, 8])
    heads = kv * rng.choice([1, 1, 2, 3, 4, 5, 6, 7, 8])
    if op == "rope":
        dim = rng.choice([64, 64, 80, 96, 128, 128, 128])
        rot = rng.choice([dim, dim, dim // 2])
        n_axes, left = rng.choice([1, 2, 3]), rot // 2
        axes = []
        for a in range(n_axes - 1):
            axes.append(max(1, min(left - (n_axes - 1 - a), round(left * rng.uniform(0.2, 0.6)))))
            left -= axes[-1]
        axes.append(left)
        cached = n_axes == 1 or rng.random() < 0.5
        return {"op": op, "dtype": rng.choice([dtype, "f32"]), "tokens": _log(rng, 1, 12000), "pad": pad if cached else 0, "heads": heads, "kv": kv, "dim": dim,
                "rot": rot, "axes": _text(axes), "local": n_axes > 1 and rng.random() < 0.5, "pairs": rng.random() < 0.5,
                "theta": rng.choice([1e4, 5e5, 1e6]), "far": _log(rng, 40, 1000000), "page": rng.choice([16, 32, 48, 64, 128]) if cached else 0}
    dim = rng.choice([32, 64, 64, 64, 72, 80, 96, 112, 128, 128, 128])
    n = _log(rng, 1, 24)
    if op == "prompt":
        most = _log(rng, 30, 9000)
        lens = [rng.choice([0, 1, rng.randint(1, most), _log(rng, 1, most), most]) for _ in range(n)]
        while sum(v * v for v in lens) > 1.5e8:
            lens = [v // 2 for v in lens]
        if not sum(lens):
            lens[0] = most
        return {"op": op, "dtype": dtype, "lens": _text(lens), "pad": pad, "heads": heads, "kv": kv, "dim": dim, "packed": rng.random() < 0.5}
    single = rng.random() < 0.5
    most, far = _log(rng, 2, 1500), _log(rng, 50, 30000)
    past = [rng.choice([0, _log(rng, 1, far), rng.randint(1, far)]) for _ in range(n)]
    new = [1 if single else rng.choice([0, 1, 1, rng.randint(1, most), _log(rng, 1, most)]) for _ in range(n)]
    if not sum(new):
        new[0] = most
    while sum((p + v / 2) * v for p, v in zip(past, new)) > 8e7 or sum(past) > 130000:
        past, new = [v // 2 for v in past], [(v + 1) // 2 for v in new]
    return {"op": op, "dtype": dtype, "past": _text(past), "new": _text(new), "pad": pad, "heads": heads, "kv": kv, "dim": dim,
            "page": rng.choice([8, 16, 16, 32, 64, 128, 256])}


def _ints(text):
    return [int(v) for v in text.split()]


# ------------------------------------------------------------------------------------------------ inputs
def _pages(n, page):
    return -(-n // page)


def _frequencies(case):
    """Radians per position and the axis of each rotated pair.  `local`: every axis has the whole ladder of frequencies in
    its own section (images, video); else one ladder runs over all sections."""
    freq, axis = [], []
    for a, n in enumerate(_ints(case["axes"])):
        for j in range(n):
            freq.append(case["theta"] ** -(j / n if case["local"] else 2 * len(freq) / case["rot"]))
            axis.append(a)
    return freq, axis


def _prepare_tables(case, st, gen):
    past, new, page = _ints(case["past"]), _ints(case["new"]), case["page"]
    dev = "cuda"
    st.n, st.cap, st.page = len(past), sum(new) + case["pad"], page
    have = [_pages(p, page) for p in past]
    take = sum(_pages(p + v, page) - h for p, v, h in zip(past, new, have))
    pool = torch.randperm(sum(have) + take + 20, generator=gen, device=dev, dtype=torch.int32)
    st.width = max(_pages(p + v, page) for p, v in zip(past, new)) + 3
    st.past, st.new = torch.tensor(past, dtype=torch.int32, device=dev), torch.tensor(new, dtype=torch.int32, device=dev)
    # the table as the steps before left it: the pages of the past, -1 behind them
    col = torch.arange(st.width, device=dev)
    h = torch.tensor(have, device=dev)
    at = (torch.cumsum(h, 0) - h)[:, None] + col
    st.table0 = torch.where(col < h[:, None], pool[at.clamp(max=pool.numel() - 1)], torch.full_like(pool[:1], -1)).contiguous()
    st.table = st.table0.clone()
    # free pages: some have been taken from the front by the steps before
    st.free = torch.cat([pool[:7], pool[sum(have):]]).contiguous()
    st.head = torch.tensor([7], dtype=torch.int32, device=dev)
    st.cu = torch.zeros(st.n + 1, dtype=torch.int32, device=dev)
    st.ctx = torch.zeros(st.n, dtype=torch.int32, device=dev)
    st.slots = torch.zeros(max(st.cap, 1), dtype=torch.int64, device=dev)[:st.cap]
    st.positions = torch.zeros(max(st.cap, 1), dtype=torch.int32, device=dev)[:st.cap]
    st.new_head = torch.zeros(1, dtype=torch.int32, device=dev)


def _prepare_rope(case, st, gen):
    dev, dt = "cuda", _DT[case["dtype"]]
    t, h, kv, d = case["tokens"] + case["pad"], case["heads"], case["kv"], case["dim"]
    st.t, st.code = t, _CODE[case["dtype"]]
    # queries, keys and values are slices of one projection, as networks have them
    qkv = torch.randn((t, h + 2 * kv, d), generator=gen, device=dev).to(dt)
    st.qkv = qkv
    st.q, st.k, st.v = qkv[:, :h], qkv[:, h:h + kv], qkv[:, h + kv:]
    axes = _ints(case["axes"])
    st.n_axes = len(axes)
    st.positions = torch.randint(0, case["far"], (len(axes), t), generator=gen, device=dev, dtype=torch.int32)
    st.freq, st.axis = _frequencies(case)
    st.q_out = torch.empty((t, h, d), dtype=dt, device=dev)
    st.k_out = st.slots = st.kc = st.vc = None
    if case["page"]:
        st.n_pages = _pages(case["tokens"], case["page"]) + 5
        st.kc = torch.zeros((st.n_pages, case["page"], kv, d), dtype=dt, device=dev)
        st.vc = torch.zeros_like(st.kc)
        slots = torch.randperm(st.n_pages * case["page"], generator=gen, device=dev)[:t]
        slots[case["tokens"]:] = -1                              # padding tokens are not stored
        st.slots = slots.contiguous()
    else:
        st.k_out = torch.empty((t, kv, d), dtype=dt, device=dev)


def _prepare_prompt(case, st, gen):
    dev, dt = "cuda", _DT[case["dtype"]]
    lens = _ints(case["lens"])
    st.lens, st.n, st.t = lens, len(lens), sum(lens) + case["pad"]
    h, kv, d = case["heads"], case["kv"], case["dim"]
    st.code = _CODE[case["dtype"]]
    x = torch.randn((st.t, h + 2 * kv, d), generator=gen, device=dev)
    x[:, :h] *= 1.5                                             # scores of standard deviation 1.5
    x = x.to(dt)
    st.q, st.k, st.v = x[:, :h], x[:, h:h + kv], x[:, h + kv:]
    if not case["packed"]:
        st.q, st.k, st.v = st.q.contiguous(), st.k.contiguous(), st.v.contiguous()
    st.cu_host = [0]
    for n in lens:
        st.cu_host.append(st.cu_host[-1] + n)
    st.cu = torch.tensor(st.cu_host, dtype=torch.int32, device=dev)
    st.out = torch.zeros((st.t, h, d), dtype=dt, device=dev)


def _prepare_paged(case, st, gen):
    dev, dt = "cuda", _DT[case["dtype"]]
    past, new, page = _ints(case["past"]), _ints(case["new"]), case["page"]
    h, kv, d = case["heads"], case["kv"], case["dim"]
    st.new_host, st.ctx_host = new, [p + v for p, v in zip(past, new)]
    st.n, st.t, st.code = len(new), sum(new) + case["pad"], _CODE[case["dtype"]]
    need = [_pages(c, page) for c in st.ctx_host]
    st.n_pages = sum(need) + 11
    st.width = max(need) + 2
    # a cache whose pages behind the last tokens hold what earlier requests left there
    st.kc = torch.randn((st.n_pages, page, kv, d), generator=gen, device=dev).to(dt)
    st.vc = torch.randn((st.n_pages, page, kv, d), generator=gen, device=dev).to(dt)
    st.q = (torch.randn((st.t, h, d), generator=gen, device=dev) * 1.5).to(dt)
    pool = torch.randperm(st.n_pages, generator=gen, device=dev, dtype=torch.int32)
    col, n = torch.arange(st.width, device=dev), torch.tensor(need, device=dev)
    at = (torch.cumsum(n, 0) - n)[:, None] + col
    st.table = torch.where(col < n[:, None], pool[at.clamp(max=st.n_pages - 1)], torch.full_like(pool[:1], -1)).contiguous()
    st.ctx = torch.tensor(st.ctx_host, dtype=torch.int32, device=dev)
    st.cu_host = [0]
    for v in new:
        st.cu_host.append(st.cu_host[-1] + v)
    st.cu = torch.tensor(st.cu_host, dtype=torch.int32, device=dev)
    st.most_new = max(new)
    st.out = torch.zeros((st.t, h, d), dtype=dt, device=dev)


def _own():
    from paper_2403_00176_b200 import binding
    return binding


def _inputs(case, seed):
    st = SimpleNamespace(case=case, op=case["op"])
    gen = torch.Generator(device="cuda").manual_seed(seed)
    {"tables": _prepare_tables, "rope": _prepare_rope, "prompt": _prepare_prompt, "paged": _prepare_paged}[st.op](case, st, gen)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:                                                       # what a serving program sets up once
        st.status = torch.zeros(1, dtype=torch.int32, device="cuda")      # where a call reports, read by the program when it likes
        if st.op == "rope":
            st.rotation = _own().Rotation(st.freq, st.axis, adjacent=case["pairs"])
        if st.op in ("prompt", "paged"):
            n = _own().sod2_attention_workspace_bytes(case["heads"], case["kv"], case["dim"])
            st.ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    return st


# ------------------------------------------------------------------------------------------------ the calls
def _rows(x):
    """Address and strides of a [tokens, heads, dim] tensor."""
    return x.data_ptr(), x.stride(0), x.stride(1)


def _cache(x):
    """Address and strides of a [pages, page, heads, dim] cache."""
    return x.data_ptr(), x.stride(0), x.stride(1), x.stride(2)


def _run_own(st):
    b, c = _own(), st.case
    stream = torch.cuda.current_stream().cuda_stream
    status = st.status.data_ptr()
    if st.op == "tables":
        b.sod2_page_tables(st.n, st.cap, st.page, st.past.data_ptr(), st.new.data_ptr(), st.free.data_ptr(), st.free.numel(), st.head.data_ptr(),
                           st.table.data_ptr(), st.width, st.width, st.cu.data_ptr(), st.ctx.data_ptr(), st.slots.data_ptr(),
                           st.positions.data_ptr(), st.new_head.data_ptr(), status, stream)
        return {"table": st.table, "cu": st.cu, "ctx": st.ctx, "slots": st.slots, "positions": st.positions, "head": st.new_head}
    if st.op == "rope":
        cached = st.kc is not None
        b.sod2_rope_store(st.code, st.t, c["heads"], c["kv"], c["dim"], st.rotation, st.positions.data_ptr(), st.positions.stride(0), _rows(st.q),
                          _rows(st.q_out), _rows(st.k), None if cached else _rows(st.k_out), _rows(st.v) if cached else None,
                          _cache(st.kc) if cached else None, _cache(st.vc) if cached else None, st.n_pages if cached else 0, c["page"],
                          st.slots.data_ptr() if cached else 0, status, stream)
        return {"q": st.q_out, "k_cache": st.kc, "v_cache": st.vc} if cached else {"q": st.q_out, "k": st.k_out}
    scale = 1 / math.sqrt(c["dim"])
    if st.op == "prompt":
        b.sod2_attention_prompt(st.code, st.n, st.t, c["heads"], c["kv"], c["dim"], _rows(st.q), _rows(st.k), _rows(st.v), _rows(st.out),
                                st.cu.data_ptr(), scale, st.ws.data_ptr(), st.ws.numel(), status, stream)
        return st.out
    b.sod2_attention_paged(st.code, st.n, st.t, st.most_new, c["heads"], c["kv"], c["dim"], _rows(st.q), _rows(st.out), st.cu.data_ptr(),
                           st.ctx.data_ptr(), _cache(st.kc), _cache(st.vc), st.n_pages, c["page"], st.table.data_ptr(), st.width, st.width,
                           scale, st.ws.data_ptr(), st.ws.numel(), status, stream)
    return st.out


# ------------------------------------------------------------------------------------------------ the plain forms
def _plain_tables(st):
    page, past, new = st.page, st.past.long(), st.new.long()
    have, want = (past + page - 1) // page, (past + new + page - 1) // page
    need = want - have
    first = torch.cumsum(need, 0) - need + st.head.long()
    col = torch.arange(st.width, device="cuda")
    fresh = (col >= have[:, None]) & (col < want[:, None])
    pick = (first[:, None] + col - have[:, None]).clamp(0, st.free.numel() - 1)
    table = torch.where(fresh, st.free[pick], st.table0)
    cu = torch.zeros(st.n + 1, dtype=torch.int64, device="cuda")
    cu[1:] = torch.cumsum(new, 0)
    t = torch.arange(st.cap, device="cuda")
    r = torch.searchsorted(cu[1:], t, right=True)
    live = r < st.n
    r = r.clamp(max=st.n - 1)
    pos = past[r] + t - cu[r]
    pos = torch.where(live, pos, torch.zeros_like(pos))
    slots = torch.where(live, table[r, pos // page].long() * page + pos % page, torch.full_like(pos, -1))
    return {"table": table, "cu": cu.int(), "ctx": (past + new).int(), "slots": slots,
            "positions": torch.where(live, pos, torch.full_like(pos, -1)).int(), "head": (st.head + need.sum()).int()}


def _plain_turn(x, cos, sin, rot, pairs):
    x = x.float()
    if pairs:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
    ra, rb = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([ra, rb], -1).flatten(-2) if pairs else torch.cat([ra, rb], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_rope(st):
    c = st.case
    freq = torch.tensor(st.freq, dtype=torch.float64, device="cuda")
    axis = torch.tensor(st.axis, device="cuda")
    angle = st.positions[axis].t().double() * freq                # far positions: 32 bits would lose the angle
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    dt = st.q.dtype
    q = _plain_turn(st.q, cos, sin, c["rot"], c["pairs"]).to(dt)
    k = _plain_turn(st.k, cos, sin, c["rot"], c["pairs"]).to(dt)
    if st.kc is None:
        return {"q": q, "k": k}
    live = (st.slots >= 0).nonzero()[:, 0]
    st.kc.view(-1, c["kv"], c["dim"])[st.slots[live]] = k[live]
    st.vc.view(-1, c["kv"], c["dim"])[st.slots[live]] = st.v[live]
    return {"q": q, "k_cache": st.kc, "v_cache": st.vc}


def _plain_attention(q, k, v, first, scale):
    """Queries [n, heads, dim] at positions first.. over keys and values [m, kv, dim], in blocks of queries."""
    n, h, d = q.shape
    kv = k.shape[1]
    k, v = k.float().permute(1, 2, 0), v.float().permute(1, 0, 2)
    out = torch.empty((n, h, d), dtype=q.dtype, device=q.device)
    step = max(1, min(1024, (1 << 28) // max(1, h * k.shape[2])))
    for i in range(0, n, step):
        m = min(n, i + step)
        seen = first + m
        s = torch.matmul(q[i:m].float().view(m - i, kv, h // kv, d).permute(1, 2, 0, 3).reshape(kv, -1, d), k[:, :, :seen]) * scale
        s = s.view(kv, h // kv, m - i, seen)
        late = torch.arange(seen, device=q.device) > first + torch.arange(i, m, device=q.device)[:, None]
        s = s.masked_fill(late, float("-inf"))
        p = torch.exp(s - s.amax(-1, keepdim=True))
        p = p / p.sum(-1, keepdim=True)
        o = torch.matmul(p.view(kv, -1, seen), v[:, :seen]).view(kv, h // kv, m - i, d)
        out[i:m] = o.permute(2, 0, 1, 3).reshape(m - i, h, d).to(q.dtype)
    return out


def _plain_prompt(st):
    out, scale = torch.zeros_like(st.out), 1 / math.sqrt(st.case["dim"])
    for a, b in zip(st.cu_host, st.cu_host[1:]):
        if b > a:
            out[a:b] = _plain_attention(st.q[a:b], st.k[a:b], st.v[a:b], 0, scale)
    return out


def _plain_paged(st):
    c, out, scale = st.case, torch.zeros_like(st.out), 1 / math.sqrt(st.case["dim"])
    for r, (n, m) in enumerate(zip(st.new_host, st.ctx_host)):
        if n:
            ids = st.table[r, :_pages(m, c["page"])].long()
            k, v = (x[ids].flatten(0, 1)[:m] for x in (st.kc, st.vc))
            a = st.cu_host[r]
            out[a:a + n] = _plain_attention(st.q[a:a + n], k, v, m - n, scale)
    return out


def run(state):
    if own:
        return _run_own(state)
    return {"tables": _plain_tables, "rope": _plain_rope, "prompt": _plain_prompt, "paged": _plain_paged}[state.op](state)


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _exact_tables(case, st):
    past, new, page = _ints(case["past"]), _ints(case["new"]), case["page"]
    table, free = st.table0.cpu().numpy().copy(), st.free.cpu().numpy()
    head = int(st.head)
    cu, slots, positions = [0], [], []
    for r, (p, n) in enumerate(zip(past, new)):
        owned = -(-p // page)
        while owned * page < p + n:
            table[r, owned] = free[head]
            head, owned = head + 1, owned + 1
        at = np.arange(p, p + n)
        positions.append(at)
        slots.append(table[r].astype(np.int64)[at // page] * page + at % page)
        cu.append(cu[-1] + n)
    rest = [np.full(st.cap - cu[-1], -1)]
    return {"table": torch.from_numpy(table), "cu": torch.tensor(cu, dtype=torch.int32),
            "ctx": torch.tensor([p + n for p, n in zip(past, new)], dtype=torch.int32),
            "slots": torch.from_numpy(np.concatenate(slots + rest).astype(np.int64)),
            "positions": torch.from_numpy(np.concatenate(positions + rest).astype(np.int32)), "head": torch.tensor([head], dtype=torch.int32)}


def _exact_rope(case, st):
    freq, axis = _frequencies(case)
    rot, d = case["rot"], case["dim"]
    # the rotation as a complex factor of each pair (first, second)
    first = torch.arange(0, rot, 2) if case["pairs"] else torch.arange(rot // 2)
    second = first + (1 if case["pairs"] else rot // 2)
    angle = torch.stack([st.positions[a].double() * f for f, a in zip(freq, axis)], 1)
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]

    def turned(x):
        x = x.double().clone()
        z = torch.complex(x[..., first], x[..., second]) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return x

    q, k = turned(st.q), turned(st.k)
    if not case["page"]:
        return {"q": q, "k": k}
    kc, vc = (torch.zeros(st.kc.shape, dtype=torch.float64, device="cuda").view(-1, case["kv"], d) for _ in range(2))
    n = case["tokens"]
    kc.index_copy_(0, st.slots[:n], k[:n])
    vc.index_copy_(0, st.slots[:n], st.v[:n].double())
    return {"q": q, "k_cache": kc.view(st.kc.shape), "v_cache": vc.view(st.vc.shape)}


def _exact_head(q, k, v, first, scale):
    """One head: queries [n, d] at positions first.. over keys and values [m, d]."""
    out = torch.empty_like(q)
    for i in range(0, q.shape[0], 2048):
        x = q[i:i + 2048] @ k.t() * scale
        at = first + i + torch.arange(x.shape[0], device=q.device)
        x[torch.arange(k.shape[0], device=q.device)[None] > at[:, None]] = -math.inf
        out[i:i + 2048] = torch.softmax(x, -1) @ v
    return out


def _exact_prompt(case, st):
    out = torch.zeros(st.out.shape, dtype=torch.float64, device="cuda")
    g = case["heads"] // case["kv"]
    for a, b in zip(st.cu_host, st.cu_host[1:]):
        for h in range(case["heads"] if b > a else 0):
            out[a:b, h] = _exact_head(st.q[a:b, h].double(), st.k[a:b, h // g].double(), st.v[a:b, h // g].double(), 0, 1 / math.sqrt(case["dim"]))
    return out


def _exact_paged(case, st):
    out = torch.zeros(st.out.shape, dtype=torch.float64, device="cuda")
    g, page = case["heads"] // case["kv"], case["page"]
    for r, (n, m) in enumerate(zip(st.new_host, st.ctx_host)):
        at = torch.arange(m, device="cuda")
        rows, within = st.table[r].long()[at // page], at % page
        a = st.cu_host[r]
        for h in range(case["heads"] if n else 0):
            k, v = st.kc[rows, within, h // g].double(), st.vc[rows, within, h // g].double()
            out[a:a + n, h] = _exact_head(st.q[a:a + n, h].double(), k, v, m - n, 1 / math.sqrt(case["dim"]))
    return out


def exact(case, seed):
    if work(case)["flops"] > 4e12:                                # minutes in 64 bits
        return None
    st = _inputs(case, seed)
    return {"tables": _exact_tables, "rope": _exact_rope, "prompt": _exact_prompt, "paged": _exact_paged}[case["op"]](case, st)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    if case["op"] == "tables":
        past, new, page = _ints(case["past"]), _ints(case["new"]), case["page"]
        n, t = len(past), sum(new)
        fresh = sum(_pages(p + v, page) - _pages(p, page) for p, v in zip(past, new))
        # lengths in, cumulative lengths and contexts out; a page id in and out per new page; slot and position per row
        return {"bytes": 16.0 * n + 8.0 * fresh + 12.0 * (t + case["pad"]), "flops": 0}
    esz = 4 if case["dtype"] == "f32" else 2
    h, kv, d = case["heads"], case["kv"], case["dim"]
    if case["op"] == "rope":
        t = case["tokens"] + case["pad"]
        rows = t * (2 * h + kv * (4 if case["page"] else 2))
        return {"bytes": float(esz * rows * d + t * (4 * len(_ints(case["axes"])) + (8 if case["page"] else 0))), "flops": 3.0 * t * (h + kv) * case["rot"]}
    if case["op"] == "prompt":
        lens = _ints(case["lens"])
        return {"bytes": float(esz * sum(lens) * (2 * h + 2 * kv) * d), "flops": 4.0 * h * d * sum(n * (n + 1) / 2 for n in lens)}
    past, new = _ints(case["past"]), _ints(case["new"])
    keys = sum(p + v for p, v in zip(past, new) if v)
    return {"bytes": float(esz * d * (2 * keys * kv + 2 * sum(new) * h)), "flops": 4.0 * h * d * sum(v * p + v * (v + 1) / 2 for p, v in zip(past, new))}
