"""The serving operators on the GPU against their plain 64-bit forms: page tables, rotary positions with the store into the
cache, causal attention over packed prompts and over the paged cache, and a run of them together."""
import math
import random

import pytest
import torch

from paper_2403_00176_b200 import binding as B
from tests import serving_ref as R
from tests.serving_ref import DT, cumulative, ints

pytestmark = pytest.mark.gpu

NAN = float("nan")


def close(got, want, tol):
    got = got.double()
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), float((got - want).abs().max()), float(((got - want).abs() / tol).max()), bad.nonzero()[:4].tolist())


def randn(*shape, seed=0, dtype="bf16", scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(DT[dtype][1])


# ------------------------------------------------------------------------------------------------ page tables
def run_tables(past, new, page, free, head, width, cap, seed=0, stride_extra=0, n_free=None, positions=True, with_head=True):
    rng = random.Random(seed)
    table = [[rng.randrange(1 << 20) if j * page < p else -7 for j in range(width)] for p in past]
    dev = torch.full((max(len(past), 1), width + stride_extra), -9, dtype=torch.int32, device="cuda")
    if past:
        dev[:, :width] = ints(table)
    cu, ctx = ints([-5] * (len(past) + 2)), ints([-5] * (len(past) + 1))
    slots, pos = ints([-5] * (cap + 1), torch.int64), ints([-5] * (cap + 1))
    head_out, status = ints([-5, -5]), ints([0])
    fr, pa, ne, he = ints(free if free else [0]), ints(past or [0]), ints(new or [0]), ints([head])
    B.sod2_page_tables(len(past), cap, page, pa.data_ptr(), ne.data_ptr(), fr.data_ptr(), len(free) if n_free is None else n_free,
                       he.data_ptr() if with_head else None, dev.data_ptr(), width + stride_extra, width, cu.data_ptr(), ctx.data_ptr(),
                       slots.data_ptr(), pos.data_ptr() if positions else None, head_out.data_ptr(), status.data_ptr(), R.stream())
    torch.cuda.synchronize()
    want = R.tables(past, new, page, free, head if with_head else 0, table, cap)
    assert dev[:len(past), :width].tolist() == want[0]
    assert (dev[:, width:] == -9).all()
    assert cu.tolist() == want[1] + [-5] and ctx.tolist() == want[2] + [-5]
    assert slots.tolist() == want[3] + [-5]
    assert pos.tolist() == (want[4] + [-5] if positions else [-5] * (cap + 1))
    assert head_out.tolist() == [want[5], -5]
    return int(status)


@pytest.mark.parametrize("n,page,most,pad,seed", [(1, 16, 1, 0, 0), (1, 1, 40, 3, 1), (7, 16, 40, 5, 2), (33, 7, 300, 0, 3), (48, 16, 1, 16, 4),
                                                  (1023, 32, 3, 1, 5), (1024, 8, 2, 0, 6), (1025, 8, 2, 9, 7), (2500, 16, 9, 700, 8), (3, 128, 5000, 0, 9)])
def test_page_tables(n, page, most, pad, seed):
    rng = random.Random(seed)
    past = [rng.choice([0, rng.randint(0, 3 * page), rng.randint(0, 900)]) for _ in range(n)]
    new = [rng.choice([0, 1, rng.randint(0, most)]) for _ in range(n)]
    width = max(-(-(p + v) // page) for p, v in zip(past, new)) + rng.randint(0, 2)
    free = [rng.randrange(1 << 22) for _ in range(sum(-(-(p + v) // page) + (-p // page) for p, v in zip(past, new)) + 5)]
    assert run_tables(past, new, page, free, 3, max(width, 1), sum(new) + pad, seed, stride_extra=seed % 3) == 0


def test_page_tables_without_requests_tokens_positions_or_head():
    assert run_tables([], [], 16, [1, 2], 1, 1, 5) == 0
    assert run_tables([5, 0], [0, 0], 16, [], 0, 1, 0) == 0
    assert run_tables([5, 0], [30, 1], 16, list(range(9)), 0, 4, 40, positions=False, with_head=False) == 0


def test_page_tables_report_what_runs_out():
    assert run_tables([0, 3], [40, 20], 16, [4, 5, 6], 1, 4, 60) == 4                      # free list
    assert run_tables([0, 3], [40, 20], 16, list(range(20)), 0, 2, 60) == 4                # width of the table
    assert run_tables([-2, 3], [4, -9], 16, list(range(20)), 0, 2, 60) == 8                # negative lengths count as zero
    assert run_tables([1, 3, 0], [40, 20, 7], 16, list(range(20)), 0, 4, 50) == 8          # more rows than max_tokens
    assert run_tables([1], [40], 16, list(range(20)), 18, 4, 50) == 0                      # the last two of the list: pages 1 and 2 of tokens 1..40
    assert run_tables([1], [40], 16, list(range(20)), 19, 4, 50) == 4                      # one of them


# ------------------------------------------------------------------------------------------------ rotary positions
def cache_of(layout, n_pages, page, kv, dim, dtype, fill):
    shape = (n_pages, page, kv, dim) if layout == "page, token, head" else (n_pages, kv, page, dim)
    c = torch.full(shape, fill, dtype=DT[dtype][1], device="cuda")
    return c if layout == "page, token, head" else c.transpose(1, 2)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,H,kv,dim,sections,local,adjacent,packed", [
    (1, 1, 1, 64, (32,), False, False, False), (5, 4, 2, 128, (64,), False, True, True), (37, 6, 2, 80, (8, 16, 16), True, False, True),
    (300, 12, 4, 96, (24,), False, True, False), (64, 32, 8, 128, (16, 24, 24), False, False, True), (1000, 3, 3, 64, (4, 12, 16), True, True, False),
    (11, 2, 1, 70, (35,), False, False, False), (9, 5, 1, 6, (1, 1, 1), False, True, True), (3, 2, 2, 256, (128,), False, False, False),
    (17, 1, 1, 66, (5,), False, False, True), (2, 64, 64, 32, (16,), False, False, False)])
def test_rope(dtype, T, H, kv, dim, sections, local, adjacent, packed):
    rot = B.Rotation.sections(sections, 10000.0, local, adjacent)
    x = randn(T, H + 2 * kv, dim, seed=T, dtype=dtype)
    q, k = x[:, :H], x[:, H:H + kv]
    if not packed:
        q, k = q.contiguous(), k.contiguous()
    pos = torch.randint(-3, 1 << 20, (len(sections), T), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(1))
    pos[:, 0] = 2 ** 31 - 1
    guard = 5
    qo, ko = (torch.full((T + guard, h, dim), 9.0, dtype=x.dtype, device="cuda") for h in (H, kv))
    B.sod2_rope_store(DT[dtype][0], T, H, kv, dim, rot, pos.data_ptr(), pos.stride(0), R.rows(q), R.rows(qo), R.rows(k), R.rows(ko), None, None, None, 0, 0,
                      None, None, R.stream())
    for src, dst in ((q, qo), (k, ko)):
        want, size = R.turn(src, pos, list(rot._freq), list(rot._axis), adjacent)
        close(dst[:T], want, R.turn_tolerance(dtype, want, size))
        assert (dst[T:] == 9).all()
        assert torch.equal(dst[:T, :, 2 * rot.n_pairs:], src[..., 2 * rot.n_pairs:])
    # in place
    qi, ki = q.clone(), k.clone()
    B.sod2_rope_store(DT[dtype][0], T, H, kv, dim, rot, pos.data_ptr(), pos.stride(0), R.rows(qi), R.rows(qi), R.rows(ki), R.rows(ki), None, None, None, 0, 0,
                      None, None, R.stream())
    assert torch.equal(qi, qo[:T]) and torch.equal(ki, ko[:T])
    # queries alone, keys alone
    q1, k1 = torch.zeros_like(qi), torch.zeros_like(ki)
    B.sod2_rope_store(DT[dtype][0], T, H, 0, dim, rot, pos.data_ptr(), pos.stride(0), R.rows(q), R.rows(q1), None, None, None, None, None, 0, 0, None, None, R.stream())
    B.sod2_rope_store(DT[dtype][0], T, 0, kv, dim, rot, pos.data_ptr(), pos.stride(0), None, None, R.rows(k), R.rows(k1), None, None, None, 0, 0, None, None, R.stream())
    assert torch.equal(q1, qi) and torch.equal(k1, ki)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["page, token, head", "page, head, token"])
@pytest.mark.parametrize("T,H,kv,dim,page", [(1, 4, 2, 64, 16), (50, 8, 2, 128, 16), (200, 6, 3, 80, 24), (13, 2, 1, 70, 1), (700, 12, 12, 64, 64)])
def test_rope_stores_keys_and_values(dtype, layout, T, H, kv, dim, page):
    rot = B.Rotation.sections((dim // 2,), 500000.0)
    x = randn(T, H + 2 * kv, dim, seed=T, dtype=dtype)
    q, k, v = x[:, :H], x[:, H:H + kv], x[:, H + kv:]
    pos = ints([[7 * t for t in range(T)]])
    n_pages = -(-T // page) + 3
    kc, vc = (cache_of(layout, n_pages, page, kv, dim, dtype, f) for f in (3.0, 4.0))
    slots = torch.randperm(n_pages * page, generator=torch.Generator().manual_seed(T))[:T]
    slots[T // 2] = -1
    if T > 20:
        slots[3], slots[9], slots[11] = n_pages * page, 1 << 40, -(1 << 40)
    sl, status, qo = slots.cuda(), ints([0]), torch.zeros(T, H, dim, dtype=x.dtype, device="cuda")
    for ko in (None, torch.zeros(T, kv, dim, dtype=x.dtype, device="cuda")):
        B.sod2_rope_store(DT[dtype][0], T, H, kv, dim, rot, pos.data_ptr(), T, R.rows(q), R.rows(qo), R.rows(k), R.rows(ko), R.rows(v), R.pages(kc), R.pages(vc),
                          n_pages, page, sl.data_ptr(), status.data_ptr(), R.stream())
    want, size = R.turn(k, pos, list(rot._freq), list(rot._axis), False)
    close(ko, want, R.turn_tolerance(dtype, want, size))
    flat_k, flat_v = kc.reshape(-1, kv, dim), vc.reshape(-1, kv, dim)
    stored = torch.zeros(n_pages * page, dtype=torch.bool)
    for t, s in enumerate(slots.tolist()):
        if 0 <= s < n_pages * page:
            stored[s] = True
            assert torch.equal(flat_k[s], ko[t]) and torch.equal(flat_v[s], v[t])
    assert (flat_k[~stored.cuda()] == 3).all() and (flat_v[~stored.cuda()] == 4).all()
    assert int(status) == (2 if T > 20 else 0)
    # values alone are not a case; keys alone are
    kc2 = cache_of(layout, n_pages, page, kv, dim, dtype, 3.0)
    B.sod2_rope_store(DT[dtype][0], T, 0, kv, dim, rot, pos.data_ptr(), T, None, None, R.rows(k), None, None, R.pages(kc2), None, n_pages, page, sl.data_ptr(),
                      None, R.stream())
    assert torch.equal(kc2, kc)


# ------------------------------------------------------------------------------------------------ attention over prompts
PROMPTS = [([1], 1, 1, 64), ([37], 12, 12, 64), ([128, 129, 127], 4, 2, 64), ([5, 0, 1, 300, 0], 6, 2, 128), ([257, 64, 513], 8, 1, 128),
           ([200, 33], 15, 3, 80), ([100, 140], 14, 2, 96), ([70, 1, 90], 5, 5, 32), ([640], 2, 1, 112), ([33, 400], 3, 1, 72), ([129], 16, 1, 8),
           ([60, 300], 7, 1, 128), ([90, 40], 48, 1, 64), ([50, 31], 4, 2, 256), ([20, 45], 3, 1, 33), ([40], 200, 1, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("lens,H,kv,dim", PROMPTS)
def test_prompt_attention(dtype, lens, H, kv, dim):
    cu, T = cumulative(lens), sum(lens) + 7
    x = randn(T, H + 2 * kv, dim, seed=sum(lens) + H, dtype=dtype)
    x[:, :H] *= 2
    x[sum(lens):] = NAN                     # rows behind the last request are no one's
    q, k, v = x[:, :H], x[:, H:H + kv], x[:, H + kv:]
    if H % 2:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    out = torch.full((T, H, dim), 5.0, dtype=x.dtype, device="cuda")
    status = ints([0])
    R.prompt(dtype, q, k, v, out, ints(cu), 1 / math.sqrt(dim), status)
    for a, b in zip(cu, cu[1:]):
        want, mass = R.attend(q[a:b], k[a:b], v[a:b], b - a, 1 / math.sqrt(dim))
        close(out[a:b], want, R.attention_tolerance(dtype, want, mass))
    assert (out[sum(lens):] == 5).all() and int(status) == 0


def test_prompts_do_not_see_each_other():
    # a request of infinities and NaN between two others, and large scores
    lens, H, kv, dim = [70, 90, 200], 4, 2, 64
    cu = cumulative(lens)
    x = randn(sum(lens), H + 2 * kv, dim, dtype="bf16", scale=4.0)
    x[70:160] = float("inf")
    x[75:100] = NAN
    q, k, v = x[:, :H], x[:, H:H + kv], x[:, H + kv:]
    out = torch.zeros(sum(lens), H, dim, dtype=x.dtype, device="cuda")
    R.prompt("bf16", q, k, v, out, ints(cu), 1.0)
    for a, b in ((0, 70), (160, 360)):
        want, mass = R.attend(q[a:b], k[a:b], v[a:b], b - a, 1.0)
        close(out[a:b], want, R.attention_tolerance("bf16", want, mass))
    assert out[70:160].isnan().all()


def test_prompt_lengths_outside_the_rows_stay_inside():
    T, H, dim = 50, 2, 64
    x = randn(T, 3 * H, dim)
    q, k, v = x[:, :H], x[:, H:2 * H], x[:, 2 * H:]
    out = torch.full((T + 4, H, dim), 5.0, dtype=x.dtype, device="cuda")
    R.prompt("bf16", q, k, v, out[:T], ints([0, 20, 1000]), 0.125)          # 980 rows that are not there
    want, mass = R.attend(q[20:], k[20:], v[20:], 30, 0.125)
    close(out[20:50], want, R.attention_tolerance("bf16", want, mass))
    assert (out[T:] == 5).all()


# ------------------------------------------------------------------------------------------------ attention over the cache
def make_cache(ctx, page, kv, dim, dtype, layout="page, token, head", seed=0, extra=3, fill=NAN):
    """Random keys and values in randomly ordered pages; everything that belongs to no request is `fill`."""
    need = [-(-c // page) for c in ctx]
    n_pages = sum(need) + extra
    kc, vc = (cache_of(layout, n_pages, page, kv, dim, dtype, fill) for _ in range(2))
    ids = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
    width = max(need + [1]) + 1
    table, at = [], 0
    for c, n in zip(ctx, need):
        table.append(ids[at:at + n] + [-1] * (width - n))
        for j in range(n):
            m = min(page, c - j * page)
            kc[ids[at + j], :m] = randn(m, kv, dim, seed=seed + 2 * at + 2 * j + 1, dtype=dtype)
            vc[ids[at + j], :m] = randn(m, kv, dim, seed=seed + 2 * at + 2 * j + 2, dtype=dtype)
        at += n
    return kc, vc, table


def check_paged(dtype, new, ctx, H, kv, dim, page, layout="page, token, head", scale=None, max_new=0, fill=NAN, pad=4):
    scale = 1 / math.sqrt(dim) if scale is None else scale
    kc, vc, table = make_cache(ctx, page, kv, dim, dtype, layout, fill=fill)
    cu = cumulative(new)
    q = randn(sum(new) + pad, H, dim, seed=9, dtype=dtype, scale=2.0)
    q[sum(new):] = NAN
    out = torch.full_like(q, 5.0)
    status = ints([0])
    R.paged(dtype, q, out, ints(cu), ints(ctx), kc, vc, ints(table), scale, max_new, status)
    for r, (n, m) in enumerate(zip(new, ctx)):
        k, v = (R.gather_pages(c, table[r], m) for c in (kc, vc))
        want, mass = R.attend(q[cu[r]:cu[r + 1]], k, v, m, scale)
        close(out[cu[r]:cu[r + 1]], want, R.attention_tolerance(dtype, want, mass))
    assert (out[sum(new):] == 5).all() and int(status) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("new,ctx,H,kv,dim,page", [
    ([1], [1], 1, 1, 64, 16), ([1], [777], 12, 4, 64, 16), ([1, 1, 1], [5, 1000, 128], 8, 2, 128, 16), ([1] * 40, list(range(1, 4000, 100)), 8, 8, 64, 32),
    ([3, 1, 0, 17], [40, 300, 9, 17], 6, 2, 80, 16), ([130, 1, 64], [400, 2000, 64], 8, 1, 128, 64), ([200], [1500], 16, 2, 96, 128),
    ([2, 5], [700, 130], 15, 3, 72, 8), ([1, 9], [3000, 700], 4, 4, 112, 256), ([4, 1], [129, 257], 2, 1, 128, 48), ([1, 6], [100, 33], 4, 2, 64, 1),
    ([1, 6], [100, 133], 4, 2, 64, 24), ([1, 3], [60, 33], 2, 2, 256, 16), ([1, 20], [70, 33], 3, 1, 33, 5), ([300], [300], 7, 1, 64, 16),
    ([1, 1], [20000, 7], 8, 1, 128, 64), ([2], [900], 300, 2, 64, 16)])
def test_paged_attention(dtype, new, ctx, H, kv, dim, page):
    check_paged(dtype, new, ctx, H, kv, dim, page, max_new=max(new))


@pytest.mark.parametrize("fill", [0.0, float("inf"), float("-inf"), 60000.0])
def test_paged_attention_whatever_the_pages_hold_behind_the_last_key(fill):
    check_paged("f16", [1, 40, 1], [3, 300, 129], 8, 2, 64, 32, fill=fill)


@pytest.mark.parametrize("max_new", [0, 1, 1000])
def test_paged_attention_of_heads_before_tokens_and_any_bound(max_new):
    check_paged("bf16", [1, 19, 2], [333, 200, 2], 6, 3, 64, 16, "page, head, token", max_new=max_new)
    check_paged("bf16", [1, 1], [333, 1], 6, 3, 128, 64, "page, head, token", max_new=max_new)


def test_paged_attention_rows_without_a_key_are_zero():
    # fewer keys than new tokens: the first rows see nothing; no keys at all; a negative context
    new, H, kv, dim, page = [5, 4, 3, 150], 4, 2, 64, 16
    ctx = [2, 0, -7, 20]
    kc, vc, table = make_cache([2, 0, 0, 20], page, kv, dim, "bf16")
    cu = cumulative(new)
    q = randn(sum(new), H, dim)
    out = torch.full_like(q, 5.0)
    R.paged("bf16", q, out, ints(cu), ints(ctx), kc, vc, ints(table), 0.125)
    for r, (n, m) in enumerate(zip(new, ctx)):
        m = max(m, 0)
        want, mass = R.attend(q[cu[r]:cu[r + 1]], R.gather_pages(kc, table[r], m), R.gather_pages(vc, table[r], m), m, 0.125)
        close(out[cu[r]:cu[r + 1]], want, R.attention_tolerance("bf16", want, mass))
    assert (out[:3] == 0).all() and (out[5:12] == 0).all() and (out[12:142] == 0).all()


def test_paged_attention_does_not_follow_bad_pages():
    H, kv, dim, page = 4, 2, 64, 16
    for new in ([1, 1], [20, 3]):
        ctx = [100, 60]
        kc, vc, table = make_cache(ctx, page, kv, dim, "bf16")
        table[0][2], table[0][4], table[1][1] = kc.shape[0], -1, 2 ** 31 - 1
        cu = cumulative(new)
        q, status = randn(sum(new), H, dim), ints([0])
        out = torch.full_like(q, 5.0)
        R.paged("bf16", q, out, ints(cu), ints(ctx), kc, vc, ints(table), 0.125, status=status)
        for r, m in enumerate(ctx):
            want, mass = R.attend(q[cu[r]:cu[r + 1]], R.gather_pages(kc, table[r], m), R.gather_pages(vc, table[r], m), m, 0.125)
            close(out[cu[r]:cu[r + 1]], want, R.attention_tolerance("bf16", want, mass))
        assert int(status) == 2


def test_paged_attention_takes_no_key_beyond_the_table():
    H, kv, dim, page, ctx = 4, 2, 64, 16, [100]
    kc, vc, table = make_cache(ctx, page, kv, dim, "bf16")
    q = randn(1, H, dim)
    out = torch.full_like(q, 5.0)
    R.paged("bf16", q, out, ints([0, 1]), ints([10 ** 9]), kc, vc, ints(table), 0.125, width=5)          # 80 keys
    want, mass = R.attend(q, R.gather_pages(kc, table[0], 80), R.gather_pages(vc, table[0], 80), 80, 0.125)
    close(out, want, R.attention_tolerance("bf16", want, mass))


def test_paged_attention_behind_four_billion_elements():
    # the last pages of a cache of more than 2^32 elements: offsets in 64 bits
    H, kv, dim, page = 4, 2, 128, 64
    n_pages = (1 << 32) // (page * kv * dim) + 40
    kc, vc = (torch.empty(n_pages, page, kv, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ids = [n_pages - 1, n_pages - 30, 0, n_pages - 17]
    for c, s in ((kc, 1), (vc, 2)):
        for i, p in enumerate(ids):
            c[p] = randn(page, kv, dim, seed=10 * s + i)
    for new in (1, 30):
        q = randn(new, H, dim)
        out = torch.zeros_like(q)
        R.paged("bf16", q, out, ints([0, new]), ints([250]), kc, vc, ints([ids]), 0.1, new)
        want, mass = R.attend(q, torch.cat([kc[p] for p in ids]), torch.cat([vc[p] for p in ids]), 250, 0.1)
        close(out, want, R.attention_tolerance("bf16", want, mass))


# ------------------------------------------------------------------------------------------------ both forms of the attention, further
def prompt_case(dtype, lens, H, kv, dim, seed=0, scale=None, change=None, packed=True):
    scale = 1 / math.sqrt(dim) if scale is None else scale
    cu, T = cumulative(lens), sum(lens)
    x = randn(T, H + 2 * kv, dim, seed=seed, dtype=dtype)
    x[:, :H] *= 2
    if change:
        change(x, cu)
    q, k, v = x[:, :H], x[:, H:H + kv], x[:, H + kv:]
    if not packed:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    out, status = torch.full((T, H, dim), 5.0, dtype=x.dtype, device="cuda"), ints([0])
    R.prompt(dtype, q, k, v, out, ints(cu), scale, status)
    assert int(status) == 0
    return cu, q, k, v, out, scale


def check_prompt(dtype, lens, *args, **kw):
    cu, q, k, v, out, scale = prompt_case(dtype, lens, *args, **kw)
    for a, b in zip(cu, cu[1:]):
        want, mass = R.attend(q[a:b], k[a:b], v[a:b], b - a, scale)
        close(out[a:b], want, R.attention_tolerance(dtype, want, mass))


def test_more_requests_than_a_cta_has_threads():
    rng = random.Random(5)
    check_prompt("bf16", [rng.randint(0, 5) for _ in range(900)], 4, 2, 64)
    check_prompt("bf16", [rng.randint(0, 3) for _ in range(400)] + [1500] + [2] * 300, 4, 2, 128)
    check_paged("f16", [1] * 700, [rng.randint(1, 90) for _ in range(700)], 4, 2, 64, 16, max_new=1)
    check_paged("bf16", [rng.choice([0, 1, 1, 30]) for _ in range(450)], [rng.randint(30, 60) for _ in range(450)], 4, 2, 128, 32)


@pytest.mark.parametrize("seed", range(24))
def test_attention_of_random_shapes(seed):
    rng = random.Random(100 + seed)
    dtype, kv = rng.choice(["bf16", "f16"]), rng.choice([1, 2, 3])
    H, dim = kv * rng.choice([1, 2, 3, 4, 7, 8, 16, 32]), rng.choice([8, 24, 40, 64, 72, 80, 96, 104, 128])
    n = rng.randint(1, 6)
    most = rng.choice([5, 60, 700])
    lens = [rng.choice([0, 1, rng.randint(1, most), most]) for _ in range(n)] + [1]
    check_prompt(dtype, lens, H, kv, dim, seed, packed=rng.random() < 0.5)
    past = [rng.choice([0, rng.randint(0, 100), rng.randint(0, 3000)]) for _ in lens]
    check_paged(dtype, lens, [p + v for p, v in zip(past, lens)], H, kv, dim, rng.choice([8, 16, 40, 64, 128, 384]),
                rng.choice(["page, token, head", "page, head, token"]), max_new=rng.choice([0, most]))


def test_one_token_alone():
    check_prompt("bf16", [1], 4, 2, 64)
    check_paged("bf16", [1], [1], 32, 1, 64, 16, pad=0)
    check_paged("bf16", [1], [900], 20, 1, 128, 16, pad=0)             # more heads a key head than rows of the few-row form


def test_references_that_rise_with_every_block():
    # keys that grow: the largest score is always in the last block, by far more than the reference may lag behind
    def grow(x, cu):
        T = x.shape[0]
        x[:, 4:6] = x[:, :1] * torch.linspace(0.05, 6, T, device="cuda")[:, None, None].to(x.dtype)
    for dim in (64, 128):
        check_prompt("bf16", [1100], 4, 2, dim, change=grow, scale=0.02)
    q_dir = randn(1, 4, 128, seed=3)
    for new in (1, 40):
        ctx, page = 1500, 16
        kc, vc, table = make_cache([ctx], page, 2, 128, "f16")
        ramp = torch.linspace(0, 4, ctx, device="cuda")
        for j, p in enumerate(table[0][:-(-ctx // page)]):
            m = min(page, ctx - j * page)
            kc[p, :m] = (q_dir[0, ::2][None] * ramp[j * page:j * page + m, None, None]).to(kc.dtype)
        q, out = q_dir.to(kc.dtype).expand(new, 4, 128).contiguous(), torch.zeros(new, 4, 128, dtype=kc.dtype, device="cuda")
        R.paged("f16", q, out, ints([0, new]), ints([ctx]), kc, vc, ints(table), 0.3, new)
        want, mass = R.attend(q, R.gather_pages(kc, table[0], ctx), R.gather_pages(vc, table[0], ctx), ctx, 0.3)
        close(out, want, R.attention_tolerance("f16", want, mass))


@pytest.mark.parametrize("bad", [NAN, float("inf"), float("-inf")])
def test_later_tokens_that_are_not_finite_do_not_reach_earlier_rows(bad):
    # keys and values from a token on; whole items, cut ones, both forms
    at = 700
    for dim in (64, 128):
        def spoil(x, cu):
            x[at:, 4:] = bad
        cu, q, k, v, out, scale = prompt_case("bf16", [1200], 4, 2, dim, change=spoil)
        want, mass = R.attend(q[:at], k[:at], v[:at], at, scale)
        close(out[:at], want, R.attention_tolerance("bf16", want, mass))
        assert not out[at:].isfinite().all(-1).any()
    H, kv, dim, page, new, ctx = 4, 2, 128, 16, 6, 3000
    for n in (new, 60):
        kc, vc, table = make_cache([ctx], page, kv, dim, "bf16")
        first = ctx - n + n // 2                                       # the first token that is not finite
        for t in range(first, ctx):
            kc[table[0][t // page], t % page] = bad
            vc[table[0][t // page], t % page] = bad
        q = randn(n, H, dim)
        out = torch.full_like(q, 5.0)
        R.paged("bf16", q, out, ints([0, n]), ints([ctx]), kc, vc, ints(table), 0.1)
        good = n // 2
        want, mass = R.attend(q[:good], R.gather_pages(kc, table[0], ctx - n + good), R.gather_pages(vc, table[0], ctx - n + good), ctx - n + good, 0.1)
        close(out[:good], want, R.attention_tolerance("bf16", want, mass))
        assert not out[good:].isfinite().all(-1).any()


@pytest.mark.parametrize("ctx", [1, 17, 1040, 5000])
@pytest.mark.parametrize("dim", [64, 128])
def test_a_visible_key_that_is_not_a_number_makes_the_row_so(ctx, dim):
    kc, vc, table = make_cache([ctx, ctx], 16, 1, dim, "bf16", fill=0.0)
    kc[table[1][(ctx - 1) // 16], (ctx - 1) % 16] = NAN         # the last key of the second request, alone among its warp's 16 for most ctx
    q, out = randn(2, 2, dim, seed=3), torch.zeros(2, 2, dim, dtype=torch.bfloat16, device="cuda")
    for max_new in (1, 0):
        R.paged("bf16", q, out, ints([0, 1, 2]), ints([ctx, ctx]), kc, vc, ints(table), dim ** -0.5, max_new=max_new)
        assert out[0].isfinite().all() and out[1].isnan().all()


@pytest.mark.parametrize("heads", range(1, 17))
def test_keys_that_are_not_numbers_in_every_part_of_a_cut_row(heads):
    # the last 256 keys: the diagonal ones lie in a block of which the row sees nothing else, for some numbers of heads in a part of its own
    q, k, v = (randn(2048, heads, 64, seed=s) for s in range(3))
    k[1792:] = NAN
    out = torch.zeros_like(q)
    R.prompt("bf16", q, k, v, out, ints([0, 2048]), 0.125)
    assert out[:1792].isfinite().all() and out[1792:].isnan().all()


def test_keys_that_all_heads_share():
    # a broadcast key head: strides of zero, which no tensor map has
    T, H, dim = 150, 4, 64
    q, k1, v1 = randn(T, H, dim), randn(T, 1, dim, seed=1), randn(T, 1, dim, seed=2)
    k, v = k1.expand(T, 2, dim), v1.expand(T, 2, dim)
    out = torch.zeros_like(q)
    R.prompt("bf16", q, k, v, out, ints([0, T]), 0.125)
    want, mass = R.attend(q, k, v, T, 0.125)
    close(out, want, R.attention_tolerance("bf16", want, mass))


def test_two_captured_graphs_share_a_workspace():
    H, kv, dim, page = 8, 2, 128, 16
    ws, cases, graphs = R.Workspace(H, kv, dim), [], []
    for new, ctx in (([1, 1], [2500, 900]), ([90, 300], [2000, 300])):
        kc, vc, table = make_cache(ctx, page, kv, dim, "bf16", seed=sum(new))
        q, cu, c, t = randn(sum(new), H, dim, seed=sum(ctx)), ints(cumulative(new)), ints(ctx), ints(table)
        out = torch.zeros_like(q)
        args = ("bf16", q, out, cu, c, kc, vc, t, 0.1, max(new), None, ws)
        R.paged(*args)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            R.paged(*args)
        cases.append((args, out.clone(), table))
        graphs.append(g)
    for _ in range(3):
        for g, (args, first, table) in zip(graphs, cases):
            args[2].fill_(7)
            g.replay()
            assert torch.equal(args[2], first)
    # lengths are read when the graph runs
    args, _, table = cases[0]
    args[4].copy_(ints([700, 33]))
    graphs[0].replay()
    for r, m in enumerate((700, 33)):
        want, mass = R.attend(args[1][r:r + 1], R.gather_pages(args[5], table[r], m), R.gather_pages(args[6], table[r], m), m, 0.1)
        close(args[2][r:r + 1], want, R.attention_tolerance("bf16", want, mass))


# ------------------------------------------------------------------------------------------------ together
def serve(dtype, prompts, steps, H, kv, dim, page, qkv, captured=False):
    """Prompts in chunks, then single tokens, through all operators; per request the outputs of all its tokens.  qkv(r, a, b): the
    projections of tokens a..b of request r, before the rotation."""
    n, rot = len(prompts), B.Rotation.sections((dim // 2,), 10000.0)
    total = [p + steps for p in prompts]
    width = max(-(-t // page) for t in total)
    n_pages = sum(-(-t // page) for t in total) + 2
    kc, vc = (torch.full((n_pages, page, kv, dim), NAN, dtype=DT[dtype][1], device="cuda") for _ in range(2))
    free = torch.randperm(n_pages, generator=torch.Generator().manual_seed(3)).int().cuda()
    table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    heads = [ints([0]), ints([0])]
    status, ws, outs, past = ints([0]), R.Workspace(H, kv, dim), [[] for _ in range(n)], [0] * n
    cap = sum(prompts) + 3
    buf = dict(past=ints(past), new=ints([0] * n), cu=ints([0] * (n + 1)), ctx=ints([0] * n), slots=ints([0] * cap, torch.int64), pos=ints([0] * cap),
               x=torch.zeros(cap, H + 2 * kv, dim, dtype=DT[dtype][1], device="cuda"), q=torch.zeros(cap, H, dim, dtype=DT[dtype][1], device="cuda"),
               out=torch.zeros(cap, H, dim, dtype=DT[dtype][1], device="cuda"))

    def step(rows, most):
        b = buf
        B.sod2_page_tables(n, rows, page, b["past"].data_ptr(), b["new"].data_ptr(), free.data_ptr(), n_pages, heads[0].data_ptr(), table.data_ptr(),
                           width, width, b["cu"].data_ptr(), b["ctx"].data_ptr(), b["slots"].data_ptr(), b["pos"].data_ptr(), heads[1].data_ptr(),
                           status.data_ptr(), R.stream())
        q, k, v = b["x"][:rows, :H], b["x"][:rows, H:H + kv], b["x"][:rows, H + kv:]
        B.sod2_rope_store(DT[dtype][0], rows, H, kv, dim, rot, b["pos"].data_ptr(), rows, R.rows(q), R.rows(b["q"]), R.rows(k), None, R.rows(v),
                          R.pages(kc), R.pages(vc), n_pages, page, b["slots"].data_ptr(), status.data_ptr(), R.stream())
        R.paged(dtype, b["q"][:rows], b["out"][:rows], b["cu"], b["ctx"], kc, vc, table, 1 / math.sqrt(dim), most, status, ws)
        heads[0].copy_(heads[1])

    graph = None
    plan = [[(p + 1) // 2 for p in prompts], [p - (p + 1) // 2 for p in prompts]] + [[1] * n] * steps
    for i, new in enumerate(plan):
        rows = sum(new) + 3 if i < 2 else n + 3          # padding rows, as of a batch of fixed size
        at = 0
        for r, m in enumerate(new):
            buf["x"][at:at + m] = qkv(r, past[r], past[r] + m)
            at += m
        buf["x"][at:rows] = NAN
        buf["past"].copy_(ints(past))
        buf["new"].copy_(ints(new))
        if captured and i >= 2:
            if graph is None:
                kept = [t.clone() for t in (heads[0], table, kc, vc)]
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    step(rows, 1)
                assert torch.equal(kept[1], table)
            graph.replay()
        else:
            step(rows, max(new))
        for r, a in enumerate(cumulative(new)[:-1]):
            outs[r].append(buf["out"][a:a + new[r]].clone())
        past = [p + m for p, m in zip(past, new)]
    assert int(status) == 0
    return [torch.cat(o) for o in outs]


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("dtype,prompts,H,kv,dim,page", [("bf16", [37, 1, 200], 8, 2, 64, 16), ("f16", [130, 64], 6, 3, 128, 32), ("bf16", [20, 9], 3, 1, 72, 24)])
def test_serving_loop(dtype, prompts, H, kv, dim, page, captured):
    # prompts in two chunks and five single tokens, against causal attention over the whole sequences
    steps = 5
    x = [randn(p + steps, H + 2 * kv, dim, seed=r, dtype=dtype) for r, p in enumerate(prompts)]
    outs = serve(dtype, prompts, steps, H, kv, dim, page, lambda r, a, b: x[r][a:b], captured)
    rot = B.Rotation.sections((dim // 2,), 10000.0)
    for r, p in enumerate(prompts):
        T = p + steps
        pos = ints([list(range(T))])
        qk = x[r][:, :H + kv].clone()
        B.sod2_rope_store(DT[dtype][0], T, H + kv, 0, dim, rot, pos.data_ptr(), T, R.rows(qk), R.rows(qk), None, None, None, None, None, 0, 0, None, None, R.stream())
        want, mass = R.attend(qk[:, :H], qk[:, H:], x[r][:, H + kv:], T, 1 / math.sqrt(dim))
        close(outs[r], want, R.attention_tolerance(dtype, want, mass))
        # the prompt call over the whole sequence agrees too
        out = torch.zeros(T, H, dim, dtype=DT[dtype][1], device="cuda")
        R.prompt(dtype, qk[:, :H], qk[:, H:], x[r][:, H + kv:], out, ints([0, T]), 1 / math.sqrt(dim))
        close(out, want, R.attention_tolerance(dtype, want, mass))


def test_calls_on_another_stream_and_again():
    # a stream of its own, and the same call twice: the same bits
    lens, H, kv, dim = [300, 77], 8, 2, 128
    x = randn(sum(lens), H + 2 * kv, dim)
    q, k, v = x[:, :H], x[:, H:H + kv], x[:, H + kv:]
    cu, outs, ws = ints(cumulative(lens)), [], R.Workspace(H, kv, dim)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(2):
            out = torch.zeros(sum(lens), H, dim, dtype=x.dtype, device="cuda")
            R.prompt("bf16", q, k, v, out, cu, 0.1, ws=ws)
            outs.append(out)
    s.synchronize()
    assert torch.equal(outs[0], outs[1])
    want, mass = R.attend(q[:300], k[:300], v[:300], 300, 0.1)
    close(outs[0][:300], want, R.attention_tolerance("bf16", want, mass))
