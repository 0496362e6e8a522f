"""Plain 64-bit forms of the serving operators, and the small drivers that call them through the binding."""
from __future__ import annotations

import math

import torch

from paper_2403_00176_b200 import binding as B

DT = {"f32": (B.DTYPE_F32, torch.float32), "bf16": (B.DTYPE_BF16, torch.bfloat16), "f16": (B.DTYPE_F16, torch.float16)}


def rows(x):
    return None if x is None else (x.data_ptr(), x.stride(0), x.stride(1))


def pages(x):
    return None if x is None else (x.data_ptr(), x.stride(0), x.stride(1), x.stride(2))


def stream():
    return torch.cuda.current_stream().cuda_stream


def cumulative(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


# ------------------------------------------------------------------------------------------------ attention
def attend(q, k, v, ctx, scale):
    """q [n, H, D] over k, v [m >= ctx, HK, D]: (output, sum of p |v|) in float64; rows without a key are zero."""
    n, H, D = q.shape
    g = H // k.shape[1]
    out, mass = torch.zeros(n, H, D, dtype=torch.float64, device=q.device), torch.zeros(n, H, D, dtype=torch.float64, device=q.device)
    for i in range(n):
        seen = min(ctx, ctx - n + i + 1)
        if seen <= 0:
            continue
        kk, vv = (x[:seen].double().repeat_interleave(g, 1) for x in (k, v))
        s = torch.einsum("hd,mhd->hm", q[i].double(), kk) * scale
        p = torch.softmax(s, -1)
        out[i] = torch.einsum("hm,mhd->hd", p, vv)
        mass[i] = torch.einsum("hm,mhd->hd", p, vv.abs())
    return out, mass


def subnormal_half_step(dtype):
    f = torch.finfo(DT[dtype][1])
    return f.smallest_normal * f.eps / 2


def attention_tolerance(dtype, want, mass):
    """|error| of a correct kernel: the output is rounded once (half a step of its value); the probabilities that go into the
    product with the values are rounded once (half a step of each term: of sum p |v| together), and are themselves off by no
    more than 2^-13 (scores and exponentials in 32 bits: 2^-24 relative of a score of at most some hundreds, an exponential to 2^-14)."""
    half = torch.finfo(DT[dtype][1]).eps / 2
    return half * want.abs() + (half + 2.0 ** -13) * mass + subnormal_half_step(dtype)


class Workspace:
    def __init__(self, heads, kv, dim):
        self.t = torch.empty(B.sod2_attention_workspace_bytes(heads, kv, dim), dtype=torch.uint8, device="cuda")
        self.args = (self.t.data_ptr(), self.t.numel())


def prompt(dtype, q, k, v, out, cu, scale, status=None, ws=None):
    H, kv, D = q.shape[1], k.shape[1], q.shape[2]
    ws = ws or Workspace(H, kv, D)
    B.sod2_attention_prompt(DT[dtype][0], cu.numel() - 1, q.shape[0], H, kv, D, rows(q), rows(k), rows(v), rows(out), cu.data_ptr(), scale, *ws.args,
                            None if status is None else status.data_ptr(), stream())


def paged(dtype, q, out, cu, ctx, kc, vc, table, scale, max_new=0, status=None, ws=None, width=None):
    H, kv, D = q.shape[1], kc.shape[2], q.shape[2]
    ws = ws or Workspace(H, kv, D)
    B.sod2_attention_paged(DT[dtype][0], cu.numel() - 1, q.shape[0], max_new, H, kv, D, rows(q), rows(out), cu.data_ptr(), ctx.data_ptr(), pages(kc),
                           pages(vc), kc.shape[0], kc.shape[1], table.data_ptr(), table.stride(0), table.shape[1] if width is None else width, scale,
                           *ws.args, None if status is None else status.data_ptr(), stream())


def gather_pages(cache, ids, m):
    """The first m rows behind the page ids, out-of-pool pages as zeros."""
    page = cache.shape[1]
    out = torch.zeros(len(ids) * page, *cache.shape[2:], dtype=torch.float64, device=cache.device)
    for i, p in enumerate(ids):
        if 0 <= p < cache.shape[0]:
            out[i * page:(i + 1) * page] = cache[p].double()
    return out[:m]


# ------------------------------------------------------------------------------------------------ rotary positions
def turn(x, positions, freq, axis, adjacent):
    """x [T, H, D] in float64, turned."""
    n = len(freq)
    first = torch.arange(n) * 2 if adjacent else torch.arange(n)
    second = first + (1 if adjacent else n)
    angle = torch.stack([positions[a].double() * f for f, a in zip(freq, axis)], 1)[:, None]
    y = x.double().clone()
    a, b = x.double()[..., first], x.double()[..., second]
    y[..., first] = a * angle.cos() - b * angle.sin()
    y[..., second] = b * angle.cos() + a * angle.sin()
    size = torch.zeros_like(y)          # |x| + |y| of the pair
    size[..., first] = size[..., second] = a.abs() + b.abs()
    return y, size


def turn_tolerance(dtype, want, size):
    """One rounding of the result (below the smallest normal number the step is absolute: f16 numbers under 2^-14 are 2^-24 apart, and a
    result that is rounded there is off by up to 2^-25 whatever its size); the angle (reduced exactly enough, half a turn at most in 32 bits), its sine and cosine (2^-23 each) and
    the two products and their sum in 32 bits: together under 2^-20 of |x| + |y|."""
    return torch.finfo(DT[dtype][1]).eps / 2 * want.abs() + subnormal_half_step(dtype) + 2.0 ** -20 * size


# ------------------------------------------------------------------------------------------------ page tables
def tables(past, new, page, free, head, table, cap):
    """Plain Python: (table, cu, ctx, slots, positions, head)."""
    table = [list(r) for r in table]
    cu, slots, positions = [0], [], []
    for r, (p, n) in enumerate(zip(past, new)):
        p, n = max(p, 0), max(n, 0)
        owned = {}
        for j in range(math.ceil(p / page), math.ceil((p + n) / page)):
            owned[j] = free[head] if head < len(free) else -1
            if j < len(table[r]):
                table[r][j] = owned[j]
            head += 1
        for t in range(p, p + n):
            j = t // page
            i = -1 if j >= len(table[r]) else table[r][j]
            slots.append(i * page + t % page if i >= 0 else -1)
            positions.append(t)
        cu.append(cu[-1] + n)
    slots, positions = slots[:cap], positions[:cap]
    slots += [-1] * (cap - len(slots))
    positions += [-1] * (cap - len(positions))
    return table, [min(c, cap) for c in cu], [max(p, 0) + max(n, 0) for p, n in zip(past, new)], slots, positions, head
