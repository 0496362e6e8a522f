// Division of the work of the attention kernels over their CTAs, on the device, where all lengths are.
// Items (some query rows of one request and key head, all its blocks of keys) are laid end to end in the order request, key head, rows; an
// item weighs its blocks and START more for its start and end.  CTA b of n takes what lies between b / n and (b + 1) / n of the whole.
// A parameter block P says what an item is: KB keys a block, START, SNAP (cuts closer than this many blocks to an item's ends move there),
// THREADS of a CTA, items(q) of a request and head, end(i): the tokens below it see the keys of item i, and takes(n): whether
// requests of n new tokens are this kernel's at all.
#pragma once
#include "attention_causal.cuh"

namespace sod2 {
namespace k {

struct CausalReq { int first, n, past; };     // n = 0: nothing to do
template <class P>
__device__ __forceinline__ CausalReq causal_request(const P& p, int r) {
  CausalReq q;
  q.first = causal_cu(p.c, r);
  const int n = causal_cu(p.c, r + 1) - q.first;
  q.past = causal_ctx(p.c, r, n) - n;      // may be negative: the first rows see nothing
  q.n = n > 0 && p.takes(n) ? n : 0;
  return q;
}
// blocks of keys that the tokens below `end` see
template <int KB>
__device__ __forceinline__ int causal_blocks(const CausalReq& q, int end) {
  const int v = q.past + (end < q.n ? end : q.n);
  return v > 0 ? (v + KB - 1) / KB : 0;
}
template <class P>
__device__ __forceinline__ int causal_item_blocks(const P& p, const CausalReq& q, int idx) { return causal_blocks<P::KB>(q, p.end(idx)); }

struct CausalSpot { long long at, item; int r, head, idx, off; };    // position, its item's first, and where that is

// Moves a position inside an item to where it may be cut.  off: 0 the item's start, else blocks ahead of the cut + START.
template <class P>
__device__ __forceinline__ int causal_snap(int off, int blocks, bool cut) {
  const int w = blocks + P::START, j = off - P::START;
  if (off == 0) return 0;
  if (!cut || blocks < 2 * P::SNAP) return 2 * off <= w ? 0 : w;
  if (j < P::SNAP) return 0;
  return blocks - j < P::SNAP ? w : off;
}

// A role's walk over the CTA's share.
struct CausalSeg { int r, head, idx, first, n, past, j0, j1; bool starts, ends; };
template <class P>
struct CausalWalk {
  long long left;
  int r, head, idx, off;
  CausalReq q;
  __device__ __forceinline__ void start(const P& p, const CausalSpot& a, long long units) {
    left = units; r = a.r; head = a.head; idx = a.idx; off = a.off;
    q.n = 0;
    if (left > 0) q = causal_request(p, r);
  }
  __device__ __forceinline__ bool next(const P& p, CausalSeg& s) {
    if (left <= 0) return false;
    while (idx >= p.items(q)) {
      idx = 0;
      if (q.n > 0 && ++head < p.c.HK) continue;
      head = 0;
      if (++r >= p.c.n_req) { left = 0; return false; }
      q = causal_request(p, r);
    }
    const int blocks = causal_item_blocks(p, q, idx), w = blocks + P::START;
    const int end = left < w - off ? off + static_cast<int>(left) : w;
    s.r = r; s.head = head; s.idx = idx; s.first = q.first; s.n = q.n; s.past = q.past;
    s.j0 = off > 0 ? off - P::START : 0;
    s.j1 = end - P::START;
    s.starts = off == 0; s.ends = end == w;
    left -= end - off;
    off = 0;
    ++idx;
    return true;
  }
};

// Finds the item that holds position x of a request whose items start at `start`; a whole warp.
template <class P>
__device__ __forceinline__ CausalSpot causal_locate(const P& p, int r, long long start, long long x, bool cut) {
  const int lane = threadIdx.x & 31;
  const CausalReq q = causal_request(p, r);
  const int np = p.items(q);
  long long per = 0;                      // weight of one key head
#pragma unroll 1
  for (int i = lane; i < np; i += 32) per += causal_item_blocks(p, q, i) + P::START;
#pragma unroll
  for (int d = 16; d; d >>= 1) per += __shfl_xor_sync(0xffffffffu, per, d);
  CausalSpot s;
  s.r = r; s.at = x;
  s.head = per > 0 ? static_cast<int>((x - start) / per) : 0;
  long long base = start + s.head * per;
#pragma unroll 1
  for (int i0 = 0; i0 < np; i0 += 32) {
    const int w = i0 + lane < np ? causal_item_blocks(p, q, i0 + lane) + P::START : 0;
    int inc = w;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) { const int y = __shfl_up_sync(0xffffffffu, inc, d); if (lane >= d) inc += y; }
    const unsigned hit = __ballot_sync(0xffffffffu, x < base + inc);
    if (hit) {
      const int l = __ffs(hit) - 1, wl = __shfl_sync(0xffffffffu, w, l), il = __shfl_sync(0xffffffffu, inc, l);
      s.idx = i0 + l;
      s.item = base + il - wl;
      const int off = causal_snap<P>(static_cast<int>(x - s.item), wl - P::START, cut);
      s.at = s.item + off;
      s.off = off;
      if (off == wl) { s.item = s.at; s.off = 0; ++s.idx; }     // the next item's start; CausalWalk goes on to the next head or request
      return s;
    }
    base += __shfl_sync(0xffffffffu, inc, 31);
  }
  s.idx = np; s.item = s.at; s.off = 0;
  return s;
}

// The CTA's share: from spot[0] to spot[1].  Called by all threads; `weight` and `spot` are shared.
template <class P>
__device__ __forceinline__ void causal_divide(const P& p, long long* weight, CausalSpot* spot) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  long long total = 0, lo = 0, hi = 0;
  // once for the total, once more for the places of the share's ends (the same chunk, with few requests)
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
    long long base = 0;
#pragma unroll 1
    for (int r0 = 0; r0 < p.c.n_req; r0 += P::THREADS) {
      const int nr = p.c.n_req - r0 < P::THREADS ? p.c.n_req - r0 : P::THREADS;
      if (pass == 0 || p.c.n_req > P::THREADS) {
        __syncthreads();
        if (static_cast<int>(threadIdx.x) < nr) {
          const CausalReq q = causal_request(p, r0 + threadIdx.x);
          const int np = p.items(q);
          long long w = 0;
          if (np <= 64)
#pragma unroll 1
            for (int i = 0; i < np; ++i) w += causal_item_blocks(p, q, i) + P::START;
          weight[threadIdx.x] = np <= 64 ? w * p.c.HK : -1;
        }
        __syncthreads();
        for (int i = warp; i < nr; i += P::THREADS / 32) {        // long requests: a warp each
          if (weight[i] >= 0) continue;
          const CausalReq q = causal_request(p, r0 + i);
          const int np = p.items(q);
          long long w = 0;
#pragma unroll 1
          for (int t = lane; t < np; t += 32) w += causal_item_blocks(p, q, t) + P::START;
#pragma unroll
          for (int d = 16; d; d >>= 1) w += __shfl_xor_sync(0xffffffffu, w, d);
          __syncwarp();
          if (lane == 0) weight[i] = w * p.c.HK;
        }
        __syncthreads();
      }
      // every warp sums the chunk: 12 requests a lane
      long long sum = 0;
#pragma unroll 1
      for (int e = 0; e < P::THREADS / 32; ++e) { const int i = lane * (P::THREADS / 32) + e; if (i < nr) sum += weight[i]; }
      long long inc = sum;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) { const long long y = __shfl_up_sync(0xffffffffu, inc, d); if (lane >= d) inc += y; }
      const long long chunk = __shfl_sync(0xffffffffu, inc, 31);
      if (pass == 1 && warp < 2) {
        const long long x = warp == 0 ? lo : hi;
        if (x >= base && x < base + chunk) {
          const long long mine = base + inc - sum;
          const unsigned own = __ballot_sync(0xffffffffu, x >= mine && x < mine + sum);
          const int l = __ffs(own) - 1;
          long long start = __shfl_sync(0xffffffffu, mine, l);
          int i = l * (P::THREADS / 32);
          while (x >= start + weight[i]) { start += weight[i]; ++i; }
          const CausalSpot s = causal_locate(p, r0 + i, start, x, p.cut);
          if (lane == 0) spot[warp] = s;
        }
      }
      base += chunk;
    }
    if (pass == 0) {
      total = base;
      lo = total * blockIdx.x / gridDim.x;
      hi = total * (blockIdx.x + 1) / gridDim.x;
      if (threadIdx.x == 0) {
        spot[0].at = spot[1].at = total; spot[0].off = spot[1].off = 0; spot[0].item = spot[1].item = total;
        spot[0].r = spot[1].r = p.c.n_req; spot[0].head = spot[1].head = spot[0].idx = spot[1].idx = 0;
      }
      __syncthreads();
    }
  }
  __syncthreads();
}

}  // namespace k
}  // namespace sod2
