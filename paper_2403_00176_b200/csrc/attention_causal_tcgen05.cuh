// Causal attention with grouped heads on tcgen05 / TMEM, over packed prompts or a paged cache (attention_causal.cuh has the
// definition and the form for what tensor maps cannot express).
//
// The query rows of a work item are TOK tokens x G heads of one key head, TOK = floor(128 / G): keys and values are read once for
// all heads of a group, and a tile of 128 rows ends at one diagonal whatever G is.  An item is two such tiles (A and B, 2 TOK
// consecutive tokens), which walk the request's keys in blocks of 128 together:
//   S = Q K^T      tcgen05.mma, M = 128, N = 128, K = head size (both operands K-major TMA tiles)
//   P = 2^(S c - m)  a thread per row: 128 scores from TMEM, P back as packed 16-bit pairs over S's first columns
//   O += P V       tcgen05.mma with A in TMEM; V is the natural [key, d] tile, used as an MN-major B operand
// While one tile is in its exponentials the tensor pipe works for the other.  P lies over S (512 columns hold two of S and
// two of O), so a tile's next S waits for its last product by commit: the order of two MMAs on different accumulators is not
// documented.  Each tile has an issuing warp of its own, so that this wait holds up nobody else.
//
// Scores, maximum, sum and O are 32-bit; P is rounded to the type of the values (the product's operand type), once.  The exponent
// reference m moves only when a row's maximum exceeds it by more than 2^8 after scaling: O is rescaled rarely, and always
// between two products, since S of a block is issued behind the products of the blocks before.
//
// Work is divided evenly over the CTAs (one per SM): items are laid end to end, an item weighing its blocks of keys and one
// more for its start and end, and cut into equal shares.  A cut inside an item makes two parts; each leaves its O, m and l in
// the workspace and causal_join puts them together.  Cuts near an item's ends move there.  All lengths are on the device, so every
// CTA works the division out itself: prefix sums over the requests, then a search.
//
// Keys behind a row's last are masked by selection before the maximum.  Values behind the request's last key may be anything: their rows of
// V in shared memory are zeroed before the product.  A value inside the request but behind a row's last key meets a probability of
// zero, which leaves it out unless it is not finite; a row whose result is not finite is therefore computed again key by key
// (causal_row).  Rows of a tile without a token, and tiles without one, are computed on whatever is there and never stored.
//
// Warps: 0..3 softmax of tile A, 4..7 of tile B, 8 loads Q and K, 9 loads V, 10 / 11 issue the MMAs of A / B.  A box of the cache
// is the part of a page that lies in a block; lanes issue boxes side by side: a lane on its own sustains one per 440 cycles
// (16 rows: 1.3 TB/s over the GPU), 16 lanes of two warps 6.5 TB/s.  Every wait is bounded (ptx.cuh).
#pragma once
#include <cuda.h>
#include "attention_causal.cuh"
#include "ptx.cuh"

namespace sod2 {
namespace k {

constexpr int CTC_THREADS = 384;
constexpr int CTC_GRID = 148;              // CTAs of the division: one per SM
constexpr int CTC_KB = 128;                // keys per block
constexpr int CTC_CHUNK = 128 * 128;       // bytes of 128 rows x 64 elements
constexpr int CTC_PLAN = CTC_THREADS;      // requests per step of the division
constexpr int CTC_SNAP = 2;                // blocks: cuts closer than this to an item's ends move there

struct CtcParams {
  CausalParams c;
  float scale_log2e;
  int G, tok;                 // heads per key head, tokens per tile
  int ksteps, n_pv;           // head size in steps of 16, and rounded up to 16
  int box_rows;               // keys per TMA box
  int cut;                    // 1: items may be cut (the workspace is there)
  float* part_o;              // [2 * CTC_GRID slots][2 tiles][DP][128 rows]
  float2* part_ml;            // [2 * CTC_GRID slots][2 tiles][128 rows]: reference (log2) and sum
  int4* desc;                 // [2 * CTC_GRID]: state (0 none, 1 part, 2 part that ends the item), request, key head, tile pair
};

template <int DP> struct CtcShape {
  static constexpr int NC = DP / 64;                    // 64-element chunks of a row
  static constexpr int TILE = NC * CTC_CHUNK;           // bytes of a Q, K or V tile
  static constexpr int ST = DP == 128 ? 5 : 8;          // K and V tiles in flight
  static constexpr int SMEM = (2 + ST) * TILE + 1024 /*align*/ + 1024 /*barriers, plan*/;
  static constexpr uint32_t TM_S = 0, TM_O = 256;       // columns: S (and P) at 128 per tile, O at DP per tile
};

// ------------------------------------------------------------------------------------------------ division of the work
struct CtcReq { int first, n, past; };     // n = 0: nothing to do
__device__ __forceinline__ CtcReq ctc_request(const CausalParams& c, int r) {
  CtcReq q;
  q.first = causal_cu(c, r);
  const int n = causal_cu(c, r + 1) - q.first;
  q.n = n > 0 ? n : 0;
  q.past = causal_ctx(c, r, q.n) - q.n;    // may be negative: the first rows see nothing
  return q;
}
// blocks of keys that the tokens below `end` see
__device__ __forceinline__ int ctc_blocks(const CtcReq& q, int end) {
  const int v = q.past + (end < q.n ? end : q.n);
  return v > 0 ? (v + CTC_KB - 1) / CTC_KB : 0;
}
__device__ __forceinline__ int ctc_pairs(const CtcReq& q, int tok) { return (q.n + 2 * tok - 1) / (2 * tok); }

struct CtcSpot { long long at, item; int r, head, pair, off; };    // position, its item's first, and where that is

// Moves a position inside an item to where it may be cut.  off: 0 the item's start, else blocks ahead of the cut + 1.
__device__ __forceinline__ int ctc_snap(int off, int blocks, bool cut) {
  const int w = blocks + 1, j = off - 1;
  if (off == 0) return 0;
  if (!cut || blocks < 2 * CTC_SNAP) return 2 * off <= w ? 0 : w;
  if (j < CTC_SNAP) return 0;
  return blocks - j < CTC_SNAP ? w : off;
}

// A role's walk over the CTA's share.
struct CtcSeg { int r, head, pair, first, n, past, j0, j1; bool starts, ends; };
struct CtcWalk {
  long long left;
  int r, head, pair, off;
  CtcReq q;
  __device__ __forceinline__ void start(const CtcParams& p, const CtcSpot& a, long long units) {
    left = units; r = a.r; head = a.head; pair = a.pair; off = a.off;
    q.n = 0;
    if (left > 0) q = ctc_request(p.c, r);
  }
  __device__ __forceinline__ bool next(const CtcParams& p, CtcSeg& s) {
    if (left <= 0) return false;
    while (pair >= ctc_pairs(q, p.tok)) {
      pair = 0;
      if (q.n > 0 && ++head < p.c.HK) continue;
      head = 0;
      if (++r >= p.c.n_req) { left = 0; return false; }
      q = ctc_request(p.c, r);
    }
    const int blocks = ctc_blocks(q, (pair + 1) * 2 * p.tok), w = blocks + 1;
    const int end = left < w - off ? off + static_cast<int>(left) : w;
    s.r = r; s.head = head; s.pair = pair; s.first = q.first; s.n = q.n; s.past = q.past;
    s.j0 = off > 0 ? off - 1 : 0;
    s.j1 = end - 1;                       // end = off + 1 with off = 0: the item's start alone, no block
    s.starts = off == 0; s.ends = end == w;
    left -= end - off;
    off = 0;
    ++pair;
    return true;
  }
};

// Finds the item that holds position x of a request whose items start at `start`; a whole warp.
__device__ __forceinline__ CtcSpot ctc_locate(const CtcParams& p, int r, long long start, long long x, bool cut) {
  const int lane = threadIdx.x & 31;
  const CtcReq q = ctc_request(p.c, r);
  const int np = ctc_pairs(q, p.tok);
  long long per = 0;                      // weight of one key head
  for (int i = lane; i < np; i += 32) per += ctc_blocks(q, (i + 1) * 2 * p.tok) + 1;
#pragma unroll
  for (int d = 16; d; d >>= 1) per += __shfl_xor_sync(0xffffffffu, per, d);
  CtcSpot s;
  s.r = r; s.at = x;
  s.head = per > 0 ? static_cast<int>((x - start) / per) : 0;
  long long base = start + s.head * per;
  for (int i0 = 0; i0 < np; i0 += 32) {
    const int w = i0 + lane < np ? ctc_blocks(q, (i0 + lane + 1) * 2 * p.tok) + 1 : 0;
    int inc = w;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) { const int y = __shfl_up_sync(0xffffffffu, inc, d); if (lane >= d) inc += y; }
    const unsigned hit = __ballot_sync(0xffffffffu, x < base + inc);
    if (hit) {
      const int l = __ffs(hit) - 1, wl = __shfl_sync(0xffffffffu, w, l), il = __shfl_sync(0xffffffffu, inc, l);
      s.pair = i0 + l;
      s.item = base + il - wl;
      const int off = ctc_snap(static_cast<int>(x - s.item), wl - 1, cut);
      s.at = s.item + off;
      s.off = off;
      if (off == wl) { s.item = s.at; s.off = 0; ++s.pair; }     // the next item's start; CtcWalk goes on to the next head or request
      return s;
    }
    base += __shfl_sync(0xffffffffu, inc, 31);
  }
  s.pair = np; s.item = s.at; s.off = 0;
  return s;
}

// The CTA's share: from spot[0] to spot[1].  Called by all threads; `weight` and `spot` are shared.
__device__ __forceinline__ void ctc_divide(const CtcParams& p, long long* weight, CtcSpot* spot) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  long long total = 0, lo = 0, hi = 0;
  // once for the total, once more for the places of the share's ends (the same chunk, with few requests)
  for (int pass = 0; pass < 2; ++pass) {
    long long base = 0;
    for (int r0 = 0; r0 < p.c.n_req; r0 += CTC_PLAN) {
      const int nr = p.c.n_req - r0 < CTC_PLAN ? p.c.n_req - r0 : CTC_PLAN;
      if (pass == 0 || p.c.n_req > CTC_PLAN) {
        __syncthreads();
        if (static_cast<int>(threadIdx.x) < nr) {
          const CtcReq q = ctc_request(p.c, r0 + threadIdx.x);
          const int np = ctc_pairs(q, p.tok);
          long long w = 0;
          if (np <= 64) for (int i = 0; i < np; ++i) w += ctc_blocks(q, (i + 1) * 2 * p.tok) + 1;
          weight[threadIdx.x] = np <= 64 ? w * p.c.HK : -1;
        }
        __syncthreads();
        for (int i = warp; i < nr; i += CTC_THREADS / 32) {        // long requests: a warp each
          if (weight[i] >= 0) continue;
          const CtcReq q = ctc_request(p.c, r0 + i);
          const int np = ctc_pairs(q, p.tok);
          long long w = 0;
          for (int t = lane; t < np; t += 32) w += ctc_blocks(q, (t + 1) * 2 * p.tok) + 1;
#pragma unroll
          for (int d = 16; d; d >>= 1) w += __shfl_xor_sync(0xffffffffu, w, d);
          __syncwarp();
          if (lane == 0) weight[i] = w * p.c.HK;
        }
        __syncthreads();
      }
      // every warp sums the chunk: 12 requests a lane
      long long sum = 0;
      for (int e = 0; e < CTC_PLAN / 32; ++e) { const int i = lane * (CTC_PLAN / 32) + e; if (i < nr) sum += weight[i]; }
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
          int i = l * (CTC_PLAN / 32);
          while (x >= start + weight[i]) { start += weight[i]; ++i; }
          const CtcSpot s = ctc_locate(p, r0 + i, start, x, p.cut);
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
        spot[0].r = spot[1].r = p.c.n_req; spot[0].head = spot[1].head = spot[0].pair = spot[1].pair = 0;
      }
      __syncthreads();
    }
  }
  __syncthreads();
}

// ------------------------------------------------------------------------------------------------ the kernel
template <class T> struct CtcType;
template <> struct CtcType<__nv_bfloat16> {
  static constexpr uint32_t fmt = (1u << 7) | (1u << 10);
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) { const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi); return *reinterpret_cast<const uint32_t*>(&h); }
};
template <> struct CtcType<__half> {
  static constexpr uint32_t fmt = 0;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) { const __half2 h = __floats2half2_rn(lo, hi); return *reinterpret_cast<const uint32_t*>(&h); }
};
// instruction descriptor, kind::f16, 32-bit accumulator, M = 128; mn_b: the B operand is MN-major
template <class T> __device__ __forceinline__ uint32_t ctc_idesc(int N, bool mn_b) {
  return (1u << 4) | CtcType<T>::fmt | (mn_b ? 1u << 16 : 0u) | (static_cast<uint32_t>(N >> 3) << 17) | (8u << 24);
}
// 128-byte swizzled MN-major tile of 64-element chunks: chunks CTC_CHUNK apart, groups of 8 rows 1024 B apart
__device__ __forceinline__ uint64_t ctc_desc_mn(uint32_t addr) {
  return (ptx::smem_desc_sw128(addr) & ~(uint64_t(0x3FFF) << 16)) | (static_cast<uint64_t>(CTC_CHUNK >> 4) << 16);
}
__device__ __forceinline__ float ctc_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float ctc_max32(float mx, const uint32_t* s) {
  float a = mx, b = -INFINITY;
#pragma unroll
  for (int e = 0; e < 32; e += 4) {
    a = fmaxf(fmaxf(a, __uint_as_float(s[e])), __uint_as_float(s[e + 1]));
    b = fmaxf(fmaxf(b, __uint_as_float(s[e + 2])), __uint_as_float(s[e + 3]));
  }
  return fmaxf(a, b);
}
template <class T>
__device__ __forceinline__ void ctc_exp32(const uint32_t* s, uint32_t* pk, float2 c2, float2 mc2, float2* l) {
#pragma unroll
  for (int e = 0; e < 32; e += 2) {
    const float2 t = ptx::fma_x2(make_float2(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), c2, mc2);
    const float2 q = make_float2(ctc_ex2(t.x), ctc_ex2(t.y));
    *l = ptx::add_x2(*l, q);
    pk[e >> 1] = CtcType<T>::pack(q.x, q.y);
  }
}

template <class T, int DP>
__global__ void __launch_bounds__(CTC_THREADS, 1)
causal_attention_tcgen05(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                         const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CtcParams p) {
  using Sh = CtcShape<DP>;
  constexpr int ST = Sh::ST;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sQ = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));   // [2 tiles]
  uint8_t* sKV = sQ + 2 * Sh::TILE;                                                                               // [ST], K and V in turn
  uint64_t* bars = reinterpret_cast<uint64_t*>(sKV + ST * Sh::TILE);
  uint64_t* q_full = bars;            // [2] per tile: Q landed
  uint64_t* q_free = bars + 2;        // [2] the item's last S is done
  uint64_t* s_full = bars + 4;        // [2] S done
  uint64_t* p_full = bars + 6;        // [2] P written
  uint64_t* o_full = bars + 8;        // [2] product done
  uint64_t* kv_full = bars + 10;      // [ST]
  uint64_t* kv_free = bars + 10 + ST; // [ST] both tiles are through with it
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 10 + 2 * ST);
  volatile int* dead = reinterpret_cast<volatile int*>(tmem_slot + 1);
  CtcSpot* spot = reinterpret_cast<CtcSpot*>(bars + 12 + 2 * ST);       // [2]
  long long* weight = reinterpret_cast<long long*>(sKV);                // [CTC_PLAN], ahead of the first load

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int b = 0; b < 2; ++b) {
      ptx::mbar_init(&q_full[b], 1); ptx::mbar_init(&q_free[b], 1);
      ptx::mbar_init(&s_full[b], 1); ptx::mbar_init(&p_full[b], 4); ptx::mbar_init(&o_full[b], 1);
    }
    for (int b = 0; b < ST; ++b) { ptx::mbar_init(&kv_full[b], 1); ptx::mbar_init(&kv_free[b], 2); }
    *dead = 0;
    ptx::fence_barrier_init();
    ptx::prefetch_tmap(&tmQ);
    ptx::prefetch_tmap(&tmK);
    ptx::prefetch_tmap(&tmV);
  }
  if (warp == 10) { ptx::tmem_alloc(tmem_slot, 512); ptx::tmem_relinquish(); }
  ptx::pdl_wait();
  ctc_divide(p, weight, spot);
  ptx::fence_proxy_async();           // the plan's scratch becomes the load ring
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const CtcSpot from = spot[0], to = spot[1];
  const long long units = to.at - from.at;
  ptx::pdl_launch();
  if (p.cut && threadIdx.x < 2) {     // what this CTA leaves in its two slots
    int4 d = make_int4(0, 0, 0, 0);
    if (threadIdx.x == 0) {           // the item that an earlier CTA began
      if (from.off > 0 && units > 0) d = make_int4(to.off > 0 && to.item == from.item ? 1 : 2, from.r, from.head, from.pair);
    } else if (to.off > 0 && to.item >= from.at) {                  // the item that this CTA begins and leaves unfinished
      d = make_int4(1, to.r, to.head, to.pair);
    }
    p.desc[2 * blockIdx.x + threadIdx.x] = d;
  }
  CtcWalk walk;
  walk.start(p, from, units);
  CtcSeg s;
  const int tok = p.tok;
  // blocks of the segment that tile t takes part in
  auto blocks_of = [&](const CtcSeg& g, int t) {
    const int t0 = (2 * g.pair + t) * tok;
    if (t0 >= g.n) return 0;
    const CtcReq q{g.first, g.n, g.past};
    const int b = ctc_blocks(q, t0 + tok);
    const int e = b < g.j1 ? b : g.j1;
    return e > g.j0 ? e - g.j0 : 0;
  };

  if (warp == 8 || warp == 9) {
    // ---- TMA producers: warp 8 Q and the K tiles (even turns of the ring), warp 9 the V tiles (odd ones)
    const bool is_k = warp == 8;
    const CUtensorMap* tm = is_k ? &tmK : &tmV;
    int turn = is_k ? 0 : 1, qn[2] = {0, 0};
    const int per = CTC_KB / p.box_rows;                  // boxes of 64 columns in a block
    const int chunk = lane / per, box = lane - chunk * per;
    const int* table = p.c.table;
    int bad = 0;
    while (walk.next(p, s)) {
      if (is_k) {
        for (int t = 0; t < 2; ++t) {
          if (blocks_of(s, t) == 0) continue;
          if (qn[t] > 0) ptx::mbar_wait_warp(&q_free[t], (qn[t] - 1) & 1, dead);
          ++qn[t];
          if (*dead) continue;
          if (lane == 0) ptx::mbar_expect_tx(&q_full[t], Sh::NC * 128 * tok * p.G);
          __syncwarp();
          if (lane < Sh::NC)
            ptx::tma_load_4d(sQ + t * Sh::TILE + lane * CTC_CHUNK, &tmQ, lane * 64, 0, s.first + (2 * s.pair + t) * tok, s.head, &q_full[t]);
          __syncwarp();
        }
      }
      const int ctx = s.past + s.n;
      const int* ids = table ? table + s.r * p.c.table_stride : nullptr;
      // the page of this lane's box, looked up a block ahead
      auto page_of = [&](int j) {
        const int row = j * CTC_KB + box * p.box_rows;
        return chunk < Sh::NC && j < s.j1 && row < ctx ? ids[row / p.c.page] : 0;
      };
      int id = table ? page_of(s.j0) : 0;
      for (int j = s.j0; j < s.j1; ++j, turn += 2) {
        const int b = turn % ST, use = turn / ST, row = j * CTC_KB + box * p.box_rows;
        const bool mine = chunk < Sh::NC && (!table || row < ctx);
        const int ahead = table ? page_of(j + 1) : 0;
        if (use > 0) ptx::mbar_wait_warp(&kv_free[b], (use - 1) & 1, dead);
        if (*dead) continue;
        const int n = __popc(__ballot_sync(0xffffffffu, mine));
        if (lane == 0) ptx::mbar_expect_tx(&kv_full[b], n * p.box_rows * 128);
        __syncwarp();
        if (mine) {
          uint8_t* dst = sKV + b * Sh::TILE + chunk * CTC_CHUNK + box * p.box_rows * 128;
          if (table) {
            int page = id;
            if (page < 0 || page >= p.c.n_pages) { page = p.c.n_pages; bad = SERVE_BAD_PAGE; }   // outside the map: zeros
            ptx::tma_load_4d(dst, tm, chunk * 64, row % p.c.page, s.head, page, &kv_full[b]);
          } else {
            ptx::tma_load_4d(dst, tm, chunk * 64, s.first + row, s.head, 0, &kv_full[b]);
          }
        }
        __syncwarp();
        id = ahead;
      }
    }
    if (bad && p.c.status) atomicOr(p.c.status, bad);
  } else if (warp >= 10) {
    // ---- MMA issuers: S of the next block behind the product of this one
    const int t = warp - 10;
    const ptx::Leader one = ptx::elect_leader();
    const uint32_t idesc_qk = ctc_idesc<T>(CTC_KB, false), idesc_pv = ctc_idesc<T>(p.n_pv, true);
    const uint32_t tS = tmem + Sh::TM_S + t * 128, tO = tmem + Sh::TM_O + t * DP;
    const uint64_t dQ = ptx::smem_desc_sw128(ptx::smem_u32(sQ + t * Sh::TILE));
    int turn = 0, items = 0, n = 0;          // ring turns, items and blocks of this tile so far
    while (walk.next(p, s)) {
      const int len = s.j1 - s.j0, mine = blocks_of(s, t);
      if (mine > 0) { ptx::mbar_wait_warp(&q_full[t], items & 1, dead); ++items; }
      auto issue_s = [&](int i) {
        const int b = (turn + 2 * i) % ST, use = (turn + 2 * i) / ST;
        const uint64_t dK = ptx::smem_desc_sw128(ptx::smem_u32(sKV + b * Sh::TILE));
        ptx::mbar_wait_lanes(&kv_full[b], use & 1, dead);
        ptx::tc_fence_after();
        for (int kk = 0; kk < p.ksteps; ++kk) {
          const uint64_t step = (kk >> 2) * (CTC_CHUNK >> 4) + 2 * (kk & 3);
          ptx::mma_bf16(one, tS, dQ + step, dK + step, idesc_qk, kk != 0);
        }
        __syncwarp();
        ptx::mma_commit(one, &s_full[t]);
        ptx::mma_commit(one, &kv_free[b]);
        if (i + 1 == mine) ptx::mma_commit(one, &q_free[t]);
      };
      auto pass = [&](int i) {                // a tile that this one has no part in
        const int b = i % ST, use = i / ST;
        ptx::mbar_wait_warp(&kv_full[b], use & 1, dead);
        ptx::mbar_arrive_warp(&kv_free[b]);
      };
      const int v_end = s.past + ((2 * s.pair + t + 1) * tok < s.n ? (2 * s.pair + t + 1) * tok : s.n);   // keys that the tile sees
      for (int i = 0; i < len; ++i) {
        if (i >= mine) { pass(turn + 2 * i); pass(turn + 2 * i + 1); continue; }
        if (i == 0) issue_s(0);
        const int b = (turn + 2 * i + 1) % ST, use = (turn + 2 * i + 1) / ST;
        const uint32_t aV = ptx::smem_u32(sKV + b * Sh::TILE);
        const int keys = v_end - (s.j0 + i) * CTC_KB, steps = keys < CTC_KB ? (keys + 15) >> 4 : CTC_KB / 16;
        ptx::mbar_wait_lanes(&kv_full[b], use & 1, dead);
        ptx::mbar_wait_lanes(&p_full[t], n & 1, dead);
        ptx::tc_fence_after();
        for (int kk = 0; kk < steps; ++kk)
          ptx::mma_bf16_a_tmem(one, tO, tS + kk * 8, ctc_desc_mn(aV + kk * 2048), idesc_pv, (i | kk) != 0);
        __syncwarp();
        ptx::mma_commit(one, &o_full[t]);
        ptx::mma_commit(one, &kv_free[b]);
        if (i + 1 < mine) {
          ptx::mbar_wait_warp(&o_full[t], n & 1, dead);       // P is read: S may be written over it
          issue_s(i + 1);
        }
        ++n;
      }
      turn += 2 * len;
    }
  } else {
    // ---- softmax warps: tile t = warp / 4, a thread per row
    const int t = warp >> 2, row = threadIdx.x & 127;
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + lane_base + Sh::TM_S + t * 128, tO = tmem + lane_base + Sh::TM_O + t * DP;
    const float c = p.scale_log2e;
    const int rt = row / p.G, rg = row - rt * p.G;
    int turn = 0, n = 0;
    while (walk.next(p, s)) {
      const int len = s.j1 - s.j0, mine = blocks_of(s, t), t0 = (2 * s.pair + t) * tok;
      const bool valid = rt < tok && t0 + rt < s.n;
      const int lim = valid ? s.past + t0 + rt + 1 : 0;       // keys that the row sees
      const bool live = __any_sync(0xffffffffu, valid);
      const int ctx = s.past + s.n;
      const int v_end = s.past + (t0 + tok < s.n ? t0 + tok : s.n);
      float m = -INFINITY;
      float2 l = make_float2(0.f, 0.f);
      for (int i = 0; i < mine; ++i, ++n) {
        const int j = s.j0 + i, b = (turn + 2 * i + 1) % ST, use = (turn + 2 * i + 1) / ST;
        if ((j + 1) * CTC_KB > ctx) {
          // values behind the request's last key, as far as the product reads: zeros
          const int first = ctx - j * CTC_KB;
          if (row >= first && row < ((first + 15) & ~15)) {
            ptx::mbar_wait_lanes(&kv_full[b], use & 1, dead);
            uint4* v = reinterpret_cast<uint4*>(sKV + b * Sh::TILE + row * 128);
#pragma unroll
            for (int h = 0; h < Sh::NC; ++h)
#pragma unroll
              for (int e = 0; e < 8; ++e) v[h * (CTC_CHUNK / 16) + e] = make_uint4(0, 0, 0, 0);
            ptx::fence_proxy_async();
          }
          __syncwarp();
        }
        ptx::mbar_wait_warp(&s_full[t], n & 1, dead);
        ptx::tc_fence_after();
        if (live) {
          uint32_t sc[128];
#pragma unroll
          for (int h = 0; h < 4; ++h) ptx::tmem_ld32(tS + h * 32, sc + h * 32);
          ptx::tmem_ld_wait();
          const int seen = lim - j * CTC_KB;
          if (__any_sync(0xffffffffu, seen < CTC_KB)) {
#pragma unroll
            for (int e = 0; e < 128; ++e) if (e >= seen) sc[e] = 0xff800000u;   // -inf
          }
          const float mx = ctc_max32(ctc_max32(ctc_max32(ctc_max32(-INFINITY, sc), sc + 32), sc + 64), sc + 96);
          const bool move = (mx - m) * c > 8.0f;            // false while both are -inf
          if (i == 0) m = mx;
          else if (__any_sync(0xffffffffu, move)) {
            float corr = 1.f;
            if (move) { corr = ctc_ex2((m - mx) * c); m = mx; l.x *= corr; l.y *= corr; }
#pragma unroll 1
            for (int h = 0; h < p.n_pv; h += 16) {
              uint32_t r[16];
              ptx::tmem_ld8(tO + h, r);
              ptx::tmem_ld8(tO + h + 8, r + 8);
              ptx::tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * corr);
              ptx::tmem_st16(tO + h, r);
            }
          }
          const float ref = m == -INFINITY ? 0.f : m;       // a row that has seen nothing: all its P are zero
          const float2 c2 = make_float2(c, c), mc2 = make_float2(-ref * c, -ref * c);
          const int upto = v_end - j * CTC_KB;              // columns that the product reads
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            if (h * 32 < upto) {
              uint32_t pk[16];
              ctc_exp32<T>(sc + h * 32, pk, c2, mc2, &l);
              ptx::tmem_st16(tS + h * 16, pk);
            }
          }
          ptx::tmem_st_wait();
        }
        ptx::tc_fence_before();
        __syncwarp();
        ptx::mbar_arrive_warp(&p_full[t]);
      }
      turn += 2 * len;
      // ---- the segment's end
      if (mine > 0) { ptx::mbar_wait_warp(&o_full[t], (n - 1) & 1, dead); ptx::tc_fence_after(); }
      const float lsum = l.x + l.y;
      if (s.starts && s.ends) {
        const float inv = lim > 0 ? 1.f / lsum : 0.f;
        const int h = s.head * p.G + rg;
        const long long orow = s.first + t0 + rt;
        T* o = static_cast<T*>(p.c.o) + orow * p.c.o_ts + h * p.c.o_hs;
        bool odd = false;                                   // something not finite
#pragma unroll 1
        for (int d = 0; d < p.c.D; d += 16) {
          uint32_t r[16];
          if (mine > 0 && live) {
            ptx::tmem_ld8(tO + d, r);
            ptx::tmem_ld8(tO + d + 8, r + 8);
            ptx::tmem_ld_wait();
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) r[e] = 0;
          }
          uint4 v[2];
          uint32_t* w = reinterpret_cast<uint32_t*>(v);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float x = __uint_as_float(r[2 * e]) * inv, y = __uint_as_float(r[2 * e + 1]) * inv;
            odd |= !(fabsf(x) < INFINITY) || !(fabsf(y) < INFINITY);
            w[e] = CtcType<T>::pack(x, y);
          }
          if (valid) {
            *reinterpret_cast<uint4*>(o + d) = v[0];
            if (d + 8 < p.c.D) *reinterpret_cast<uint4*>(o + d + 8) = v[1];
          }
        }
        unsigned redo = __ballot_sync(0xffffffffu, valid && odd);
        __syncwarp();                                       // the rows written above are written again by the whole warp
        while (redo) {                                      // rare: see the top of the file
          const int src = __ffs(redo) - 1;
          redo &= redo - 1;
          const int rr = __shfl_sync(0xffffffffu, static_cast<int>(orow), src), hh = __shfl_sync(0xffffffffu, h, src), seen = __shfl_sync(0xffffffffu, lim, src);
          causal_row<T>(p.c, s.r, s.first, rr, hh, seen);
        }
      } else {
        const long long tile = (2LL * blockIdx.x + (s.starts ? 1 : 0)) * 2 + t;
        float* po = p.part_o + tile * DP * 128 + row;
        if (live) {
#pragma unroll 1
          for (int d = 0; d < p.n_pv; d += 16) {
            uint32_t r[16];
            if (mine > 0) {
              ptx::tmem_ld8(tO + d, r);
              ptx::tmem_ld8(tO + d + 8, r + 8);
              ptx::tmem_ld_wait();
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) po[(d + e) * 128] = mine > 0 ? __uint_as_float(r[e]) : 0.f;
          }
          p.part_ml[tile * 128 + row] = make_float2(mine > 0 && m != -INFINITY ? m * c : -INFINITY, mine > 0 ? lsum : 0.f);
        }
      }
      ptx::tc_fence_before();
      __syncwarp();
    }
  }
  __syncwarp();
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == 10) ptx::tmem_dealloc(tmem, 512);
  if (threadIdx.x == 0 && *dead && p.c.status) atomicOr(p.c.status, 1);
}

// Puts the parts of a cut item together: CTA (c, t, quarter) the 32 rows of tile t of the item that CTA c of the attention began and
// left unfinished, if any.  out = sum 2^(m_i - m) O_i / sum 2^(m_i - m) l_i over the parts in their order: the same result every time.
template <class T, int DP>
__global__ void __launch_bounds__(256) causal_join(const __grid_constant__ CtcParams p) {
  __shared__ float out_s[32][DP + 1];
  __shared__ int odd_s[32];
  const int c = blockIdx.x, t = blockIdx.y >> 2, row = (blockIdx.y & 3) * 32 + (threadIdx.x & 31), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  ptx::pdl_wait();
  const int4 d = p.desc[2 * c + 1];
  if (d.x == 0) return;
  const CtcReq q = ctc_request(p.c, d.y);
  const int t0 = (2 * d.w + t) * p.tok, rt = row / p.G;
  const bool valid = rt < p.tok && t0 + rt < q.n;
  if (threadIdx.x < 32) odd_s[lane] = 0;
  if (!__syncthreads_or(valid)) return;
  int last = c;                       // the CTA that ends the item
  while (last + 1 < CTC_GRID) { ++last; if (p.desc[2 * last].x == 2) break; }
  auto tile_of = [&](int i) { return (2LL * i + (i == c ? 1 : 0)) * 2 + t; };
  float m = -INFINITY;
  for (int i = c; i <= last; ++i) if (i == c || p.desc[2 * i].x) m = fmaxf(m, valid ? p.part_ml[tile_of(i) * 128 + row].x : -INFINITY);
  constexpr int PER = DP / 8;         // columns of a warp
  float l = 0.f, acc[PER] = {};
  for (int i = c; i <= last && valid; ++i) {
    if (i != c && !p.desc[2 * i].x) continue;
    const float2 ml = p.part_ml[tile_of(i) * 128 + row];
    const float w = ml.x == -INFINITY ? 0.f : exp2f(ml.x - m);
    l = fmaf(w, ml.y, l);
    const float* po = p.part_o + (tile_of(i) * DP + warp * PER) * 128 + row;
    if (ml.x != -INFINITY)            // (a part in which the row saw nothing; NaN goes on)
#pragma unroll
      for (int e = 0; e < PER; ++e) if (warp * PER + e < p.n_pv) acc[e] = fmaf(w, po[e * 128], acc[e]);
  }
  const int lim = valid ? q.past + t0 + rt + 1 : 0;
  const float inv = lim > 0 ? 1.f / l : 0.f;
  bool odd = false;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const float x = acc[e] * inv;
    odd |= warp * PER + e < p.c.D && !(fabsf(x) < INFINITY);
    out_s[lane][warp * PER + e] = x;
  }
  if (odd && valid) odd_s[lane] = 1;
  __syncthreads();
  for (int r = warp; r < 32; r += 8) {
    const int rr = (blockIdx.y & 3) * 32 + r, tt = rr / p.G;
    if (tt >= p.tok || t0 + tt >= q.n) continue;
    const int h = d.z * p.G + rr - tt * p.G, orow = q.first + t0 + tt;
    if (odd_s[r]) { causal_row<T>(p.c, d.y, q.first, orow, h, q.past + t0 + tt + 1); continue; }
    T* o = static_cast<T*>(p.c.o) + orow * p.c.o_ts + h * p.c.o_hs;
    for (int e = lane; e < p.c.D; e += 32) o[e] = rope_store<T>(out_s[r][e]);
  }
}

}  // namespace k
}  // namespace sod2
