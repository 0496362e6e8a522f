// Page tables and slot maps of a paged cache, and rotary positions with the store of keys and values into it.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "ptx.cuh"

namespace sod2 {
namespace k {

// bits of the status word of the serving operators (include/sod2.h)
constexpr int SERVE_BAD_PAGE = 2, SERVE_NO_PAGE = 4, SERVE_BAD_LENGTH = 8;

// ---------------------------------------------------------------------------------------------- page tables
struct PageTableParams {
  const int* past; const int* fresh;            // per request: tokens in the cache, new tokens
  const int* free_pages; const int* free_head;  // ids, first id not yet taken (null: 0)
  int* table;
  int* cu; int* ctx; long long* slots; int* positions; int* head_out; int* status;
  long long table_stride;
  int n_req, cap, page, n_free, width;
};

constexpr int PT_THREADS = 256;
constexpr int PT_CHUNK = 1024;      // requests per scan step, four per thread
constexpr int PT_TILE = 1024;       // rows of the slot map per CTA

// With have = ceil(past / page) and want = ceil((past + new) / page), request r takes the pages have .. want-1 from the free
// list at head + sum over s < r of (want_s - have_s).  Two prefix sums over the requests give that and the packed row of each
// request; every CTA makes both over all requests (8 bytes a request, out of L2) instead of a launch that hands them on,
// then fills its own tile of rows and every gridDim-th request's table entries.  A new token's page is looked up where the
// table's new entry comes from, not in the table, which other CTAs are writing.  Sums are 64-bit: lengths are any int.
__global__ void __launch_bounds__(PT_THREADS) page_tables(const __grid_constant__ PageTableParams p) {
  __shared__ long long cu_s[PT_CHUNK + 1], need_s[PT_CHUNK + 1];
  __shared__ int past_s[PT_CHUNK];
  __shared__ long long warp_s[2][PT_THREADS / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long t0 = static_cast<long long>(blockIdx.x) * PT_TILE;
  const long long t1 = t0 + PT_TILE < p.cap ? t0 + PT_TILE : p.cap;
  ptx::pdl_launch();
  ptx::pdl_wait();
  const long long head = p.free_head ? *p.free_head : 0;
  const long long page = p.page;
  long long tok = 0, need = 0;      // totals ahead of this chunk
  int bad = 0;
  for (int c0 = 0; c0 < p.n_req; c0 += PT_CHUNK) {
    long long tv[4], nv[4], ts = 0, ns = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = tid * 4 + e, r = c0 + i;
      long long a = 0, b = 0;
      if (r < p.n_req) {
        const int ra = p.past[r], rb = p.fresh[r];
        if (ra < 0 || rb < 0) bad |= SERVE_BAD_LENGTH;
        a = ra < 0 ? 0 : ra;
        b = rb < 0 ? 0 : rb;
        past_s[i] = static_cast<int>(a);
      }
      tv[e] = ts; nv[e] = ns;
      ts += b;
      ns += (a + b + page - 1) / page - (a + page - 1) / page;
    }
    long long ti = ts, ni = ns;     // inclusive over the warp's threads
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long x = __shfl_up_sync(0xffffffffu, ti, d), y = __shfl_up_sync(0xffffffffu, ni, d);
      if (lane >= d) { ti += x; ni += y; }
    }
    if (lane == 31) { warp_s[0][warp] = ti; warp_s[1][warp] = ni; }
    __syncthreads();
    long long tb = tok + ti - ts, nb = need + ni - ns;
    for (int w = 0; w < PT_THREADS / 32; ++w) {
      if (w < warp) { tb += warp_s[0][w]; nb += warp_s[1][w]; }
      tok += warp_s[0][w]; need += warp_s[1][w];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) { cu_s[tid * 4 + e] = tb + tv[e]; need_s[tid * 4 + e] = nb + nv[e]; }
    if (tid == 0) { cu_s[PT_CHUNK] = tok; need_s[PT_CHUNK] = need; }
    __syncthreads();
    const int nr = p.n_req - c0 < PT_CHUNK ? p.n_req - c0 : PT_CHUNK;
    // tables, cumulative lengths and contexts: requests in turn over all warps of the grid
    const int step = gridDim.x * (PT_THREADS / 32);
    for (int i = blockIdx.x * (PT_THREADS / 32) + warp; i < nr; i += step) {
      const long long a = past_s[i], n = cu_s[i + 1] - cu_s[i], have = (a + page - 1) / page, k = need_s[i + 1] - need_s[i];
      for (long long j = lane; j < k; j += 32) {
        const long long f = head + need_s[i] + j;
        int id = -1;
        if (f >= 0 && f < p.n_free) id = p.free_pages[f]; else bad |= SERVE_NO_PAGE;
        if (have + j < p.width) p.table[(c0 + i) * p.table_stride + have + j] = id; else bad |= SERVE_NO_PAGE;
      }
      if (lane == 0) {
        p.cu[c0 + i] = static_cast<int>(cu_s[i] < p.cap ? cu_s[i] : p.cap);
        const long long m = a + n;
        if (m > 0x7fffffff) bad |= SERVE_BAD_LENGTH;
        p.ctx[c0 + i] = static_cast<int>(m < 0x7fffffff ? m : 0x7fffffff);
      }
    }
    // slots and positions of this CTA's rows that belong to the chunk's requests
    const long long lo = t0 > cu_s[0] ? t0 : cu_s[0], hi = t1 < cu_s[nr] ? t1 : cu_s[nr];
    for (long long t = lo + tid; t < hi; t += PT_THREADS) {
      int a = 0, b = nr;            // last request whose first row is not behind t; empty requests share a first row
      while (b - a > 1) { const int m = (a + b) >> 1; if (cu_s[m] <= t) a = m; else b = m; }
      const long long pos = past_s[a] + (t - cu_s[a]), j = pos / page, have = (past_s[a] + page - 1) / page;
      int id = -1;
      if (j < p.width) {
        if (j < have) id = p.table[(c0 + a) * p.table_stride + j];
        else { const long long f = head + need_s[a] + (j - have); if (f >= 0 && f < p.n_free) id = p.free_pages[f]; }
      }
      if (p.positions) p.positions[t] = static_cast<int>(pos < 0x7fffffff ? pos : 0x7fffffff);
      p.slots[t] = id < 0 ? -1 : static_cast<long long>(id) * page + (pos - j * page);
    }
    __syncthreads();
  }
  // rows behind the last request: nothing is stored for them
  for (long long t = (t0 > tok ? t0 : tok) + tid; t < t1; t += PT_THREADS) {
    if (p.positions) p.positions[t] = -1;
    p.slots[t] = -1;
  }
  if (blockIdx.x == 0 && tid == 0) {
    if (tok > p.cap) bad |= SERVE_BAD_LENGTH;
    p.cu[p.n_req] = static_cast<int>(tok < p.cap ? tok : p.cap);
    const long long h = head + need;
    p.head_out[0] = static_cast<int>(h < 0x7fffffff ? h : 0x7fffffff);
  }
  if (bad && p.status) atomicOr(p.status, bad);
}

// ---------------------------------------------------------------------------------------------- rotary positions
constexpr int ROPE_MAX_PAIRS = 128;
struct RopeParams {
  const void* q; void* q_out; const void* k; void* k_out; const void* v;
  void* kc; void* vc; const long long* slots;
  const int* positions;
  int* status;
  long long q_ts, q_hs, qo_ts, qo_hs, k_ts, k_hs, ko_ts, ko_hs, v_ts, v_hs, pos_stride;
  long long kc_ps, kc_ts, kc_hs, vc_ps, vc_ts, vc_hs;
  long long n_slots;
  int n_tokens, H, HK, D, pairs, adjacent, page, tile;
  double turns[ROPE_MAX_PAIRS];           // turns per position of each pair: frequency / 2 pi
  unsigned char axis[ROPE_MAX_PAIRS];
};

template <class T, int V> struct alignas(sizeof(T) * V) RopeVec { T e[V]; };

__device__ __forceinline__ float rope_load(float x) { return x; }
__device__ __forceinline__ float rope_load(__half x) { return __half2float(x); }
__device__ __forceinline__ float rope_load(__nv_bfloat16 x) { return __bfloat162float(x); }
template <class T> __device__ __forceinline__ T rope_store(float x);
template <> __device__ __forceinline__ float rope_store<float>(float x) { return x; }
template <> __device__ __forceinline__ __half rope_store<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 rope_store<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// (x, y) -> (x cos a - y sin a, y cos a + x sin a) with a = position * frequency, for every pair of every query and key head of
// a token; values go to the cache as they are.  One pass over the rows: nothing but them moves, so memory bounds it.
// The angle is reduced in 64 bits: at position 10^6 a 32-bit product is off by 0.06 radians.  What is left of it, at most
// half a turn, goes into sincospif in 32 bits (2^-24 relative).  Rotated values are rounded once, to the type of the rows.
// A CTA takes `tile` tokens (and one of gridDim.y shares of their heads): the angles of its tokens go to shared memory once, for all heads.
// A thread keeps one place in the head (V elements and the V they are paired with: 16 bytes each) over the heads it takes.
template <class T, int V>
__global__ void __launch_bounds__(256) rope_store_rows(const __grid_constant__ RopeParams p) {
  extern __shared__ float2 turn_s[];       // [tile][pairs]
  ptx::pdl_launch();
  ptx::pdl_wait();
  const int t0 = blockIdx.x * p.tile;
  const int nt = p.n_tokens - t0 < p.tile ? p.n_tokens - t0 : p.tile;
  for (int i = threadIdx.x; i < nt * p.pairs; i += 256) {
    const int t = i / p.pairs, j = i - t * p.pairs;
    const double x = p.turns[j] * static_cast<double>(p.positions[p.axis[j] * p.pos_stride + t0 + t]);
    float s, c;
    sincospif(2.f * static_cast<float>(x - rint(x)), &s, &c);
    turn_s[i] = make_float2(c, s);
  }
  __syncthreads();
  using Vec = RopeVec<T, V>;
  // units of a query or key head: `ru` of two vectors that are rotated, then single vectors that are copied
  const int ru = p.pairs / V, rot = 2 * p.pairs, cu = (p.D - rot) / V, U = ru + cu;
  const int HT = p.H + p.HK, rows = nt * HT;
  if (U > 0) {
    const int unit = threadIdx.x % U, per = 256 / U, slot = threadIdx.x / U;
    if (slot < per) {
      for (int i = blockIdx.y * per + slot; i < rows; i += per * gridDim.y) {
        const int t = i / HT, h = i - t * HT;
        const long long row = t0 + t;
        const T* src; T* dst; T* dst2 = nullptr;
        if (h < p.H) {
          src = static_cast<const T*>(p.q) + row * p.q_ts + h * p.q_hs;
          dst = static_cast<T*>(p.q_out) + row * p.qo_ts + h * p.qo_hs;
        } else {
          src = static_cast<const T*>(p.k) + row * p.k_ts + (h - p.H) * p.k_hs;
          dst = p.k_out ? static_cast<T*>(p.k_out) + row * p.ko_ts + (h - p.H) * p.ko_hs : nullptr;
          if (p.kc) {
            const long long s = p.slots[row];
            if (s >= 0 && s < p.n_slots) dst2 = static_cast<T*>(p.kc) + (s / p.page) * p.kc_ps + (s % p.page) * p.kc_ts + (h - p.H) * p.kc_hs;
          }
        }
        if (unit < ru) {
          const int a = p.adjacent ? unit * 2 * V : unit * V, b = p.adjacent ? a + V : a + p.pairs;
          Vec x = *reinterpret_cast<const Vec*>(src + a), y = *reinterpret_cast<const Vec*>(src + b);
          const float2* cs = turn_s + t * p.pairs + unit * V;
          if (p.adjacent) {
            if constexpr (V == 1) {
              const float u = rope_load(x.e[0]), w = rope_load(y.e[0]);
              x.e[0] = rope_store<T>(u * cs[0].x - w * cs[0].y);
              y.e[0] = rope_store<T>(w * cs[0].x + u * cs[0].y);
            } else {
#pragma unroll
              for (int e = 0; e < V / 2; ++e) {
                float u = rope_load(x.e[2 * e]), w = rope_load(x.e[2 * e + 1]);
                float2 c = cs[e];
                x.e[2 * e] = rope_store<T>(u * c.x - w * c.y);
                x.e[2 * e + 1] = rope_store<T>(w * c.x + u * c.y);
                u = rope_load(y.e[2 * e]); w = rope_load(y.e[2 * e + 1]);
                c = cs[V / 2 + e];
                y.e[2 * e] = rope_store<T>(u * c.x - w * c.y);
                y.e[2 * e + 1] = rope_store<T>(w * c.x + u * c.y);
              }
            }
          } else {
#pragma unroll
            for (int e = 0; e < V; ++e) {
              const float u = rope_load(x.e[e]), w = rope_load(y.e[e]);
              x.e[e] = rope_store<T>(u * cs[e].x - w * cs[e].y);
              y.e[e] = rope_store<T>(w * cs[e].x + u * cs[e].y);
            }
          }
          if (dst) { *reinterpret_cast<Vec*>(dst + a) = x; *reinterpret_cast<Vec*>(dst + b) = y; }
          if (dst2) { *reinterpret_cast<Vec*>(dst2 + a) = x; *reinterpret_cast<Vec*>(dst2 + b) = y; }
        } else {
          const int a = rot + (unit - ru) * V;
          const Vec x = *reinterpret_cast<const Vec*>(src + a);
          if (dst) *reinterpret_cast<Vec*>(dst + a) = x;
          if (dst2) *reinterpret_cast<Vec*>(dst2 + a) = x;
        }
      }
    }
  }
  if (!p.vc && !p.kc) return;
  // values, and what the slots say
  const int vu = p.D / V;
  for (int i = blockIdx.y * 256 + threadIdx.x; i < nt * p.HK * vu; i += 256 * gridDim.y) {
    const int r = i / vu, u = i - r * vu, t = r / p.HK, h = r - t * p.HK;
    const long long row = t0 + t, s = p.slots[row];
    if (s >= p.n_slots && p.status && u == 0 && h == 0) atomicOr(p.status, SERVE_BAD_PAGE);
    if (!p.vc || s < 0 || s >= p.n_slots) continue;
    const Vec x = *reinterpret_cast<const Vec*>(static_cast<const T*>(p.v) + row * p.v_ts + h * p.v_hs + u * V);
    *reinterpret_cast<Vec*>(static_cast<T*>(p.vc) + (s / p.page) * p.vc_ps + (s % p.page) * p.vc_ts + h * p.vc_hs + u * V) = x;
  }
}

}  // namespace k
}  // namespace sod2
