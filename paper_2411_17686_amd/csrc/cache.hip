// Pages of the decoder's key / value cache: handing them out, sharing, rewriting and giving them back, and the blocks
// of 8 bits that hold the tokens.
//
// A call that hands out pages is two launches: one workgroup decides (a thread per sequence: what it needs, prefix sums
// over the call, the free pages with the lowest numbers found by a scan of `refs`), then the chip moves the bytes.
// Nothing is decided by the order in which workgroups run: every result is the same in every run.
#include <algorithm>

#include "cache.hpp"

namespace ficoco {
namespace {

constexpr int kMaxPlanThreads = kMaxCall;
constexpr int kNone = 0x7fffffff;

struct PlanLds {
  int owner[kMaxSlots];      // the first entry of the call that names a slot
  int end[kMaxCall];         // pages needed by entries 0 .. b
  int scratch[kMaxPlanThreads / kWave];
  int served;
};

__device__ __forceinline__ bool slot_ok(const ficoco_cache& c, int s) { return s >= 0 && s < c.n_seqs; }
__device__ __forceinline__ bool page_ok(const ficoco_cache& c, int p) { return p >= 0 && p < c.n_pages; }
__device__ __forceinline__ int pages_of(const ficoco_cache& c, int64_t tokens) { return (int)((tokens + c.page_size - 1) / c.page_size); }

// owner[s] = the first entry b of the call with slot(b) == s
template <int NT, typename F>
__device__ __forceinline__ void find_owners(const ficoco_cache& c, PlanLds& l, int n, F slot) {
  for (int i = threadIdx.x; i < c.n_seqs; i += NT) l.owner[i] = kNone;
  if (threadIdx.x == 0) l.served = 0;
  __syncthreads();
  if ((int)threadIdx.x < n) {
    const int s = slot(threadIdx.x);
    if (slot_ok(c, s)) atomicMin(&l.owner[s], (int)threadIdx.x);
  }
  __syncthreads();
}

// Eight refs of a thread, page i0 on: their free ones as a bit mask.
__device__ __forceinline__ int free_mask(const ficoco_cache& c, int i0) {
  int m = 0;
  if (i0 + 8 <= c.n_pages) {
    int r[8];
    __builtin_memcpy(r, c.refs + i0, 32);
#pragma unroll
    for (int j = 0; j < 8; ++j) m |= (r[j] == 0) << j;
  } else {
    for (int j = 0; i0 + j < c.n_pages; ++j) m |= (c.refs[i0 + j] == 0) << j;
  }
  return m;
}

// `first_mask`: free_mask() of this thread's pages among the first 8 * NT, read ahead of the rest of the plan.
// Every entry's thread (tid < n, others need = 0) asks for `need` pages; take(b, k, page) gets page k of entry b, the free pages
// in ascending order.  Entries are served in order as long as the pages last.  Returns whether this thread's entry is.
template <int NT, typename F>
__device__ __forceinline__ bool hand_out(const ficoco_cache& c, PlanLds& l, int n, int need, int first_mask, F take) {
  int total;
  const int end = block_scan_inclusive(need, l.scratch, &total);
  if ((int)threadIdx.x < n) l.end[threadIdx.x] = end;
  if (total == 0) return true;                            // (uniform)
  int n_free;
  const int first_rank = block_scan_inclusive(__popc(first_mask), l.scratch, &n_free) - __popc(first_mask), first_free = n_free;
  for (int base = 8 * NT; base < c.n_pages && n_free < total; base += 8 * NT) {
    int t;
    (void)block_scan_inclusive(__popc(free_mask(c, base + 8 * (int)threadIdx.x)), l.scratch, &t);
    n_free += t;
  }
  const bool ok = need == 0 || end <= n_free;
  if (need > 0 && ok) atomicMax(&l.served, end);
  __syncthreads();
  const int give = l.served;
  int given = 0;
  for (int base = 0; base < c.n_pages && given < give; base += 8 * NT) {
    const int i0 = base + 8 * (int)threadIdx.x, m = base == 0 ? first_mask : free_mask(c, i0);
    int t = first_free, r = first_rank;
    if (base > 0) r = given + block_scan_inclusive(__popc(m), l.scratch, &t) - __popc(m);
    for (int j = 0; j < 8; ++j) {
      if (!(m >> j & 1)) continue;
      if (r < give) {
        int lo = 0, hi = n - 1;                           // first entry whose end lies behind r
        while (lo < hi) {
          const int mid = (lo + hi) / 2;
          if (l.end[mid] > r) hi = mid; else lo = mid + 1;
        }
        take(lo, r - (lo ? l.end[lo - 1] : 0), i0 + j);
      }
      ++r;
    }
    given += t;
  }
  return ok;
}

// One workgroup: bound by its chain of scans.  48 sequences of one token 3.6 us on average, 8 of 2979 5.5.
template <int NT>
__global__ __launch_bounds__(NT) void cache_reserve_kernel(ficoco_cache c, int n, const int32_t* __restrict__ seq,
                                                                     const int32_t* __restrict__ n_new, int n_each, int32_t* __restrict__ start) {
  __shared__ PlanLds l;
  __shared__ int slot[kMaxCall], have[kMaxCall];
  const int b = threadIdx.x, first_mask = free_mask(c, 8 * (int)threadIdx.x);
  auto slot_of = [&](int i) { return seq ? seq[i] : i; };
  find_owners<NT>(c, l, n, slot_of);
  int need = 0, len = 0, add = 0;
  bool ok = false;
  if (b < n) {
    const int s = slot_of(b);
    add = n_new ? n_new[b] : n_each;
    ok = slot_ok(c, s) && l.owner[s] == b && add >= 0;
    if (ok) {
      len = c.len[s];
      ok = len >= 0 && (int64_t)len + add <= (int64_t)c.max_pages * c.page_size;
    }
    if (ok) {
      have[b] = pages_of(c, len);
      need = pages_of(c, (int64_t)len + add) - have[b];
    }
    slot[b] = s;
  }
  __syncthreads();
  const bool served = hand_out<NT>(c, l, n, need, first_mask, [&](int e, int k, int page) {
    c.table[(int64_t)slot[e] * c.max_pages + have[e] + k] = page;
    c.refs[page] = 1;
  });
  if (b < n) {
    if (ok && served) c.len[slot[b]] = len + add;
    start[b] = ok && served ? len : -1;
  }
}

// ---- tokens in and out of blocks ----------------------------------------------------------------------------
__device__ __forceinline__ void load8f(const bf16_t* p, float (&x)[8]) {
  uint4 r;
  __builtin_memcpy(&r, p, 16);
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8f(const float* p, float (&x)[8]) { __builtin_memcpy(x, p, 32); }
__device__ __forceinline__ void store8f(float* p, const float (&x)[8]) { __builtin_memcpy(p, x, 32); }
__device__ __forceinline__ void store8f(bf16_t* p, const float (&x)[8]) {      // (exact: three mantissa bits)
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (__float_as_uint(x[2 * i]) >> 16) | (__float_as_uint(x[2 * i + 1]) & 0xffff0000u);
  __builtin_memcpy(p, w, 16);
}

struct TokenSide {       // K or V of a call
  const void* x;
  int64_t sb, sh, sn;
  uint8_t* pool;
  uint8_t* exps;
};

__device__ __forceinline__ float block_max(float v, float* scratch) {
  v = wave_reduce(v, [](float a, float b) { return fmaxf(a, b); });
  const int nw = blockDim.x / kWave;
  __syncthreads();
  if (threadIdx.x % kWave == 0) scratch[threadIdx.x / kWave] = v;
  __syncthreads();
  for (int w = 0; w < nw; ++w) v = fmaxf(v, scratch[w]);
  return v;
}

// What a call writes to one sequence: positions [first, stop) of slot `slot`, none where first < 0.
struct Span { int slot, first; int64_t stop; };
__device__ __forceinline__ Span span_of(const ficoco_cache& c, int b, int n_max, const int32_t* seq, const int32_t* start, const int32_t* n_new) {
  const int s = seq ? seq[b] : b, first = start[b];
  int n = n_new ? n_new[b] : n_max;
  n = n < n_max ? n : n_max;
  return slot_ok(c, s) && first >= 0 && n > 0 ? Span{s, first, (int64_t)first + n} : Span{0, -1, -1};
}

// One workgroup per touched page, head, sequence and K / V: the new tokens' largest magnitude, then all of them.  GPT: groups of
// sixteen values a thread.  The tokens are on their way before the page is looked up.
//
// Bound by memory (8 prompts of up to 2979 tokens, 8 heads of 128, bfloat16, 107 MB: 26 to 28 us, 3.9 to 4.1 TB/s).
template <typename T, int GPT>
__global__ __launch_bounds__(kMoveThreads) void cache_append_kernel(ficoco_cache c, int64_t layer_pages, TokenSide ks, TokenSide vs, int n_max,
                                                                    const int32_t* __restrict__ seq, const int32_t* __restrict__ start,
                                                                    const int32_t* __restrict__ n_new) {
  __shared__ float scratch[kMoveThreads / kWave];
  const int b = blockIdx.z >> 1, h = blockIdx.y, shift = __builtin_ctz(c.page_size), P = 1 << shift, row_shift = __builtin_ctz(c.d_head / 16);
  const TokenSide& side = blockIdx.z & 1 ? vs : ks;
  const Span sp = span_of(c, b, n_max, seq, start, n_new);
  const int64_t at = (sp.first >> shift) + (int64_t)blockIdx.x, pos0 = at << shift;
  if (sp.first < 0 || pos0 >= sp.stop || at >= c.max_pages) return;
  const T* x = (const T*)side.x + (int64_t)b * side.sb + (int64_t)h * side.sh;
  float v[GPT][2][8];
#pragma unroll
  for (int j = 0; j < GPT; ++j) {
    const int g = threadIdx.x + j * kMoveThreads, row = g >> row_shift;
    const int64_t pos = pos0 + row;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[j][0][i] = v[j][1][i] = 0.0f;
    if (row < P && pos >= sp.first && pos < sp.stop) {
      const T* from = x + (pos - sp.first) * side.sn + (g & ((1 << row_shift) - 1)) * 16;
      load8f(from, v[j][0]);
      load8f(from + 8, v[j][1]);
    }
  }
  const int page = c.table[(int64_t)sp.slot * c.max_pages + at];
  if (!page_ok(c, page)) return;
  const int64_t block = (layer_pages + page) * c.heads + h;
  uint8_t* pool = side.pool + block * P * c.d_head;
  const int old = pos0 < sp.first ? side.exps[block] : 0;
  float top = 0.0f;
#pragma unroll
  for (int j = 0; j < GPT; ++j) {
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, finite_magnitude(v[j][i / 8][i % 8]));
  }
  int e = block_exponent(block_max(top, scratch));
  e = e > old ? e : old;
  const float inv = exp_inverse(e);
  if (e == kExpTop) {                                       // (uniform)
#pragma unroll
    for (int j = 0; j < GPT; ++j) {
      keep_finite(v[j][0]);
      keep_finite(v[j][1]);
    }
  }
  __syncthreads();                                         // the byte is read before it is written
#pragma unroll
  for (int j = 0; j < GPT; ++j) {
    const int g = threadIdx.x + j * kMoveThreads, row = g >> row_shift;
    const int64_t pos = pos0 + row;
    if (row >= P || pos >= sp.stop) continue;
    uint4* to = (uint4*)(pool + (int64_t)g * 16);
    if (pos < sp.first) {
      if (e == old) continue;
      const uint4 q = *to;
      from_e4m3(uint2{q.x, q.y}, exp_scale(old), v[j][0]);
      from_e4m3(uint2{q.z, q.w}, exp_scale(old), v[j][1]);
    }
    const uint2 q0 = to_e4m3(v[j][0], inv), q1 = to_e4m3(v[j][1], inv);
    *to = uint4{q0.x, q0.y, q1.x, q1.y};
  }
  if (threadIdx.x == 0) side.exps[block] = (uint8_t)e;
}

// One token a sequence (a decoder's step): eight values a lane, so a row of 16 lanes (heads of 64: half of one) holds the token of one head, K or V.
// Older tokens of the page are touched only where the new one raises the exponent: one by one, a trip to memory each, by the lanes of that block.  48 sequences, 32
// heads, pages of 64: 3.3 us where no exponent rises, a launch and its trips (with the kernel above, a workgroup per block, 8.5 us).  A decoder's new tokens
// raise some block in most steps: 256 steps with normal keys and values 19 us at the median, 29 for a tenth of them, 34 at most; every block raised by
// the last token of a page of 128 57 us.
template <typename T, int D>
__global__ __launch_bounds__(kMoveThreads) void cache_append_token_kernel(ficoco_cache c, int64_t layer_pages, TokenSide ks, TokenSide vs, int items,
                                                                          const int32_t* __restrict__ seq, const int32_t* __restrict__ start,
                                                                          const int32_t* __restrict__ n_new) {
  constexpr int L = D / 8;
  const int item = (blockIdx.x * kMoveThreads + threadIdx.x) / L, g = threadIdx.x % L;      // V behind K, heads behind sequences
  const bool there = item < items;
  const int i = there ? item : items - 1, b = i / (2 * c.heads), h = i / 2 % c.heads;
  const TokenSide& side = i & 1 ? vs : ks;
  const Span sp = span_of(c, b, 1, seq, start, n_new);
  const int shift = __builtin_ctz(c.page_size), slot = sp.first & ((1 << shift) - 1), at = sp.first >> shift;
  float v[8] = {};
  if (sp.first >= 0) load8f((const T*)side.x + (int64_t)b * side.sb + (int64_t)h * side.sh + 8 * g, v);
  const int page = sp.first >= 0 && at < c.max_pages ? c.table[(int64_t)sp.slot * c.max_pages + at] : -1;
  const bool ok = there && page_ok(c, page);
  const int64_t block = ok ? (layer_pages + page) * c.heads + h : 0;
  const int old = ok && slot > 0 ? side.exps[block] : 0;
  float top = 0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) top = fmaxf(top, finite_magnitude(v[j]));
  top = fmaxf(top, dpp_move<0xB1>(top));
  top = fmaxf(top, dpp_move<0x4E>(top));
  top = fmaxf(top, dpp_move<0x141>(top));
  if constexpr (L == 16) top = fmaxf(top, dpp_move<0x140>(top));
  if (!ok) return;
  int e = block_exponent(top);
  e = e > old ? e : old;
  uint8_t* pool = side.pool + (block << shift) * D + 8 * g;
  if (e == kExpTop) keep_finite(v);
  const uint2 q = to_e4m3(v, exp_inverse(e));
  *(uint2*)(pool + slot * D) = q;
  if (e != old && slot > 0) {
    for (int r = 0; r < slot; ++r) {
      float x[8];
      from_e4m3(*(const uint2*)(pool + r * D), exp_scale(old), x);
      *(uint2*)(pool + r * D) = to_e4m3(x, exp_inverse(e));
    }
  }
  if (e != old && g == 0) side.exps[block] = (uint8_t)e;   // (the rows of a wavefront read the byte in one instruction, before)
}

// Eight values a lane.  Bound by memory (the same prompts into single precision, 178 MB: 30 us, 6.0 TB/s).
template <typename T>
__global__ __launch_bounds__(kMoveThreads) void cache_read_kernel(ficoco_cache c, int64_t layer_pages, TokenSide ks, TokenSide vs, int n_max,
                                                                  const int32_t* __restrict__ seq, const int32_t* __restrict__ start,
                                                                  const int32_t* __restrict__ n_new) {
  const int b = blockIdx.z >> 1, h = blockIdx.y, shift = __builtin_ctz(c.page_size), per_row = c.d_head / 8;
  const TokenSide& side = blockIdx.z & 1 ? vs : ks;
  if (!side.x) return;
  const int s = seq ? seq[b] : b, first = start ? start[b] : 0;
  int n = n_new ? n_new[b] : n_max;
  n = n < n_max ? n : n_max;
  if (first < 0) return;
  const int g = threadIdx.x % per_row;
  const int t = (int)(blockIdx.x * (kMoveThreads / per_row) + threadIdx.x / per_row);
  if (t >= n) return;
  const int64_t pos = (int64_t)first + t, at = pos >> shift;
  float v[8] = {};
  const int page = slot_ok(c, s) && at < c.max_pages ? c.table[(int64_t)s * c.max_pages + at] : -1;
  if (page_ok(c, page)) {
    const int64_t block = (layer_pages + page) * c.heads + h;
    uint2 q;
    __builtin_memcpy(&q, side.pool + ((block << shift) + (pos & (c.page_size - 1))) * c.d_head + g * 8, 8);
    from_e4m3(q, exp_scale(side.exps[block]), v);
  }
  store8f((T*)const_cast<void*>(side.x) + (int64_t)b * side.sb + (int64_t)h * side.sh + (int64_t)t * side.sn + g * 8, v);
}

// ---- fork -------------------------------------------------------------------------------------------------------
template <int NT>
__global__ __launch_bounds__(NT) void cache_fork_kernel(ficoco_cache c, int n, const int32_t* __restrict__ src, const int32_t* __restrict__ dst,
                                                                  int whole, int32_t* __restrict__ done) {
  __shared__ PlanLds l;
  __shared__ int to[kMaxCall], shared[kMaxCall];
  const int b = threadIdx.x, first_mask = free_mask(c, 8 * (int)threadIdx.x);
  find_owners<NT>(c, l, n, [&](int i) { return dst[i]; });
  int need = 0, len = 0;
  bool ok = false;
  if (b < n) {
    const int s = src[b], d = dst[b];
    ok = slot_ok(c, s) && slot_ok(c, d) && l.owner[d] == b && l.owner[s] == kNone;
    if (ok) {
      len = c.len[s];
      ok = c.len[d] == 0 && len >= 0 && pages_of(c, len) <= c.max_pages;
    }
    to[b] = d;
    shared[b] = ok && !whole ? len / c.page_size : 0;
    need = ok ? pages_of(c, len) - shared[b] : 0;
  }
  __syncthreads();
  const bool served = ok & hand_out<NT>(c, l, n, need, first_mask, [&](int e, int k, int page) {
    c.table[(int64_t)to[e] * c.max_pages + shared[e] + k] = page;
    c.refs[page] = 1;
  });
  if (b < n) {
    if (served) c.len[to[b]] = len;
    done[b] = served;
  }
}

// Whole pages of all layers, as they are.  Workgroups of one sequence, layer, head and K / V walk its copied pages; one of a sequence's has its
// shared ones entered (by the plan's one workgroup: 128 sequences of ten pages 27 us instead of 22).  Where src has no page to copy, dst gets none: the one
// that the plan entered is given back by the workgroups of the first layer and head (the others have no use for the entry).  Whole copies are bound by memory:
// 4 sequences of 2979 tokens, 16 layers of 8 heads, 788 MB: 157 us, 5.0 TB/s.
__global__ __launch_bounds__(kMoveThreads) void cache_copy_kernel(ficoco_cache c, const int32_t* __restrict__ src, const int32_t* __restrict__ dst,
                                                                  int whole, const int32_t* __restrict__ done) {
  const int b = blockIdx.z >> 1;
  if (!done[b]) return;
  const int from = src[b], to = dst[b], len = c.len[to], pages = pages_of(c, len);
  if (!whole && (blockIdx.x | blockIdx.y | blockIdx.z & 1) == 0) {
    for (int i = threadIdx.x; i < len / c.page_size; i += kMoveThreads) {
      const int page = c.table[(int64_t)from * c.max_pages + i];
      c.table[(int64_t)to * c.max_pages + i] = page;
      if (page_ok(c, page)) atomicAdd(&c.refs[page], 1);
    }
  }
  const int layer = blockIdx.y / c.heads, h = blockIdx.y % c.heads;
  uint8_t* pool = (uint8_t*)(blockIdx.z & 1 ? c.v : c.k);
  uint8_t* exps = blockIdx.z & 1 ? c.v_exp : c.k_exp;
  const int block_bytes = c.page_size * c.d_head;
  for (int i = (whole ? 0 : len / c.page_size) + blockIdx.x; i < pages; i += gridDim.x) {
    int32_t* at = c.table + (int64_t)to * c.max_pages + i;
    const int p = c.table[(int64_t)from * c.max_pages + i], q = *at;
    if (!page_ok(c, p) || !page_ok(c, q)) {
      if (!page_ok(c, p) && page_ok(c, q) && (blockIdx.y | blockIdx.z & 1) == 0 && threadIdx.x == 0) {
        c.refs[q] = 0;
        *at = -1;
      }
      continue;
    }
    const int64_t bp = ((int64_t)layer * c.n_pages + p) * c.heads + h, bq = ((int64_t)layer * c.n_pages + q) * c.heads + h;
    const uint4* x = (const uint4*)(pool + bp * block_bytes);
    uint4* y = (uint4*)(pool + bq * block_bytes);
    for (int j = threadIdx.x; j < block_bytes / 16; j += kMoveThreads) y[j] = x[j];
    if (threadIdx.x == 0) exps[bq] = exps[bp];
  }
}

// ---- compact ------------------------------------------------------------------------------------------------------
struct CompactMeta { int first, pages, tokens, had; };      // pages kept, pages and tokens now, pages before (0: not served)

template <int NT>
__global__ __launch_bounds__(NT) void cache_compact_plan_kernel(ficoco_cache c, int n, const int32_t* __restrict__ src, const int32_t* __restrict__ dst,
                                                                          int vis_begin, int N, int n_keep, const int32_t* __restrict__ keep_idx,
                                                                          int32_t* __restrict__ done, CompactMeta* __restrict__ meta, int32_t* __restrict__ rows) {
  __shared__ PlanLds l;
  __shared__ int from[kMaxCall], to[kMaxCall], moved[kMaxCall], first[kMaxCall], had[kMaxCall];
  const int b = threadIdx.x, lane = threadIdx.x % kWave, first_mask = free_mask(c, 8 * (int)threadIdx.x);
  find_owners<NT>(c, l, n, [&](int i) { return dst[i]; });
  // the first preserved token that moves: its rank among the preserved ones
  for (int e = threadIdx.x / kWave; e < n; e += NT / kWave) {
    const int32_t* k = keep_idx + (int64_t)e * n_keep;
    int at = n_keep;
    for (int i0 = 0; i0 < n_keep; i0 += kWave) {
      const int i = i0 + lane;
      const uint64_t m = __ballot(i < n_keep && k[i] != i);
      if (m) {
        at = i0 + __ffsll((long long)m) - 1;
        break;
      }
    }
    if (lane == 0) moved[e] = at;
  }
  __syncthreads();
  int need = 0, new_len = 0, now = 0;
  bool ok = false;
  if (b < n) {
    const int s = src[b], d = dst[b];
    ok = slot_ok(c, s) && slot_ok(c, d) && l.owner[d] == b && (s == d || l.owner[s] == kNone);
    int f = 0, pages = 0, have = 0;
    if (ok) {
      const int len = c.len[s];
      have = pages_of(c, len > 0 ? len : 0);
      ok = (int64_t)len >= (int64_t)vis_begin + N && have <= c.max_pages && (s == d || c.len[d] == 0);
      new_len = len - (N - n_keep);
      pages = pages_of(c, new_len > 0 ? new_len : 0);
      const int change = moved[b] < n_keep ? vis_begin + moved[b] : n_keep == N ? new_len : vis_begin + n_keep;
      f = s == d && moved[b] == n_keep && n_keep == N ? pages : change / c.page_size;
    }
    from[b] = s;
    to[b] = d;
    first[b] = ok ? f : 0;
    had[b] = ok ? have : 0;
    now = pages;
    need = ok ? pages - f : 0;
  }
  __syncthreads();
  // A token that has no page cannot move.  Whether page i of entry e, which has none, holds one that is preserved (keep_idx ascends):
  auto in_use = [&](int e, int i) {
    const int64_t lo = (int64_t)i * c.page_size - vis_begin, hi = min(lo + c.page_size, (int64_t)c.len[from[e]] - vis_begin);
    if (lo < 0 || hi > N) return true;
    const int32_t* k = keep_idx + (int64_t)e * n_keep;
    int x = 0, y = n_keep;
    while (x < y) {
      const int mid = (x + y) / 2;
      if (k[mid] < lo) x = mid + 1; else y = mid;
    }
    return x < n_keep && k[x] < hi;
  };
  for (int e = threadIdx.x / kWave; e < n; e += NT / kWave) {
    bool stuck = false;
    for (int i = lane; i < had[e]; i += kWave) {
      const int page = c.table[(int64_t)from[e] * c.max_pages + i];
      rows[(int64_t)e * c.max_pages + i] = page;
      if (!page_ok(c, page) && i >= first[e]) stuck |= in_use(e, i);
    }
    stuck = __any(stuck);
    if (lane == 0) moved[e] = stuck;                       // (its value so far has served)
  }
  __syncthreads();                                         // the rows are saved before new pages go into them
  if (b < n && moved[b]) {
    ok = false;
    need = 0;
  }
  const bool served = ok & hand_out<NT>(c, l, n, need, first_mask, [&](int e, int k, int page) {
    c.table[(int64_t)to[e] * c.max_pages + first[e] + k] = page;
    c.refs[page] = 1;
  });
  if (b < n) {
    if (served) c.len[to[b]] = new_len;
    done[b] = served;
    meta[b] = CompactMeta{first[b], served ? now : 0, new_len, served ? had[b] : 0};
  }
}

// The largest magnitude of 16 E4M3 numbers that is not NaN, in units of their scale.  Bytes without their sign ascend with the magnitude;
// one added, NaN (127) becomes 0 and the others 1 .. 127.
__device__ __forceinline__ float largest_e4m3(const uint4& q) {
  typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
  u16x2_t m = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t y = (w[i] & 0x7f7f7f7fu) + 0x01010101u;
    m = __builtin_elementwise_max(m, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, y & 0x007f007fu), __builtin_bit_cast(u16x2_t, y >> 8 & 0x007f007fu)));
  }
  const int top = m.x > m.y ? m.x : m.y;
  return top > 0 ? __builtin_amdgcn_cvt_f32_fp8(top - 1, 0) : 0.0f;
}
// 16 numbers from one scale to another, as to_e4m3() has them.
__device__ __forceinline__ uint4 rescale_e4m3(const uint4& q, int from, int to) {
  const int d = from - to + kExpBias;
  const float f = exp_scale(d < 1 ? 1 : d < 254 ? d : 254);      // (beyond: nothing is left, or there is nothing but zeros)
  float x[8];
  from_e4m3(uint2{q.x, q.y}, f, x);
  const uint2 a = to_e4m3(x, 1.0f);
  from_e4m3(uint2{q.z, q.w}, f, x);
  const uint2 b = to_e4m3(x, 1.0f);
  return uint4{a.x, a.y, b.x, b.y};
}

// The new pages of one sequence: where a page's tokens come from is found once, in LDS, and holds for every layer, head, K and V;
// then a wavefront, or a TEAM of them, takes a block (one page of one head, K or V) at a time, its 16-byte pieces in registers.
// Blocks whose exponent stays keep their bytes.  The pages read are not among those written: they are held until the plan of a later call.
//
// Bound by memory (five crops, 4 sequences of 2979 tokens to 739, 16 layers of 8 heads, 194 MB: 45 us, 4.4 TB/s).  A workgroup that took the blocks of one
// head, one after the other, found every block's rows anew, four loads one behind the other: 103 us.  The next block's pieces on their way in registers, too,
// cost wavefronts: 3 us more here.
template <int NG, int TEAM>
__global__ __launch_bounds__(kMoveThreads) void cache_compact_kernel(ficoco_cache c, int layer_begin, int blocks, int per_wg, int vis_begin, int N, int n_keep,
                                                                     const int32_t* __restrict__ src, const int32_t* __restrict__ dst, const int32_t* __restrict__ keep_idx,
                                                                     const CompactMeta* __restrict__ meta, const int32_t* __restrict__ rows) {
  __shared__ int from_page[128], from_slot[128];
  __shared__ float tops[kMoveThreads / kWave];
  constexpr int TEAMS = kMoveThreads / kWave / TEAM;
  const int b = blockIdx.z;
  const CompactMeta m = meta[b];
  const int shift = __builtin_ctz(c.page_size), P = 1 << shift, per_row = c.d_head / 16, block_bytes = P * c.d_head;
  const int lane = threadIdx.x % kWave, wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int end = min(blocks, (int)blockIdx.y * per_wg + per_wg);
  if ((blockIdx.x | blockIdx.y) == 0) {                    // the pages kept (shared) and those of before (given back)
    int32_t* row = c.table + (int64_t)dst[b] * c.max_pages;
    const bool in_place = src[b] == dst[b];
    for (int i = threadIdx.x; i < m.had; i += kMoveThreads) {
      const int old = rows[(int64_t)b * c.max_pages + i];
      if (i < m.first) {
        if (!in_place) {
          row[i] = old;
          if (page_ok(c, old)) atomicAdd(&c.refs[old], 1);
        }
      } else if (in_place) {
        if (page_ok(c, old)) atomicSub(&c.refs[old], 1);
        if (i >= m.pages) row[i] = -1;
      }
    }
  }
  for (int page_at = m.first + blockIdx.x; page_at < m.pages; page_at += gridDim.x) {
    const int page = c.table[(int64_t)dst[b] * c.max_pages + page_at];
    if ((int)threadIdx.x < P) {
      const int64_t r = ((int64_t)page_at << shift) + threadIdx.x;
      int p = -1;
      int64_t t = r;
      if (r < m.tokens) {
        if (r >= vis_begin + n_keep) {
          t = r + (N - n_keep);
        } else if (r >= vis_begin) {
          const int k = keep_idx[(int64_t)b * n_keep + (r - vis_begin)];
          t = vis_begin + (k < 0 ? 0 : k < N ? k : N - 1);
        }
        p = rows[(int64_t)b * c.max_pages + (t >> shift)];
        if (!page_ok(c, p)) p = -1;
      }
      from_page[threadIdx.x] = r < m.tokens ? p : -2;       // -1: zeros (keep_idx out of order alone), -2: behind the last token, left as it is
      from_slot[threadIdx.x] = (int)(t & (P - 1));
    }
    __syncthreads();
    if (page_ok(c, page)) {                                  // (uniform)
      struct Piece { uint4 q[NG]; int e[NG]; };
      // block i: V behind K, heads behind layers
      auto block_of = [&](int i, int p) { return ((int64_t)(layer_begin + i / 2 / c.heads) * c.n_pages + p) * c.heads + i / 2 % c.heads; };
      auto load = [&](Piece& x, int i) {
        const uint8_t* pool = (const uint8_t*)(i & 1 ? c.v : c.k);
        const uint8_t* exps = i & 1 ? c.v_exp : c.k_exp;
#pragma unroll
        for (int j = 0; j < NG; ++j) {
          const int g = lane + (wv % TEAM * NG + j) * kWave, row = g / per_row, p = from_page[row];
          x.q[j] = uint4{0, 0, 0, 0};
          x.e[j] = kExpMin;
          if (p >= 0) {
            const int64_t block = block_of(i, p);
            x.q[j] = *(const uint4*)(pool + block * block_bytes + from_slot[row] * c.d_head + g % per_row * 16);
            x.e[j] = exps[block];
          }
        }
      };
      auto put = [&](const Piece& x, int i, int e) {
        const int64_t block = block_of(i, page);
        uint8_t* pool = (uint8_t*)(i & 1 ? c.v : c.k) + block * block_bytes;
#pragma unroll
        for (int j = 0; j < NG; ++j) {
          const int g = lane + (wv % TEAM * NG + j) * kWave;
          if (from_page[g / per_row] == -2) continue;
          *(uint4*)(pool + (int64_t)g * 16) = x.e[j] == e ? x.q[j] : rescale_e4m3(x.q[j], x.e[j], e);
        }
        if (lane == 0 && wv % TEAM == 0) (i & 1 ? c.v_exp : c.k_exp)[block] = (uint8_t)e;
      };
      Piece x;
      for (int i0 = blockIdx.y * per_wg; i0 < end; i0 += TEAMS) {
        const int i = i0 + wv / TEAM;
        float top = 0.0f;
        if (i < end) {
          load(x, i);
#pragma unroll
          for (int j = 0; j < NG; ++j) top = fmaxf(top, largest_e4m3(x.q[j]) * exp_scale(x.e[j]));
          top = wave_reduce(top, [](float u, float v) { return fmaxf(u, v); });
        }
        if constexpr (TEAM > 1) {
          __syncthreads();
          if (lane == 0) tops[wv] = top;
          __syncthreads();
#pragma unroll
          for (int w = 0; w < TEAM; ++w) top = fmaxf(top, tops[wv / TEAM * TEAM + w]);
        }
        if (i < end) put(x, i, block_exponent(top));
      }
    }
    __syncthreads();
  }
}

// ---- free -----------------------------------------------------------------------------------------------------------
// A workgroup per entry; an entry of the table is taken out by one exchange, so a slot named twice gives its pages back once.
__global__ __launch_bounds__(kMoveThreads) void cache_free_kernel(ficoco_cache c, const int32_t* __restrict__ seq) {
  const int s = seq ? seq[blockIdx.x] : (int)blockIdx.x;
  if (!slot_ok(c, s)) return;
  for (int i = threadIdx.x; i < c.max_pages; i += kMoveThreads) {
    int32_t* at = c.table + (int64_t)s * c.max_pages + i;
    if (*at < 0) continue;
    const int page = atomicExch(at, -1);
    if (page_ok(c, page)) atomicSub(&c.refs[page], 1);
  }
  if (threadIdx.x == 0) c.len[s] = 0;
}

TokenSide side_of(const ficoco_tokens& t, const ficoco_cache& c, bool v) {
  return v ? TokenSide{t.V, t.v_stride_b, t.v_stride_h, t.v_stride_n, (uint8_t*)c.v, c.v_exp}
           : TokenSide{t.K, t.k_stride_b, t.k_stride_h, t.k_stride_n, (uint8_t*)c.k, c.k_exp};
}

// Whether a plan is made by 256 threads instead of 1024: pages that these see at one look, and no more entries than `most`.  Four wavefronts wait less for
// each other: one prompt shared by 8, 15.6 us instead of 16.6; by 128, 22.3 and 23.3.  Where a wavefront takes one entry after the other (compact), sixteen get
// on faster: 4 sequences 15.3 and 16.6, 8 17.7 and 18.5, 16 22.2 and 21.9, 64 45 and 38.
bool small_plan(const ficoco_cache& c, int n, int most = 256) { return n <= most && c.n_pages <= 8 * 256 && c.n_seqs <= 8 * 256; }

// Workgroups that walk the pages of one sequence, layer, head and K / V.
int page_walkers(const ficoco_cache& c, int64_t others) {
  const int64_t want = (8192 + others - 1) / others;
  return (int)(want < 1 ? 1 : want < c.max_pages ? want : c.max_pages);
}

template <int NG, int TEAM>
void launch_compact_pages(const ficoco_cache& c, dim3 grid, int layer_begin, int blocks, int per_wg, int vis_begin, int N, int n_keep, const int32_t* src, const int32_t* dst,
                          const int32_t* keep_idx, const CompactMeta* meta, const int32_t* rows, hipStream_t s) {
  hipLaunchKernelGGL((cache_compact_kernel<NG, TEAM>), grid, dim3(kMoveThreads), 0, s, c, layer_begin, blocks, per_wg, vis_begin, N, n_keep, src, dst, keep_idx, meta, rows);
}

template <typename T>
void append_groups(const ficoco_cache& c, int layer, const ficoco_tokens& t, hipStream_t s) {
  const TokenSide k = side_of(t, c, false), v = side_of(t, c, true);
  const int64_t lp = (int64_t)layer * c.n_pages;
  const int64_t items = (int64_t)2 * t.n * c.heads;
  if (t.n_max == 1 && items <= 0x7fffffff / 16) {
    const dim3 grid((unsigned)((items * (c.d_head / 8) + kMoveThreads - 1) / kMoveThreads));
    if (c.d_head == 128) hipLaunchKernelGGL((cache_append_token_kernel<T, 128>), grid, dim3(kMoveThreads), 0, s, c, lp, k, v, (int)items, t.seq, t.start, t.n_new);
    else hipLaunchKernelGGL((cache_append_token_kernel<T, 64>), grid, dim3(kMoveThreads), 0, s, c, lp, k, v, (int)items, t.seq, t.start, t.n_new);
    return;
  }
  const dim3 grid(append_pages(c, t.n_max), c.heads, 2 * t.n);
  const int groups = c.page_size * c.d_head / 16;
  // (no threads without tokens: 16 prompts of 1000, 4 heads of 64, pages of 16, written and read back 23 us with 256, 18 with 64)
  if (groups <= 256) hipLaunchKernelGGL((cache_append_kernel<T, 1>), grid, dim3(groups), 0, s, c, lp, k, v, t.n_max, t.seq, t.start, t.n_new);
  else if (groups <= 512) hipLaunchKernelGGL((cache_append_kernel<T, 2>), grid, dim3(kMoveThreads), 0, s, c, lp, k, v, t.n_max, t.seq, t.start, t.n_new);
  else hipLaunchKernelGGL((cache_append_kernel<T, 4>), grid, dim3(kMoveThreads), 0, s, c, lp, k, v, t.n_max, t.seq, t.start, t.n_new);
}

}  // namespace

void launch_cache_reserve(const ficoco_cache& c, int n, const int32_t* seq, const int32_t* n_new, int n_each, int32_t* start, hipStream_t s) {
  if (small_plan(c, n)) hipLaunchKernelGGL(cache_reserve_kernel<256>, dim3(1), dim3(256), 0, s, c, n, seq, n_new, n_each, start);
  else hipLaunchKernelGGL(cache_reserve_kernel<kMaxPlanThreads>, dim3(1), dim3(kMaxPlanThreads), 0, s, c, n, seq, n_new, n_each, start);
}

void launch_cache_append(const ficoco_cache& c, int layer, const ficoco_tokens& t, hipStream_t s) {
  if (t.dtype == FICOCO_BF16) append_groups<bf16_t>(c, layer, t, s); else append_groups<float>(c, layer, t, s);
}

void launch_cache_read(const ficoco_cache& c, int layer, const ficoco_tokens& t, hipStream_t s) {
  const int rows = kMoveThreads / (c.d_head / 8);
  const dim3 grid((t.n_max + rows - 1) / rows, c.heads, 2 * t.n);
  const TokenSide k = side_of(t, c, false), v = side_of(t, c, true);
  const int64_t lp = (int64_t)layer * c.n_pages;
  if (t.dtype == FICOCO_BF16) hipLaunchKernelGGL(cache_read_kernel<bf16_t>, grid, dim3(kMoveThreads), 0, s, c, lp, k, v, t.n_max, t.seq, t.start, t.n_new);
  else hipLaunchKernelGGL(cache_read_kernel<float>, grid, dim3(kMoveThreads), 0, s, c, lp, k, v, t.n_max, t.seq, t.start, t.n_new);
}

void launch_cache_fork(const ficoco_cache& c, int n, const int32_t* src, const int32_t* dst, bool whole, int32_t* done, hipStream_t s) {
  if (small_plan(c, n)) hipLaunchKernelGGL(cache_fork_kernel<256>, dim3(1), dim3(256), 0, s, c, n, src, dst, (int)whole, done);
  else hipLaunchKernelGGL(cache_fork_kernel<kMaxPlanThreads>, dim3(1), dim3(kMaxPlanThreads), 0, s, c, n, src, dst, (int)whole, done);
  const int walkers = whole ? page_walkers(c, (int64_t)c.layers * c.heads * n * 2) : 1;
  hipLaunchKernelGGL(cache_copy_kernel, dim3(walkers, c.layers * c.heads, 2 * n), dim3(kMoveThreads), 0, s, c, src, dst, (int)whole, done);
}

void launch_cache_compact(const ficoco_cache& c, int layer_begin, int n_layers, int n, const int32_t* src, const int32_t* dst, int vis_begin, int N,
                          int n_keep, const int32_t* keep_idx, int32_t* done, char* ws, hipStream_t s) {
  CompactMeta* meta = (CompactMeta*)ws;
  int32_t* rows = (int32_t*)(ws + (size_t)n * sizeof(CompactMeta));
  if (small_plan(c, n, 8)) hipLaunchKernelGGL(cache_compact_plan_kernel<256>, dim3(1), dim3(256), 0, s, c, n, src, dst, vis_begin, N, n_keep, keep_idx, done, meta, rows);
  else hipLaunchKernelGGL(cache_compact_plan_kernel<kMaxPlanThreads>, dim3(1), dim3(kMaxPlanThreads), 0, s, c, n, src, dst, vis_begin, N, n_keep, keep_idx, done, meta, rows);
  // A wavefront takes one block, four together where it has 16 KB (pages of 128 tokens, heads of 128; a wavefront each: 70 us instead of 60 for four
  // sequences of 2979 tokens, 92 and 81 for three that keep 1200).  Blocks below 4 KB are less work than finding their rows: up to eight of them in turn, fewer where the chip
  // would not be filled (1024 workgroups; a sequence's pages count as eight): pages of 16, heads of 64, 55 us by ones, 48 so.  Of 8 KB (five crops) two in turn 59.8, one 57.7.
  const int blocks = 2 * n_layers * c.heads, block_bytes = c.page_size * c.d_head, teams = block_bytes == 16384 ? 1 : kMoveThreads / kWave;
  const int64_t want = block_bytes >= 4096 ? 0 : (int64_t)blocks * n * 8 / 1024;
  const int per_wg = std::max((int)(want < teams ? teams : want < 8 * teams ? want / teams * teams : 8 * teams), (blocks + 32767) / 32768);
  const dim3 grid(c.max_pages < 64 ? c.max_pages : 64, n_layers == 0 ? 1 : (blocks + per_wg - 1) / per_wg, n);
  switch (block_bytes / 1024) {
    case 1: launch_compact_pages<1, 1>(c, grid, layer_begin, blocks, per_wg, vis_begin, N, n_keep, src, dst, keep_idx, meta, rows, s); break;
    case 2: launch_compact_pages<2, 1>(c, grid, layer_begin, blocks, per_wg, vis_begin, N, n_keep, src, dst, keep_idx, meta, rows, s); break;
    case 4: launch_compact_pages<4, 1>(c, grid, layer_begin, blocks, per_wg, vis_begin, N, n_keep, src, dst, keep_idx, meta, rows, s); break;
    case 8: launch_compact_pages<8, 1>(c, grid, layer_begin, blocks, per_wg, vis_begin, N, n_keep, src, dst, keep_idx, meta, rows, s); break;
    default: launch_compact_pages<4, 4>(c, grid, layer_begin, blocks, per_wg, vis_begin, N, n_keep, src, dst, keep_idx, meta, rows, s); break;
  }
}

void launch_cache_free(const ficoco_cache& c, int n, const int32_t* seq, hipStream_t s) {
  hipLaunchKernelGGL(cache_free_kernel, dim3(n), dim3(kMoveThreads), 0, s, c, seq);
}

}  // namespace ficoco
