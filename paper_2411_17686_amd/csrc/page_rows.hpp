// Attention over pages of 8 bits for many rows: the work of one workgroup (128 rows, some of the keys), wherever its rows come from.
#pragma once
#include "attend.hpp"

namespace ficoco {

constexpr int kStages = 4;                   // steps in LDS: one computed with (its values, the next one's keys), the others on their way
constexpr int kGroup = 16;                   // keys that certainly share a page
constexpr int kGroups = kTileKeys / kGroup;  // of a step
constexpr int kChunk = 64;                   // steps whose pages are looked up at once
constexpr int kHole = 1 << 16;               // (beside two exponent bytes) keys that would be seen have no page

typedef int i32x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2_t* lds_i32x2_t;

// Rows of keys and of values in LDS, as they are in the pages, 16-byte chunks; chunk c of a row lies at c ^ swizzle.  Sixteen
// rows of keys are read at one chunk, eight rows of values (keys 0 .. 3 and 8 .. 11, or 4 .. 7 and 12 .. 15 of a group) at two: these put either
// on all 64 banks.
template <int D> __device__ __forceinline__ int key_swizzle(int row) { return D == 128 ? row >> 1 & 7 : row >> 2 & 3; }
template <int D> __device__ __forceinline__ int value_swizzle(int row) { return D == 128 ? (row & 2) | (row >> 1 & 4) : row >> 2 & 2; }

// Arrays of their own, so that the compiler can tell loads into one from reads of another; what else a kernel has to do may use them too.
template <int D>
struct PageLds {
  template <int I>
  static __device__ __forceinline__ uint8_t* array() {
    __shared__ __align__(16) uint8_t x[kTileKeys * D];
    return x;
  }
  static __device__ __forceinline__ int2* meta() {
    __shared__ int2 x[2 * kChunk * kGroups];
    return x;
  }
};

// As tile_rows_kernel (tile_attn.hip): 128 rows a workgroup, 32 a wavefront, 64 keys a step, 32 x 32 x 16 products, a step's weights formed
// beside the products of the next step's logits.  Pages go straight into LDS as bytes, three steps ahead, and become bfloat16 (exactly, with
// their block's scale) in front of the products, in every wavefront: that costs 128 conversions of 2 ns a step and saves the registers and
// the second trip through LDS that a common conversion takes.
//
// Bound by the vector instructions beside the products: a step of a wavefront is 0.53 us of products and about as much of conversions, exponentials
// and sums, and takes 1.6 to 1.7 us beside another wavefront on its SIMD (workgroups of 54 steps 95 us at best).  Questions of 64 tokens behind 1251 .. 2400, 8 sequences, 32 heads on 8: 33 us (a third of it
// before the first step and after the last), 7 more for the join.  Weights are rounded to bfloat16 for the second product, as in few_rows() (few_rows.hpp).  Sixty-four rows a wavefront, one wavefront a SIMD, halve the conversions,
// but nothing then fills its waits for LDS and barriers: 57 us instead of 40 with the queries in LDS (73 without, for lack of registers), and with heads of 64, where nothing is
// short of registers, 102 instead of 69 behind 9600 tokens.
//
// tid: the thread.  A lane's row (lane % 32 of its wavefront's) has its queries at q and sees `sight`: rows_of() says both.  Keys of head h are those of blocks begin .. end - 1 and of `table`; lo, hi: first and last
// position of the wavefront's rows, keys: how many keys each of them has at least.  part_ms (the lane's, null for none): where maxima and sums of parts go; part(row, piece) and out(row, piece): the
// places of 16 bytes of row 0 .. 31 of the wavefront as floats, relative to the maximum, or as bfloat16, null for nowhere.
struct TileRow {
  const bf16_t* q;
  RowSight sight;
};
template <int D, typename Rows, typename Part, typename Out>
__device__ __forceinline__ void page_rows(const AttendArgs& a, int tid, int h, Rows rows_of, int lo, int hi, int keys, const int32_t* table,
                                          const Blocks<kTileKeys>& blocks, int begin, int end, bool parts, float2* part_ms, Part part, Out out) {
  constexpr int DT = D / 32, KS = D / 16, CH = D / 16;
  constexpr int NL = D / 64;                       // loads into LDS of a wavefront, keys and values each
  constexpr int RL = 64 / CH;                      // rows of a load
  uint8_t *const k0 = PageLds<D>::template array<0>(), *const k1 = PageLds<D>::template array<1>(), *const k2 = PageLds<D>::template array<2>(), *const k3 = PageLds<D>::template array<3>();
  uint8_t *const v0 = PageLds<D>::template array<4>(), *const v1 = PageLds<D>::template array<5>(), *const v2 = PageLds<D>::template array<6>(), *const v3 = PageLds<D>::template array<7>();
  int2* const meta = PageLds<D>::meta();           // page (or -1) and exponents (keys, values << 8, kHole) of the groups
  const int lane = tid % kWave, wv = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int c32 = lane % 32, half = lane / 32;
  f32x16_t o[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) o[i] = f32x16_t{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
  float top = kNoLogit, sum = 0.0f;

  // ---- pages of a chunk of steps, a group a thread
  auto wanted = [&](int key) { return key < blocks.end && (key >= blocks.near_key || key < blocks.first_keys); };
  auto page_of = [&](int chunk) {                  // of a group: its page, -1 where none is needed, -2 where there is none
    const int step = begin + chunk * kChunk + tid / kGroups;
    int p = -1;
    if (step < end) {
      const int key = blocks.block(step) * kTileKeys + tid % kGroups * kGroup;
      if (key < blocks.end && (key + kGroup > blocks.near_key || key < blocks.first_keys)) {     // (then key lies inside the row: see sight_of)
        p = table[key >> a.page_shift];
        p = p >= 0 && p < a.n_pages ? p : -2;
      }
    }
    return p;
  };
  auto exps_of = [&](int p) {
    const int64_t block = (int64_t)p * a.H_kv + h;
    return p >= 0 ? a.k_exp[block] | a.v_exp[block] << 8 : p == -2 ? kHole : 0;
  };
  auto look_up = [&](int chunk) {
    const int p = page_of(chunk);
    return int2{p < 0 ? -1 : p, exps_of(p)};
  };
  // What does not wait for each other is on its way at once: the first pages and what rows_of() reads; queries, exponents, and the keys and values that the pages hold.
  const int first_page = page_of(0);
  const TileRow mine = rows_of();
  const RowSight sight = mine.sight;
  // a lane's 16 bytes of a key are features 32 l + 16 half .. + 16, for two products
  bf16x8_t qf[KS];
#pragma unroll
  for (int k = 0; k < KS; ++k) __builtin_memcpy(&qf[k], mine.q + 16 * half + 32 * (k / 2) + 8 * (k % 2), 16);
  auto meta_at = [&](int step) { return (step - begin) % (2 * kChunk) * kGroups; };

  // ---- a step's keys and values into LDS.  Keys that no row of the workgroup sees become zeros (loads behind the end of their buffer): their
  // weights are zero, and zero times what memory happens to hold may be NaN.
  const int d_row = RL * wv + lane / CH;                                // rows of load j: d_row + RL * kTileWaves * j
  const int k_off = lane / CH * D + (lane % CH ^ key_swizzle<D>(d_row)) * 16, v_off = lane / CH * D + (lane % CH ^ value_swizzle<D>(d_row)) * 16;
  int pages[NL];                                                        // of the step to be loaded next
  auto read_pages = [&](int step) {
#pragma unroll
    for (int j = 0; j < NL; ++j) pages[j] = meta[meta_at(step) + (j * kTileWaves + wv) * RL / kGroup].x;
  };
  auto load = [&](uint8_t* to_k, uint8_t* to_v, int step) {
    if (step < end) {
      const int key0 = blocks.block(step) * kTileKeys;
      const bool whole = key0 + kTileKeys <= blocks.end && (key0 >= blocks.near_key || key0 + kTileKeys <= blocks.first_keys);
#pragma unroll
      for (int j = 0; j < NL; ++j) {
        const int p = __builtin_amdgcn_readfirstlane(pages[j]), key = key0 + (j * kTileWaves + wv) * RL;
        const int64_t at = ((((int64_t)(p < 0 ? 0 : p) * a.H_kv + h) << a.page_shift) + (key & ((1 << a.page_shift) - 1))) * D;
        const int bytes = p < 0 ? 0 : RL * D, skip = whole || wanted(key + lane / CH) ? 0 : 1 << 20;
        const __amdgpu_buffer_rsrc_t fk = __builtin_amdgcn_make_buffer_rsrc((void*)(a.k + at), 0, bytes, 0x00027000);
        const __amdgpu_buffer_rsrc_t fv = __builtin_amdgcn_make_buffer_rsrc((void*)(a.v + at), 0, bytes, 0x00027000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(fk, (__attribute__((address_space(3))) void*)(to_k + (j * kTileWaves + wv) * 1024), 16, k_off + skip, 0, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(fv, (__attribute__((address_space(3))) void*)(to_v + (j * kTileWaves + wv) * 1024), 16, v_off + skip, 0, 0, 0);
      }
    }
    read_pages(step + 1);
  };

  // ---- one step
  int k_at[DT], v_at[DT];                          // a lane's places: chunk 2 l + half of key c32; features 32 i + lane % 32 of its eight keys
  {
    const int vr = lane % 16 / 2, key = (vr < 4 ? vr : vr + 4) + 4 * half;
#pragma unroll
    for (int i = 0; i < DT; ++i) {
      k_at[i] = c32 * D + (2 * i + half ^ key_swizzle<D>(c32)) * 16;
      v_at[i] = key * D + (2 * i + lane / 16 % 2 ^ value_swizzle<D>(key)) * 16 + lane % 2 * 8;
    }
  }
  int exps[kGroups];                               // of the step whose values come next
  auto read_exps = [&](int (&e)[kGroups], int step) {
#pragma unroll
    for (int i = 0; i < kGroups; ++i) e[i] = meta[meta_at(step) + i].y;
  };
  auto key_scale = [&](const int (&e)[kGroups], int kb) {
    const int first = e[2 * kb], second = e[2 * kb + 1];
    return exp_scale((c32 < kGroup ? first : second) & 255);
  };
  auto widen_key = [&](const uint4& x, int w, float scale) {
    const uint2 p = widen_e4m3(w ? x.z : x.x, scale), q = widen_e4m3(w ? x.w : x.y, scale);
    return __builtin_bit_cast(bf16x8_t, uint4{p.x, p.y, q.x, q.y});
  };
  auto all_seen = [&](const int (&e)[kGroups], int step) {      // every key of a step by every row of the wavefront
    const int key0 = blocks.block(step) * kTileKeys, last = key0 + kTileKeys - 1;
    return last < keys && last <= lo && (a.window <= 0 || (int64_t)key0 > (int64_t)hi - a.window || last < a.sinks) &&
           !(__builtin_amdgcn_readfirstlane(e[0] | e[1] | e[2] | e[3]) & kHole);
  };
  auto largest = [&](const f32x16_t (&S)[2]) {
    float m = fmaxf(S[0][0], S[1][0]);
#pragma unroll
    for (int i = 1; i < 16; ++i) m = max3(m, S[0][i], S[1][i]);
    return m;
  };
  auto mask = [&](f32x16_t (&S)[2], const int (&e)[kGroups], int step) __attribute__((always_inline)) {    // what a row does not see: -infinity; a lane's largest logit
    const int key0 = blocks.block(step) * kTileKeys + 4 * half;
    const bool firsts = a.window > 0 && blocks.block(step) * kTileKeys < a.sinks;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = key0 + kb * 32 + i / 4 * 8 + i % 4;
        const bool seen = (sight.sees(key) | (firsts & (key < sight.first))) & !(e[2 * kb + i / 8] & kHole);
        S[kb][i] = seen ? S[kb][i] : -__builtin_huge_valf();
      }
    }
    return largest(S);
  };
  auto raise = [&](float m) {                      // the running maximum, moved where a logit (m: a lane's largest one) lies far above it
    if (__any(m > top + kSlack)) {
      const float n = fmaxf(top, halves_max(m)), f = __builtin_amdgcn_exp2f(top - n);
      top = n;
      sum *= f;
#pragma unroll
      for (int i = 0; i < DT; ++i) o[i] *= f;
    }
  };
  // (kn: keys of the next step, v: values of this one;  kl, vl: of the step that is loaded)
  auto advance = [&](f32x16_t (&S)[2], f32x16_t (&next)[2], const uint8_t* kn, const uint8_t* v, uint8_t* kl, uint8_t* vl, int i) __attribute__((always_inline)) {
    constexpr int NA = 2 * KS, NB = 4 * DT;        // products of either kind
    constexpr int AHEAD = 4;                       // value operands on their way out of LDS; keys: half as many, for two products each
    // Weights: logit, exponential and sum three places apart, so that none waits for the one before; `place` p takes logit p + 3, exponential p and sum
    // p - 3.  The first places beside the first kind of product (three operands of the second kind are then there), the others beside the second.
    constexpr int PLACES = 35, PA = 28;
    const bool turn = (i - begin) % kChunk == 0 && i + kChunk < end;
    int2 m2 = {-1, 0};
    if (turn) m2 = look_up((i - begin) / kChunk + 1);
    load(kl, vl, i + kStages - 1);
    int e_next[kGroups];
    read_exps(e_next, i + 1);
    uint4 kr[AHEAD / 2];
    uint2 vr[AHEAD];
    bf16x8_t P[4];
    float x[32], w[32];
    auto read_k = [&](int p) { kr[p % (AHEAD / 2)] = *(const uint4*)(kn + p / DT * 32 * D + k_at[p % DT]); };
    auto read_v = [&](int n) { vr[n % AHEAD] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2_t)(v + 16 * (n / DT) * D + v_at[n % DT]))); };
    auto place = [&](int p) {
      if (p + 3 < 32) x[p + 3] = fmaf(S[(p + 3) / 16][(p + 3) % 16], a.scale_log2e, -top);
      if (p < 32) w[p] = __builtin_amdgcn_exp2f(x[p]);
      const int e = p - 3;
      if (e >= 0) sum += w[e];
      if (e >= 0 && e % 8 == 7)
        P[e / 8] = __builtin_bit_cast(bf16x8_t, uint4{pack_bf16(w[e - 7], w[e - 6]), pack_bf16(w[e - 5], w[e - 4]), pack_bf16(w[e - 3], w[e - 2]), pack_bf16(w[e - 1], w[e])});
    };
#pragma unroll
    for (int e = 0; e < 3; ++e) x[e] = fmaf(S[0][e], a.scale_log2e, -top);
#pragma unroll
    for (int p = 0; p < AHEAD / 2; ++p) read_k(p);
    const float ks[2] = {key_scale(e_next, 0), key_scale(e_next, 1)};
#pragma unroll
    for (int n = 0; n < NA; ++n) {
      __builtin_amdgcn_sched_barrier(0);
      const bf16x8_t kf = widen_key(kr[n / 2 % (AHEAD / 2)], n % 2, ks[n / KS]);
      next[n / KS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[n % KS], n % KS == 0 ? f32x16_t{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0} : next[n / KS], 0, 0, 0);
      if (n % 2 == 1 && n / 2 + AHEAD / 2 < NA / 2) read_k(n / 2 + AHEAD / 2);
      if (n >= NA - AHEAD) read_v(n - (NA - AHEAD));
#pragma unroll
      for (int p = n * PA / NA; p < (n + 1) * PA / NA; ++p) place(p);
    }
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      __builtin_amdgcn_sched_barrier(0);
      const float scale = exp_scale(exps[n / DT] >> 8 & 255);
      const uint2 x = widen_e4m3(vr[n % AHEAD].x, scale), y = widen_e4m3(vr[n % AHEAD].y, scale);
      o[n % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, uint4{x.x, x.y, y.x, y.y}), P[n / DT], o[n % DT], 0, 0, 0);
      if (n + AHEAD < NB) read_v(n + AHEAD);
#pragma unroll
      for (int p = PA + n * 16 / NB; p < PA + (n + 1) * 16 / NB && p < PLACES; ++p) place(p);
    }
    products_settle();
    if (i + 1 < end) raise((all_seen(e_next, i + 1) ? largest(next) : mask(next, e_next, i + 1)) * a.scale_log2e);
#pragma unroll
    for (int j = 0; j < kGroups; ++j) exps[j] = e_next[j];
    if (turn) meta[((i - begin) / kChunk + 1) % 2 * kChunk * kGroups + tid] = m2;
    // all but the loads of this step have arrived
    if (i + kStages - 1 < end) __builtin_amdgcn_s_waitcnt(0x0f70 | 2 * NL);
    else __builtin_amdgcn_s_waitcnt(0x0f70);
    __syncthreads();
  };
  static_assert(kChunk * kGroups == kTileThreads, "a group a thread");

  f32x16_t S0[2], S1[2];
  meta[tid].x = first_page < 0 ? -1 : first_page;
  const int first_exps = exps_of(first_page);
  __syncthreads();
  if (begin < end) {
    read_pages(begin);
    load(k0, v0, begin);
    load(k1, v1, begin + 1);
    load(k2, v2, begin + 2);
  }
  meta[tid].y = first_exps;
  meta[kChunk * kGroups + tid] = int2{-1, 0};
  __builtin_amdgcn_s_waitcnt(0x0f70);
  __syncthreads();
  if (begin < end) {
    read_exps(exps, begin);
#pragma unroll
    for (int n = 0; n < 2 * KS; ++n) {
      const bf16x8_t kf = widen_key(*(const uint4*)(k0 + n / KS * 32 * D + k_at[n % KS / 2]), n % 2, key_scale(exps, n / KS));
      S0[n / KS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[n % KS], n % KS == 0 ? f32x16_t{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0} : S0[n / KS], 0, 0, 0);
    }
    products_settle();
    raise((all_seen(exps, begin) ? largest(S0) : mask(S0, exps, begin)) * a.scale_log2e);
  }
  for (int i = begin; i < end; i += 4) {
    advance(S0, S1, k1, v0, k3, v3, i);
    if (i + 1 < end) advance(S1, S0, k2, v1, k0, v0, i + 1);
    if (i + 2 < end) advance(S0, S1, k3, v2, k1, v1, i + 2);
    if (i + 3 < end) advance(S1, S0, k0, v3, k2, v2, i + 3);
  }

  sum += __shfl_xor(sum, 32);
  uint8_t* rows = wv < 2 ? wv == 0 ? k0 : k1 : wv == 2 ? k2 : k3;
  if (parts) {
    if (half == 0 && part_ms) *part_ms = float2{top, sum};
    float_rows_out<D>(o, rows, part, lane);
    return;
  }
  rows_out<D>(o, sum > 0.0f ? 1.0f / sum : 0.0f, rows, out, lane);
}

}  // namespace ficoco
