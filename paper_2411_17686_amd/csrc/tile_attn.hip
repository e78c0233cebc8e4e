// Attention for many rows: dense prompts with a window, and questions of many tokens over pages of 8 bits.
#include <algorithm>

#include "attend.hpp"

namespace ficoco {
namespace {

constexpr int kTileWaves = 4;
constexpr int kTileThreads = kTileWaves * kWave;
constexpr int kTileRows = 32 * kTileWaves;   // rows of a workgroup
constexpr int kTileKeys = 64;                // keys of a step
constexpr float kSlack = 8.0f;               // (units of log2) growth of a row's maximum that is put up with

constexpr int kHole = 1 << 16;                // (beside two exponent bytes) a key that would be seen has no page

typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4_t* lds_i16x4_t;

// Rows of keys and values in LDS, in bfloat16.  A key row is read 16 bytes a lane by 16 rows at once: 16 bytes of padding put
// them on all 64 banks.  Of the values, groups of 16 lanes read four keys x 16 features: rows 64 bytes further on modulo 256.
template <int D> constexpr int kKeyPitch = D + 8;
template <int D> constexpr int kValuePitch = D + 32;

template <int D, bool PAGED> struct TileRaw;       // one step's share of a thread
template <int D> struct TileRaw<D, false> { uint4 k[D / 32], v[D / 32]; };
template <int D> struct TileRaw<D, true> { uint4 k[D / 64], v[D / 64]; int exps[D / 64]; };

__device__ __forceinline__ float halves_max(float v) { return fmaxf(v, __shfl_xor(v, 32)); }

// One pass with a running maximum and sum, 128 rows a workgroup, 32 a wavefront, 64 keys a step.  32 x 32 x 16 products:
//   S^T[key][row] = K Q^T, the queries in registers; a lane holds 32 logits of one row
//   O^T[feature][row] += V^T P^T, the contraction in the order in which the lanes hold the weights; V^T out of LDS by transposing reads
// The next step's keys and values travel from memory to registers while one is computed (8 bits are widened, with their
// block's scale, on the way into LDS) and are written to the other of two buffers.
template <int D, bool PAGED>
__global__ __launch_bounds__(kTileThreads, 2) void tile_rows_kernel(AttendArgs a) {
  constexpr int KP = kKeyPitch<D>, VP = kValuePitch<D>, DT = D / 32, KS = D / 16;
  constexpr int NL = PAGED ? D / 64 : D / 32;      // 16-byte loads of a thread, keys and values each
  constexpr int CH = PAGED ? D / 16 : D / 8;       // of a row
  __shared__ __align__(16) bf16_t sk[2][kTileKeys * KP];
  __shared__ __align__(16) bf16_t sv[2][kTileKeys * VP];
  __shared__ int hole[2];                          // 1 + the last step in this buffer some of whose keys have no page
  const int tid = threadIdx.x, lane = tid % kWave, wv = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int c32 = lane % 32, half = lane / 32;
  const int per_head = a.row_tiles * a.splits, total = a.B * a.H_kv * per_head;
  const int id = xcd_logical_id(blockIdx.x, total);
  if (id >= total) return;
  const int bh = id / per_head, in_head = id % per_head, h = bh % a.H_kv, b = bh / a.H_kv;
  const int split = in_head % a.splits, tile = a.row_tiles - 1 - in_head / a.splits;    // (the last rows see most keys)
  int slot;
  const Sight s = sight_of<PAGED>(a, b, slot);
  const int rows = s.queries * a.group, row0 = tile * kTileRows;
  if (s.queries <= 0 || row0 >= rows) return;
  auto pos_of = [&](int r) { return s.first + (r < rows ? r : rows - 1) / a.group; };
  const Blocks<kTileKeys> blocks(a, s, pos_of(row0), pos_of(row0 + kTileRows - 1));
  const int per = (blocks.count + a.splits - 1) / a.splits;
  const int begin = split * per, end = begin + per < blocks.count ? begin + per : blocks.count;

  const int r = row0 + 32 * wv + c32, my_r = r < rows ? r : rows - 1;
  const int t = my_r / a.group, g = my_r % a.group, pos = s.first + t;
  const int lo = pos_of(row0 + 32 * wv), hi = pos_of(row0 + 32 * wv + 31);      // positions of the wavefront
  bf16x8_t qf[KS];
  {
    const bf16_t* q = a.Q + (int64_t)b * a.q_sb + (int64_t)(h * a.group + g) * a.q_sh + (int64_t)t * a.q_sn + 8 * half;
#pragma unroll
    for (int k = 0; k < KS; ++k) __builtin_memcpy(&qf[k], q + 16 * k, 16);
  }
  f32x16_t o[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) o[i] = f32x16_t{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
  float top = kNoLogit, sum = 0.0f;

  // keys and values of a step: memory -> registers -> LDS
  const int32_t* table = PAGED ? a.table + (int64_t)slot * a.max_pages : nullptr;
  auto wanted = [&](int key) { return key < blocks.end && (key >= blocks.near_key || key < blocks.first_keys); };
  auto page_at = [&](int step, int j) {
    const int key = blocks.block(step) * kTileKeys + (tid + j * kTileThreads) / CH;
    int p = -1;
    if (step < end && wanted(key)) p = table[key >> a.page_shift];       // (keys lie inside the row: see sight_of)
    return p < a.n_pages ? p : -1;
  };
  int pages[NL];
  auto load = [&](TileRaw<D, PAGED>& raw, int step) {
    const int key0 = blocks.block(step) * kTileKeys;
#pragma unroll
    for (int j = 0; j < NL; ++j) {
      const int at = tid + j * kTileThreads, key = key0 + at / CH, ch = at % CH;
      raw.k[j] = raw.v[j] = uint4{0, 0, 0, 0};
      if constexpr (PAGED) {
        raw.exps[j] = pages[j] < 0 && wanted(key) ? kHole : 0;
        if (pages[j] >= 0) {
          const int64_t block = (int64_t)pages[j] * a.H_kv + h;
          const int64_t from = ((block << a.page_shift) + (key & ((1 << a.page_shift) - 1))) * D + 16 * ch;
          raw.k[j] = *(const uint4*)(a.k + from);
          raw.v[j] = *(const uint4*)(a.v + from);
          raw.exps[j] = a.k_exp[block] | a.v_exp[block] << 8;
        }
      } else if (wanted(key)) {
        __builtin_memcpy(&raw.k[j], a.K + (int64_t)b * a.k_sb + (int64_t)h * a.k_sh + (int64_t)key * a.k_sn + 8 * ch, 16);
        __builtin_memcpy(&raw.v[j], a.V + (int64_t)b * a.v_sb + (int64_t)h * a.v_sh + (int64_t)key * a.v_sn + 8 * ch, 16);
      }
    }
    if constexpr (PAGED) {
#pragma unroll
      for (int j = 0; j < NL; ++j) pages[j] = page_at(step + 1, j);
    }
  };
  auto store = [&](const TileRaw<D, PAGED>& raw, int step, int buf) {
#pragma unroll
    for (int j = 0; j < NL; ++j) {
      const int at = tid + j * kTileThreads, key = at / CH, ch = at % CH;
      if constexpr (PAGED) {
        if (raw.exps[j] & kHole) hole[buf] = step + 1;
        const float ks = exp_scale(raw.exps[j] & 255), vs = exp_scale(raw.exps[j] >> 8 & 255);
        const uint2 k0 = widen_e4m3(raw.k[j].x, ks), k1 = widen_e4m3(raw.k[j].y, ks), k2 = widen_e4m3(raw.k[j].z, ks), k3 = widen_e4m3(raw.k[j].w, ks);
        const uint2 v0 = widen_e4m3(raw.v[j].x, vs), v1 = widen_e4m3(raw.v[j].y, vs), v2 = widen_e4m3(raw.v[j].z, vs), v3 = widen_e4m3(raw.v[j].w, vs);
        uint4* k = (uint4*)&sk[buf][key * KP + 16 * ch];
        uint4* v = (uint4*)&sv[buf][key * VP + 16 * ch];
        k[0] = uint4{k0.x, k0.y, k1.x, k1.y};
        k[1] = uint4{k2.x, k2.y, k3.x, k3.y};
        v[0] = uint4{v0.x, v0.y, v1.x, v1.y};
        v[1] = uint4{v2.x, v2.y, v3.x, v3.y};
      } else {
        *(uint4*)&sk[buf][key * KP + 8 * ch] = raw.k[j];
        *(uint4*)&sv[buf][key * VP + 8 * ch] = raw.v[j];
      }
    }
  };

  auto compute = [&](int step, int buf) {
    const int key0 = blocks.block(step) * kTileKeys, last = key0 + kTileKeys - 1;
    if (key0 > hi || (a.window > 0 && (int64_t)last <= (int64_t)lo - a.window && key0 >= a.sinks)) return;      // nothing for this wavefront
    f32x16_t S[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const bf16x8_t kf = *(const bf16x8_t*)&sk[buf][(kb * 32 + c32) * KP + 16 * k + 8 * half];
        S[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[k], k == 0 ? f32x16_t{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0} : S[kb], 0, 0, 0);
      }
    }
    bool all_seen = last < s.keys && last <= lo && (a.window <= 0 || (int64_t)key0 > (int64_t)hi - a.window || last < a.sinks);
    if (PAGED) all_seen = all_seen && __builtin_amdgcn_readfirstlane(hole[buf]) != step + 1;
    if (!all_seen) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = key0 + kb * 32 + i / 4 * 8 + 4 * half + i % 4;
          bool seen = key_seen(a, key, pos, s.keys);
          if (PAGED) {
            const int at = key >> a.page_shift;
            const int p = seen ? table[at] : -1;
            seen = p >= 0 && p < a.n_pages;
          }
          S[kb][i] = seen ? S[kb][i] : -__builtin_huge_valf();
        }
      }
    }
    float m = fmaxf(S[0][0], S[1][0]);
#pragma unroll
    for (int i = 1; i < 16; ++i) m = fmaxf(m, fmaxf(S[0][i], S[1][i]));
    m *= a.scale_log2e;
    if (__any(m > top + kSlack)) {
      const float n = fmaxf(top, halves_max(m)), f = __builtin_amdgcn_exp2f(top - n);
      top = n;
      sum *= f;
#pragma unroll
      for (int i = 0; i < DT; ++i) o[i] *= f;
    }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          p[i] = __builtin_amdgcn_exp2f(fmaf(S[kb][8 * u + i], a.scale_log2e, -top));
          sum += p[i];
        }
        const bf16x8_t P = __builtin_bit_cast(bf16x8_t, uint4{pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7])});
        const bf16_t* v = &sv[buf][(kb * 32 + 16 * u + 4 * half + lane % 16 / 4) * VP + lane / 16 % 2 * 16 + lane % 4 * 4];
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          const i16x4_t v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t)(v + 32 * i));
          const i16x4_t v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t)(v + 8 * VP + 32 * i));
          const uint2 x = __builtin_bit_cast(uint2, v0), y = __builtin_bit_cast(uint2, v1);
          o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, uint4{x.x, x.y, y.x, y.y}), P, o[i], 0, 0, 0);
        }
      }
    }
  };

  TileRaw<D, PAGED> raw;
  if (begin < end) {
    if constexpr (PAGED) {
#pragma unroll
      for (int j = 0; j < NL; ++j) pages[j] = page_at(begin, j);
    }
    load(raw, begin);
  }
  if (tid < 2) hole[tid] = 0;
  __syncthreads();
  if (begin < end) store(raw, begin, 0);
  __syncthreads();
  for (int i = begin; i < end; ++i) {
    const int buf = (i - begin) & 1;
    if (i + 1 < end) load(raw, i + 1);
    compute(i, buf);
    if (i + 1 < end) store(raw, i + 1, buf ^ 1);
    __syncthreads();
  }

  sum += __shfl_xor(sum, 32);
  if (r >= rows) return;
  if (a.splits > 1) {
    const int64_t at = ((int64_t)bh * a.splits + split) * a.part_rows + r;
    if (half == 0) a.part_ms[at] = float2{top, sum};
#pragma unroll
    for (int i = 0; i < DT; ++i) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *(f32x4_t*)(a.part_o + at * D + 32 * i + 8 * j + 4 * half) = f32x4_t{o[i][4 * j], o[i][4 * j + 1], o[i][4 * j + 2], o[i][4 * j + 3]};
    }
    return;
  }
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  bf16_t* out = a.O + (int64_t)b * a.o_sb + (int64_t)(h * a.group + g) * a.o_sh + (int64_t)t * a.o_sn + 4 * half;
#pragma unroll
  for (int i = 0; i < DT; ++i) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint2 w = {pack_bf16(o[i][4 * j] * inv, o[i][4 * j + 1] * inv), pack_bf16(o[i][4 * j + 2] * inv, o[i][4 * j + 3] * inv)};
      __builtin_memcpy(out + 32 * i + 8 * j, &w, 8);
    }
  }
}

}  // namespace

AttendPlan attend_plan(const ficoco_attention& a, int heads, int64_t max_keys, bool paged) {
  AttendPlan pl{};
  const int64_t rows = (int64_t)a.n_q * (a.H / heads), bh = (int64_t)a.B * heads;
  pl.few = paged && rows <= 16;
  pl.rows = pl.few ? 16 : kTileRows;
  pl.row_tiles = (int)std::max<int64_t>(1, (rows + pl.rows - 1) / pl.rows);
  pl.splits = 1;
  if (paged && bh > 0) {
    int64_t seen = max_keys;
    if (a.window > 0) seen = std::min(seen, (int64_t)a.window + a.sinks + a.n_q);
    // about two workgroups a compute unit, but at least two steps a wavefront, and four of a tile
    const int64_t least = pl.few ? 256 : 256, want = (512 + bh * pl.row_tiles - 1) / (bh * pl.row_tiles);
    pl.splits = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(want, seen / least), 256));
  }
  const size_t parts = pl.splits > 1 ? (size_t)bh * pl.splits * pl.row_tiles * pl.rows : 0;
  pl.part_ms = 0;
  pl.part_o = (parts * sizeof(float2) + 255) / 256 * 256;
  pl.total = std::max<size_t>(256, pl.part_o + (parts * a.d_head * sizeof(float) + 255) / 256 * 256);
  return pl;
}

void launch_tile_rows(const AttendArgs& a, int d_head, bool paged, hipStream_t s) {
  const dim3 grid((unsigned)xcd_padded_total(a.B * a.H_kv * a.row_tiles * a.splits)), threads(kTileThreads);
  if (paged) {
    if (d_head == 128) hipLaunchKernelGGL((tile_rows_kernel<128, true>), grid, threads, 0, s, a);
    else hipLaunchKernelGGL((tile_rows_kernel<64, true>), grid, threads, 0, s, a);
  } else {
    if (d_head == 128) hipLaunchKernelGGL((tile_rows_kernel<128, false>), grid, threads, 0, s, a);
    else hipLaunchKernelGGL((tile_rows_kernel<64, false>), grid, threads, 0, s, a);
  }
}

}  // namespace ficoco
