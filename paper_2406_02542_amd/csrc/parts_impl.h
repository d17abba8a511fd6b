// Dense attention over a batch's caches in runs of rows (Section 2, Eq. 1 of arXiv 2406.02542): how a batch is dealt out over
// blocks by length, and one run of it, which leaves (max, sum, output) per query head and, where asked for, the
// logits of its rows.  Shared by the kernels that weigh rows (weigh.hip) and that have a prefix in front (shared.hip).
#pragma once

#include "attend_mfma_impl.h"

namespace loki {

__device__ __forceinline__ int part_rows_held(const Ragged& rg, int b, int S_max) {
  return rg.seq_lens == nullptr ? S_max : min(max(rg.seq_lens[b], 0), S_max);
}
// How a batch is dealt out: the X = nsplit B blocks that a KV head has are runs of `run` rows, the same for all sequences, so
// that blocks have about the same work whatever the lengths; of X runs as many are used as the sequences fill.  run is the
// smaller of what cuts the longest sequence into nsplit and what leaves every sequence one partial run more than its share,
// total / (X - B): either keeps the sum of the sequences' runs within X.  Whole steps of 32 rows, so that a step's logits are
// stored 16 bytes at a time.  Every wave works it out for itself, 64 sequences at a time.
struct Dealt {
  int run;
  float total;
};
// The largest of the wave's non-negative values, the same in every lane, without LDS.
__device__ __forceinline__ int wave_max_i32(int x) {
  x = max(x, (int)dpp_u32<0x111, 0xf, true>((uint32_t)x));   // (as wave_inclusive_scan_u32)
  x = max(x, (int)dpp_u32<0x112, 0xf, true>((uint32_t)x));
  x = max(x, (int)dpp_u32<0x114, 0xf, true>((uint32_t)x));
  x = max(x, (int)dpp_u32<0x118, 0xf, true>((uint32_t)x));
  x = max(x, (int)dpp_u32<0x142, 0xa, false>((uint32_t)x));
  x = max(x, (int)dpp_u32<0x143, 0xc, false>((uint32_t)x));
  return __builtin_amdgcn_readlane(x, 63);
}
__device__ __forceinline__ Dealt deal_runs(const Ragged& rg, int B, int S_max, int nsplit) {
  float total = (float)B * (float)S_max;
  int longest = S_max;
  const int lane = threadIdx.x & 63;
  if (rg.seq_lens != nullptr) {
    total = 0.f;
    longest = 0;
    for (int b0 = 0; b0 < B; b0 += 64) {
      const int len = b0 + lane < B ? part_rows_held(rg, b0 + lane, S_max) : 0;
      total += wave_sum_f32((float)len);
      longest = max(longest, wave_max_i32(len));
    }
  }
  const int spare = (nsplit - 1) * B;  // X - B
  int run = (longest + nsplit - 1) / max(nsplit, 1);
  // (2^-16 more than the quotient: above it for all that the sum, the product and the reciprocal round)
  if (spare > 0) run = (int)fminf((float)run, ceilf(total * (1.0f / (float)spare) * 1.0000153f));
  return {max(32, (run + 31) & ~31), total};
}
// The sequence and the run of it that run x of a KV head is, and the place of its part (sequences one after the other); b = B: none.
// The whole runs come first, then what is left over of each sequence, so that the blocks end together (and the heads of a run
// are neighbours in the grid).  us in the order of the sequences and so: 24 sequences of 32/8 bf16 heads up to 7000 rows 96.8, 90.7, up to
// 8192 110.5, 102.3, 16 up to 16384 145, 141; 9 of 24 up to 3000 46.1, 42.9; 13 of 32/8 up to 300 12.1, 11.1.
struct RunAt {
  int b, i, len, place;
};
__device__ __forceinline__ RunAt find_run(const Ragged& rg, int B, int S_max, int run, int x) {
  if (rg.seq_lens == nullptr) {
    const int each = (S_max + run - 1) / run, whole = S_max / run;
    const bool rest = x >= B * whole;
    const int b = rest ? (each > whole ? x - B * whole : B) : x / whole, i = rest ? whole : x - b * whole;
    return {min(b, B), i, S_max, b * each + i};
  }
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int rest = 0; rest < 2; ++rest) {
    int before = 0;  // places of the sequences in front
    for (int b0 = 0; b0 < B; b0 += 64) {
      const int len = b0 + lane < B ? part_rows_held(rg, b0 + lane, S_max) : 0, runs = (len + run - 1) / run;
      const int whole = runs * run > len ? runs - 1 : runs, mine = rest ? runs - whole : whole;
      const int incl = (int)wave_inclusive_scan_u32((uint32_t)mine), places = (int)wave_inclusive_scan_u32((uint32_t)runs);
      const unsigned long long behind = __ballot(incl > x);
      if (behind != 0ull) {
        const int at = __ffsll((long long)behind) - 1;
        const int i = rest ? __builtin_amdgcn_readlane(whole, at) : x - (__builtin_amdgcn_readlane(incl, at) - __builtin_amdgcn_readlane(mine, at));
        return {b0 + at, i, __builtin_amdgcn_readlane(len, at),
                before + __builtin_amdgcn_readlane(places, at) - __builtin_amdgcn_readlane(runs, at) + i};
      }
      x -= __builtin_amdgcn_readlane(incl, 63);
      before += __builtin_amdgcn_readlane(places, 63);
    }
  }
  return {B, 0, 0, 0};
}
// The first run of sequence b.
__device__ __forceinline__ int first_run(const Ragged& rg, int S_max, int run, int b) {
  if (rg.seq_lens == nullptr) return b * ((S_max + run - 1) / run);
  const int lane = threadIdx.x & 63;
  int at = 0;
  for (int b0 = 0; b0 < b; b0 += 64) {
    const int runs = b0 + lane < b ? (part_rows_held(rg, b0 + lane, S_max) + run - 1) / run : 0;
    at += __builtin_amdgcn_readlane((int)wave_inclusive_scan_u32((uint32_t)runs), 63);
  }
  return at;
}

template <typename Keep>
struct KeepIn {  // (handed over by value: the rows' loop is compiled for callers without logits too)
  static constexpr bool kAny = true;
  Keep* keep;
  __device__ __forceinline__ void operator()(int g, int row, const float4& x) const { (*keep)(g, row, x); }
  __device__ __forceinline__ void step(int b0) const { keep->step(b0); }
};

template <int NH>
constexpr bool parts_mfma() {  // four heads and more: matrix cores (fp32, with the merge: 16 sequences of 64/8 heads with 4096 rows
  return NH >= 4;              // 181 us on the vector units, 113 so, of 32/8 113, 107; one of 32/4 with 16384 rows 37, 21)
}

// The logits of the unit's heads, [head][pitch]: on the vector units one lane of a row's group stores them.
struct StoreLogits {
  static constexpr bool kAny = true;
  float* p;  // of the unit's first head
  size_t pitch;
  bool writer;
  __device__ __forceinline__ void operator()(int g, int row, bool ok, float x) const {
    if (writer && ok) p[g * pitch + row] = x;
  }
};
// fp32 on the matrix cores: four rows of a head at a time (the rows of the sequence's last step past its end lie inside the pitch,
// which is a multiple of 32).
template <int NH>
struct StoreSteps {
  static constexpr bool kAny = true;
  float* p;
  size_t pitch;
  __device__ __forceinline__ void operator()(int g, int row, const float4& x) const {
    if (g < NH) *reinterpret_cast<float4*>(p + g * pitch + row) = x;
  }
};
// bf16 on the matrix cores: a wave keeps those of some steps in LDS and stores them together, whole lines: memory operations are
// waited for in their order, so a store of every step is waited for with the next rows.  16 sequences of 32/8 heads up to
// 16384 rows: the launch 136, 134, 130 and 130 us for runs of 2, 4, 16 and 32 steps; 118 with the stores left out.
template <int NH>
constexpr int kept_steps() {
  return 64 / NH;
}
template <int NH, int WAVES>
struct KeepLogits {
  static constexpr bool kAny = true;
  float* p;  // of the unit's first head
  size_t pitch;
  float* kept;  // the wave's [kept_steps][NH][32]
  int n = 0, base = 0;
  __device__ __forceinline__ void operator()(int g, int row, const float4& x) const {
    if (g < NH) *reinterpret_cast<float4*>(kept + (n * NH + g) * kAmRows + row) = x;
  }
  __device__ __forceinline__ void step(int b0) {  // the step that begins at row b0 is complete
    if (n == 0) base = b0;
    if (++n == kept_steps<NH>()) flush();
  }
  // (the rows of the sequence's last step past its end lie inside the pitch, which is a multiple of 32)
  __device__ __forceinline__ void flush() {
    __builtin_amdgcn_wave_barrier();
    for (int i = threadIdx.x & 63; i < n * NH * 8; i += 64) {
      const int s = i / (NH * 8), g = i / 8 % NH;
      const float4 x = *reinterpret_cast<const float4*>(kept + i * 4);
      *reinterpret_cast<float4*>(p + g * pitch + base + s * (WAVES * kAmRows) + i % 8 * 4) = x;
    }
    __builtin_amdgcn_wave_barrier();
    n = 0;
  }
};

// ---- fp32 on the matrix cores, straight from registers --------------------------------------------------------------
// A wave takes steps of 16 keys and holds QG groups of 16 query rows:
//   S^T[key, query] = K Q^T         v_mfma_f32_16x16x4_f32; lane (key, c) loads 16 bytes of its key's row at a time, columns
//                                   16 j + 4 c .. + 3, one for each of four products, and the queries the same columns
//   O^T[column, query] += V^T P^T   the weights as they come out of the first product are operand i's keys 4 c + i; lane (m, c)
//                                   loads 16 bytes of each of these rows, columns 4 m .. + 3 of either half
// A logit is summed in four chains of 32 columns: its error, which sets the output's, is a third of one chain's (relative to 64 bits,
// one sequence of 32/4 heads, 300 rows 0.4e-6 to 1.1e-6, one chain 1.9e-6 to 3.5e-6), for no time.
// A step's keys and values are in registers before it begins.  The block's waves take steps in turn and are joined in LDS.
// STREAM: the values come past the caches, whole lines; a key's line comes in two halves (64/8 heads, 32 sequences of 8192 rows 433 us,
// with the keys past the caches too 454).
// Two groups at most, so that two waves share a SIMD: 64 sequences of 64/8 heads behind 16384 rows with one, two and four groups
// 400, 353, 371 us (two: 103 TFLOP/s; a large fp32 product reaches 134 on this card), 16 of 32/8 behind 8192 49, 40, 50.
// The reference of the exponentials follows the maximum only when a step's weights sum up to more than 2^8.
typedef float pf_f32x4_t __attribute__((ext_vector_type(4)));
constexpr int kF32Keys = 16;         // of a step
constexpr float kPfGrowth = 256.0f;

template <int QG, int WAVES>
struct AttendF32Smem {
  float o[WAVES / 2][QG][32][64];
  float2 ml[WAVES][QG][16];
};

// Rows [r0, r1) (r0 < r1) of the cache at k, v, by the whole block.  query(i): query row i < 16 QG; part(i): where its part goes, or
// null; logits: as attend_rows', four rows of one query at a time (those at or past r1 are not there).
template <int QG, int WAVES, bool STREAM, typename Query, typename Part, typename Logits>
__device__ __forceinline__ void attend_f32(AttendF32Smem<QG, WAVES>& sm, const float* __restrict__ k, const float* __restrict__ v, int r0,
                                           int r1, Query query, Part part, Logits logits) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int l16 = lane & 15, c4 = lane >> 4;
  const float *kh = k + 4 * c4, *vh = v + 4 * l16;

  float4 q[QG][8];
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    const float* src = query(16 * g + l16) + 4 * c4;
#pragma unroll
    for (int j = 0; j < 8; ++j) q[g][j] = *reinterpret_cast<const float4*>(src + 16 * j);
  }
  float m[QG], l[QG];
  pf_f32x4_t o[QG][8];
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    m[g] = kNegBig;
    l[g] = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) o[g][c] = pf_f32x4_t{};
  }
  float4 kr[8], vr[4][2];
  auto load_k = [&](int at) __attribute__((always_inline)) {  // (past the end: the last row again)
    const float* p = kh + (size_t)min(at + l16, r1 - 1) * kD;
#pragma unroll
    for (int j = 0; j < 8; ++j) kr[j] = *reinterpret_cast<const float4*>(p + 16 * j);
  };
  auto load_v = [&](int at) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float* p = vh + (size_t)min(at + 4 * c4 + i, r1 - 1) * kD;
      vr[i][0] = __builtin_bit_cast(float4, load16_hint<STREAM>(p));
      vr[i][1] = __builtin_bit_cast(float4, load16_hint<STREAM>(p + 64));
    }
  };
  int at = r0 + wave * kF32Keys;
  if (at < r1) {  // (uniform for the wave)
    load_k(at);
    load_v(at);
  }
  for (; at < r1; at += WAVES * kF32Keys) {
    pf_f32x4_t s[QG], chain[QG][4];
#pragma unroll
    for (int g = 0; g < QG; ++g)
#pragma unroll
      for (int e = 0; e < 4; ++e) chain[g][e] = pf_f32x4_t{};
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int g = 0; g < QG; ++g) {
        chain[g][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[j].x, q[g][j].x, chain[g][0], 0, 0, 0);
        chain[g][1] = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[j].y, q[g][j].y, chain[g][1], 0, 0, 0);
        chain[g][2] = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[j].z, q[g][j].z, chain[g][2], 0, 0, 0);
        chain[g][3] = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[j].w, q[g][j].w, chain[g][3], 0, 0, 0);
      }
#pragma unroll
    for (int g = 0; g < QG; ++g)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[g][i] = (chain[g][0][i] + chain[g][1][i]) + (chain[g][2][i] + chain[g][3][i]);
    load_k(at + WAVES * kF32Keys);
#pragma unroll
    for (int g = 0; g < QG; ++g) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[g][i] = at + 4 * c4 + i < r1 ? s[g][i] * kSoftmaxScaleLog2 : kNegBig;
      if constexpr (Logits::kAny) logits(16 * g + l16, at + 4 * c4, make_float4(s[g][0], s[g][1], s[g][2], s[g][3]));
      float p[4], sum;
      auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = fast_exp2(s[g][i] - m[g]);
        sum = (p[0] + p[1]) + (p[2] + p[3]);
      };
      weights();
      if (__ballot(!(sum <= kPfGrowth)) != 0ull) {
        float top = fmaxf(fmaxf(s[g][0], s[g][1]), fmaxf(s[g][2], s[g][3]));
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float mn = fmaxf(m[g], top), corr = fast_exp2(m[g] - mn);
        m[g] = mn;
        l[g] *= corr;
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[g][c][i] *= corr;
        weights();
      }
      l[g] += sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) s[g][i] = p[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int g = 0; g < QG; ++g)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          o[g][4 * c] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr[i][c].x, s[g][i], o[g][4 * c], 0, 0, 0);
          o[g][4 * c + 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr[i][c].y, s[g][i], o[g][4 * c + 1], 0, 0, 0);
          o[g][4 * c + 2] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr[i][c].z, s[g][i], o[g][4 * c + 2], 0, 0, 0);
          o[g][4 * c + 3] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr[i][c].w, s[g][i], o[g][4 * c + 3], 0, 0, 0);
        }
    load_v(at + WAVES * kF32Keys);
  }

  // the waves' shares of the keys
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    l[g] += __shfl_xor(l[g], 16);
    l[g] += __shfl_xor(l[g], 32);
    if (c4 == 0) sm.ml[wave][g][l16] = make_float2(m[g], l[g]);
  }
  __syncthreads();
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    float mn = kNegBig, ls = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) mn = fmaxf(mn, sm.ml[w][g][l16].x);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) ls = fmaf(sm.ml[w][g][l16].y, fast_exp2(sm.ml[w][g][l16].x - mn), ls);
    const float f = fast_exp2(m[g] - mn);
    m[g] = mn;
    l[g] = ls;
#pragma unroll
    for (int c = 0; c < 8; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[g][c][i] *= f;
  }
#pragma unroll
  for (int n = WAVES / 2; n >= 1; n /= 2) {
    if (wave >= n && wave < 2 * n) {
#pragma unroll
      for (int g = 0; g < QG; ++g)
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) sm.o[wave - n][g][4 * c + i][lane] = o[g][c][i];
    }
    __syncthreads();
    if (wave < n) {
#pragma unroll
      for (int g = 0; g < QG; ++g)
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[g][c][i] += sm.o[wave][g][4 * c + i][lane];
    }
    __syncthreads();
  }
  if (wave != 0) return;
  // o[4 c + t][i] is column 64 c + 4 (4 c4 + i) + t of query l16
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    float* pr = part(16 * g + l16);
    if (pr == nullptr) continue;
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(pr + 64 * c + 16 * c4 + 4 * i) =
            make_float4(o[g][4 * c][i], o[g][4 * c + 1][i], o[g][4 * c + 2][i], o[g][4 * c + 3][i]);
    if (c4 == 0) *reinterpret_cast<float2*>(pr + kD) = make_float2(m[g], l[g]);
  }
}

// What a run's waves are joined through.
template <typename T, int NH, int WAVES>
using PartsSmem = std::conditional_t<T::EPC == 4 && parts_mfma<NH>(), AttendF32Smem<1, WAVES>, MergeSmem<WAVES, NH>>;

// One run by a block of WAVES waves: part at.place of the X that each query head of KV head h has.
template <typename T, int NH, bool LOGITS, bool STREAM, int WAVES>
__device__ __forceinline__ void parts_body(PartsSmem<T, NH, WAVES>& s_merge, float* kept, const RunAt& at, int run, int h, int X,
                                           const void* __restrict__ k, const void* __restrict__ v, const void* __restrict__ qv,
                                           float* __restrict__ partial, float* __restrict__ logits, size_t pitch, int Hkv, int S_cap) {
  using ST = typename T::store_t;
  constexpr bool MFMA = parts_mfma<NH>();
  const int tid = threadIdx.x, unit = at.b * Hkv + h;
  const int r0 = at.i * run, r1 = min(at.len, r0 + run);
  const size_t head0 = (size_t)unit * NH;
  const ST* q = static_cast<const ST*>(qv) + head0 * kD;
  float* lg = logits + head0 * pitch;
  if constexpr (MFMA && T::EPC == 4) {
    auto query = [&](int i) { return q + (size_t)min(i, NH - 1) * kD; };
    auto part = [&](int i) { return i < NH ? partial + ((size_t)(h * NH + i) * X + at.place) * kPartStride : nullptr; };
    const float *ku = static_cast<const float*>(k) + (size_t)unit * S_cap * kD, *vu = static_cast<const float*>(v) + (size_t)unit * S_cap * kD;
    auto& sm = s_merge;
    if constexpr (LOGITS)
      attend_f32<1, WAVES, STREAM>(sm, ku, vu, r0, r1, query, part, StoreSteps<NH>{lg, pitch});
    else
      attend_f32<1, WAVES, STREAM>(sm, ku, vu, r0, r1, query, part, NoLogits{});
  } else if constexpr (MFMA) {
    const int lane = tid & 63, r16 = lane & 15, kgrp = lane >> 4;
    am_bf16x8_t bq[4][1];
#pragma unroll
    for (int step = 0; step < 4; ++step) {
      uint4 raw = load16(q + (size_t)(r16 < NH ? r16 : 0) * kD + 32 * step + 8 * kgrp);
      if (r16 >= NH) raw = make_uint4(0, 0, 0, 0);
      bq[step][0] = __builtin_bit_cast(am_bf16x8_t, raw);
    }
    const AmAddr<4> ad = am_make_addr<4, false>(k, nullptr, v, (size_t)unit, S_cap, kD);
    AmState st;
    st.init();
    if constexpr (LOGITS) {
      KeepLogits<NH, WAVES> keep{lg, pitch, kept + (tid >> 6) * (kept_steps<NH>() * NH * kAmRows)};
      am_attend_rows<false, 4, 1, STREAM>(ad, bq, nullptr, r0, AmRoundRobin<WAVES>(r0, r1), st, [] {}, KeepIn<KeepLogits<NH, WAVES>>{&keep});
      keep.flush();
    } else
      am_attend_rows<false, 4, 1, STREAM>(ad, bq, nullptr, r0, AmRoundRobin<WAVES>(r0, r1), st, [] {});
    am_publish<NH, WAVES>(st, s_merge);
  } else {
    constexpr int EPC = T::EPC, LPRV = kD / EPC, RPW = 64 / LPRV;
    const int lane = tid & 63, wave = tid >> 6, c = lane % LPRV;
    float qr[NH][EPC];
#pragma unroll
    for (int g = 0; g < NH; ++g) T::unpack(load16(q + (size_t)g * kD + c * EPC), qr[g]);
    const RowAddr ra = make_row_addr<T, false>(k, nullptr, v, (size_t)unit, S_cap, kD, c);
    AttendAcc<T, NH> acc;
    acc.init();
    const int gid = wave * RPW + lane / LPRV;
    if constexpr (LOGITS)
      attend_rows<T, NH, WAVES * RPW, false, false, false, false, STREAM>(acc, qr, ra, nullptr, nullptr, gid, r0, r1,
                                                                             StoreLogits{lg, pitch, c == 0});
    else
      attend_rows<T, NH, WAVES * RPW, false, false, false, false, STREAM>(acc, qr, ra, nullptr, nullptr, gid, r0, r1);
    attend_publish<T, NH, WAVES>(acc, s_merge);
  }
  if constexpr (!(MFMA && T::EPC == 4)) {
    for (int i = tid; i < NH * kD; i += (64 * WAVES)) {
      const int g = i / kD, col = i % kD;
      float mn, ls, os;
      attend_merged<WAVES, NH>(s_merge, g, col, mn, ls, os);
      float* pr = partial + ((size_t)(h * NH + g) * X + at.place) * kPartStride;
      pr[col] = os;
      if (col == 0) {
        pr[kD] = mn;
        pr[kD + 1] = ls;
      }
    }
  }
}

}  // namespace loki
