// Attention over a cache held whole, contiguous or on pages (Section 2, Eq. 1 of arXiv 2406.02542), each token over the last rows of its
// sequence and the first few (span_impl.h): one token of every sequence, several, or chunks of prompts.
//
// Up to 16 query rows of a KV head (span_rows_kernel, span_f32_kernel): memory bounds it, a wave takes steps of rows straight from
// registers, a block's waves take steps in turn.  More, in bf16 (span_tiles_kernel): the matrix cores bound it, tiles of keys and
// values go through LDS for all of the block's query rows.
#include "span_tiles_impl.h"

#include <cmath>

namespace loki {

constexpr int kSpWaves = 4;

// ---- bf16, up to 16 query rows ------------------------------------------------------------------------------------
// A wave takes steps of 32 rows:
//   S[row, query] = K Q^T           v_mfma_f32_16x16x32_bf16, A = 16 bytes of a row for each lane (row, c), two tiles of 16 rows
//   O^T[column, query] += V^T P^T   lane (m, c) loads 16 bytes, columns 8 m .., of the 8 rows whose weights its own column of P has, and pairs
//                                   rows up (v_perm_b32); the weights in two bf16 terms, 2^-16 of each (as the library's other attention)
// so a query's maximum, sum and outputs are its own lanes'.  The reference of the exponentials follows the maximum only when a
// lane's weights of a step sum up to more than 2^8.  64 tokens of 64/8 heads over 4100 rows (1.08 GB) 165 us, 6.5 TB/s; one of 32/8 over 1028 6.1 us in front
// of the merge's 1.8.
template <bool STREAM, bool DEALT>
__global__ __launch_bounds__(64 * kSpWaves) void span_rows_kernel(SpanArgs a) {
  constexpr int KEYS = 32;
  __shared__ __align__(16) SpanMerge<16, kSpWaves> sm;
  const SpanTile tile = span_tile<KEYS, DEALT>(a);
  if (tile.h < 0) return;  // (uniform for the block)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), r16 = lane & 15, kgrp = lane >> 4;
  const int M = a.m * a.G, r0 = tile.tile * 16, live = min(16, M - r0), lg = 31 - __builtin_clz(a.G);
  const SpanRows rows = tile.rows;
  const SpanSteps<KEYS> steps(rows);
  if (tile.s0 >= tile.s1 && tile.part > 0) return span_none<DEALT>(a, tile, live);  // (uniform for the block)
  const int s1 = tile.s1;
  const RowPlaces places(a.cache, tile.b, tile.h, a.Hkv);
  const int len = r16 < live ? span_len(a, tile.b, (r0 + r16) >> lg) : 0;

  am_bf16x8_t bq[4];
  {
    const uint16_t* src = static_cast<const uint16_t*>(a.q) + span_place(a, tile.b, tile.h, r0 + min(r16, live - 1)) * kD + 8 * kgrp;
#pragma unroll
    for (int s = 0; s < 4; ++s) bq[s] = __builtin_bit_cast(am_bf16x8_t, load16(src + 32 * s));
  }
  float m = kNegBig, l = 0.f;
  am_f32x4_t o[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) o[c] = am_f32x4_t{};
  const char *kb = static_cast<const char*>(a.cache.k), *vb = static_cast<const char*>(a.cache.v);
  uint4 kraw[2][4], vraw[8];
  SpanPlaces<2> place;
  auto load_k = [&](const SpanStep& st) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const char* p = kb + (place.at[t] + span_near(st, t, r16)) * (kD * 2) + 16 * kgrp;
#pragma unroll
      for (int i = 0; i < 4; ++i) kraw[t][i] = load16(p + 64 * i);
    }
  };
  auto load_v = [&](const SpanStep& st) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) vraw[e] = load16_hint<STREAM>(vb + (place.at[e / 4] + span_near(st, e / 4, 4 * kgrp + e % 4)) * (kD * 2) + 16 * r16);
  };
  int s = tile.s0 + wave;
  if (s < s1) {  // (uniform for the wave)
    const SpanStep st = span_step(steps, rows, s);
    place.ask(places, st);
    place.settle(places, st);
    load_k(st);
    load_v(st);
    place.ask(places, span_step(steps, rows, min(s + kSpWaves, steps.total - 1)));
#pragma unroll
    for (int i = 0; i < 4; ++i) bq[i] = __builtin_bit_cast(am_bf16x8_t, span_query(__builtin_bit_cast(uint4, bq[i]), len));  // (rows are on their way)
  }
  for (; s < s1; s += kSpWaves) {
    const SpanStep st = span_step(steps, rows, s), next = span_step(steps, rows, min(s + kSpWaves, steps.total - 1));
    am_f32x4_t acc[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      acc[t] = am_f32x4_t{};
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(am_bf16x8_t, kraw[t][i]), bq[i], acc[t], 0, 0, 0);
    }
    place.settle(places, next);
    load_k(next);
    uint32_t seen = 0xffu;
    if (!span_full(a, rows, st, KEYS)) {  // (uniform)
      seen = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) seen |= (span_sees(a, st, len, st.at + 16 * (e / 4) + 4 * kgrp + e % 4) ? 1u : 0u) << e;
      uint32_t odd = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int w = 0; w < 4; ++w) odd |= bf16_not_finite(am_word(vraw[e], w));
      if (__ballot(odd != 0) != 0ull) {  // (span_mark)
        uint32_t ones[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) ones[i] = (seen >> (2 * i) & 1u ? 0x3f80u : 0u) | (seen >> (2 * i + 1) & 1u ? 0x3f800000u : 0u);
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          uint32_t x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            x[i] = bf16_marks(__builtin_amdgcn_perm(am_word(vraw[2 * i + 1], c / 2), am_word(vraw[2 * i], c / 2), c % 2 ? 0x07060302u : 0x05040100u));
          const am_f32x4_t count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(am_bf16x8_t, make_uint4(x[0], x[1], x[2], x[3])),
                                                                           __builtin_bit_cast(am_bf16x8_t, make_uint4(ones[0], ones[1], ones[2], ones[3])), am_f32x4_t{}, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) o[c][i] = span_mark(o[c][i], count[i]);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) vraw[e] = make_uint4(bf16_finite(vraw[e].x), bf16_finite(vraw[e].y), bf16_finite(vraw[e].z), bf16_finite(vraw[e].w));
      }
    }
    float p[8], sum;
    auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = seen >> e & 1u ? fast_exp2(fmaf(acc[e / 4][e % 4], kSoftmaxScaleLog2, -m)) : 0.f;
      sum = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    };
    weights();
    if (__ballot(!(sum <= kPfGrowth)) != 0ull) {
      float top = kNegBig;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, seen >> e & 1u ? acc[e / 4][e % 4] * kSoftmaxScaleLog2 : kNegBig);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float mn = fmaxf(m, top), corr = fast_exp2(m - mn);
      m = mn;
      l *= corr;
#pragma unroll
      for (int c = 0; c < 8; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[c][i] *= corr;
      weights();
    }
    l += sum;
    uint32_t w[2][4];  // the weights' two terms
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[0][i] = BF16::round2(p[2 * i], p[2 * i + 1]);
      w[1][i] = BF16::round2(p[2 * i] - __uint_as_float(w[0][i] << 16), p[2 * i + 1] - __uint_as_float(w[0][i] & 0xffff0000u));
    }
    const am_bf16x8_t b_hi = __builtin_bit_cast(am_bf16x8_t, make_uint4(w[0][0], w[0][1], w[0][2], w[0][3]));
    const am_bf16x8_t b_lo = __builtin_bit_cast(am_bf16x8_t, make_uint4(w[1][0], w[1][1], w[1][2], w[1][3]));
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      uint32_t x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        x[i] = __builtin_amdgcn_perm(am_word(vraw[2 * i + 1], c / 2), am_word(vraw[2 * i], c / 2), c % 2 ? 0x07060302u : 0x05040100u);
      const am_bf16x8_t av = __builtin_bit_cast(am_bf16x8_t, make_uint4(x[0], x[1], x[2], x[3]));
      o[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, b_lo, o[c], 0, 0, 0);
      o[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, b_hi, o[c], 0, 0, 0);
    }
    load_v(next);
    place.ask(places, span_step(steps, rows, min(s + 2 * kSpWaves, steps.total - 1)));
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (len == 0) {  // (a padded token's lanes took whatever full steps gave, a maximum too)
    m = kNegBig;
    l = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) o[c] = am_f32x4_t{};
  }
  if (kgrp == 0) sm.ml[wave][r16] = make_float2(m, l);
  // o[c][i] is column 8 (4 kgrp + i) + c
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float4* dst = reinterpret_cast<float4*>(&sm.o[wave][r16][8 * (4 * kgrp + i)]);
    dst[0] = make_float4(o[0][i], o[1][i], o[2][i], o[3][i]);
    dst[1] = make_float4(o[4][i], o[5][i], o[6][i], o[7][i]);
  }
  span_store<BF16, DEALT>(a, sm, tile, r0, live);
}

// ---- fp32 -----------------------------------------------------------------------------------------------------------
// The products of parts_impl.h's attend_f32, v_mfma_f32_16x16x4_f32, straight from registers, for QG groups of 16 query rows; steps of 16 rows.
// 5 x 3 tokens of 24 heads over 702 rows (86 MB, memory) 21.5 us with the merge; 2 x 512 tokens of 16/8 heads behind 4096 rows (keys and
// values again for each 32 query rows) 347 us, 105 TFLOP/s.
template <int QG, bool STREAM>
__global__ __launch_bounds__(64 * kSpWaves, 2) void span_f32_kernel(SpanArgs a) {
  constexpr int KEYS = 16;
  __shared__ __align__(16) SpanMerge<16 * QG, kSpWaves> sm;
  const SpanTile tile = span_tile<KEYS, false>(a);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l16 = lane & 15, c4 = lane >> 4;
  const int M = a.m * a.G, r0 = tile.tile * (16 * QG), live = min(16 * QG, M - r0), lg = 31 - __builtin_clz(a.G);
  const SpanRows rows = tile.rows;
  const SpanSteps<KEYS> steps(rows);
  if (tile.s0 >= tile.s1 && tile.part > 0) return span_none<false>(a, tile, live);  // (uniform for the block)
  const int s1 = tile.s1;
  const RowPlaces places(a.cache, tile.b, tile.h, a.Hkv);

  int len[QG];
  float4 q[QG][8];
  float m[QG], l[QG];
  pf_f32x4_t o[QG][8];
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    const int r = 16 * g + l16;
    len[g] = r < live ? span_len(a, tile.b, (r0 + r) >> lg) : 0;
    const float* src = static_cast<const float*>(a.q) + span_place(a, tile.b, tile.h, r0 + min(r, live - 1)) * kD + 4 * c4;
#pragma unroll
    for (int j = 0; j < 8; ++j) q[g][j] = *reinterpret_cast<const float4*>(src + 16 * j);
    m[g] = kNegBig;
    l[g] = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) o[g][c] = pf_f32x4_t{};
  }
  const char *kb = static_cast<const char*>(a.cache.k), *vb = static_cast<const char*>(a.cache.v);
  float4 kr[8], vr[4][2];
  SpanPlaces<1> place;
  auto load_k = [&](const SpanStep& st) __attribute__((always_inline)) {
    const char* p = kb + (place.at[0] + span_near(st, 0, l16)) * (kD * 4) + 16 * c4;
#pragma unroll
    for (int j = 0; j < 8; ++j) kr[j] = *reinterpret_cast<const float4*>(p + 64 * j);
  };
  auto load_v = [&](const SpanStep& st) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const char* p = vb + (place.at[0] + span_near(st, 0, 4 * c4 + i)) * (kD * 4) + 16 * l16;
      vr[i][0] = __builtin_bit_cast(float4, load16_hint<STREAM>(p));
      vr[i][1] = __builtin_bit_cast(float4, load16_hint<STREAM>(p + 256));
    }
  };
  int s = tile.s0 + wave;
  if (s < s1) {  // (uniform for the wave)
    const SpanStep st = span_step(steps, rows, s);
    place.ask(places, st);
    place.settle(places, st);
    load_k(st);
    load_v(st);
    place.ask(places, span_step(steps, rows, min(s + kSpWaves, steps.total - 1)));
#pragma unroll
    for (int g = 0; g < QG; ++g)
#pragma unroll
      for (int j = 0; j < 8; ++j) q[g][j] = __builtin_bit_cast(float4, span_query(__builtin_bit_cast(uint4, q[g][j]), len[g]));  // (rows are on their way)
  }
  for (; s < s1; s += kSpWaves) {
    const SpanStep st = span_step(steps, rows, s), next = span_step(steps, rows, min(s + kSpWaves, steps.total - 1));
    pf_f32x4_t p[QG], chain[QG][4];
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
    place.settle(places, next);
    load_k(next);
    const bool full = span_full(a, rows, st, KEYS);
#pragma unroll
    for (int g = 0; g < QG; ++g) {
      float x[4], sum;
      bool seen[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = ((chain[g][0][i] + chain[g][1][i]) + (chain[g][2][i] + chain[g][3][i])) * kSoftmaxScaleLog2;
        seen[i] = full || span_sees(a, st, len[g], st.at + 4 * c4 + i);
      }
      auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) p[g][i] = seen[i] ? fast_exp2(x[i] - m[g]) : 0.f;
        sum = (p[g][0] + p[g][1]) + (p[g][2] + p[g][3]);
      };
      weights();
      if (__ballot(!(sum <= kPfGrowth)) != 0ull) {
        float top = kNegBig;
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, seen[i] ? x[i] : kNegBig);
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
    }
    if (!full) {  // (uniform)
      uint32_t odd = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c) odd |= f32_not_finite(vr[i][c].x) | f32_not_finite(vr[i][c].y) | f32_not_finite(vr[i][c].z) | f32_not_finite(vr[i][c].w);
      if (__ballot(odd != 0) != 0ull) {  // (span_mark)
        uint32_t mine[QG];  // bit i: whether the lane's token sees the row
#pragma unroll
        for (int g = 0; g < QG; ++g) {
          mine[g] = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) mine[g] |= span_sees(a, st, len[g], st.at + 4 * c4 + i) ? 1u << i : 0u;
          asm volatile("" : "+v"(mine[g]));  // (else their masks stay in scalar registers, which there are too few of)
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            float ones[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float& x = t == 0 ? vr[i][c].x : t == 1 ? vr[i][c].y : t == 2 ? vr[i][c].z : vr[i][c].w;
              asm volatile("" : "+v"(x));  // (else what was found above is kept, in as many registers)
              const uint32_t bad = f32_not_finite(x);
              ones[i] = (float)bad;
              x = __uint_as_float(__float_as_uint(x) & (bad - 1u));
            }
#pragma unroll
            for (int g = 0; g < QG; ++g) {
              pf_f32x4_t count = pf_f32x4_t{};
#pragma unroll
              for (int i = 0; i < 4; ++i)
                count = __builtin_amdgcn_mfma_f32_16x16x4f32(ones[i], (float)(mine[g] >> i & 1u), count, 0, 0, 0);
#pragma unroll
              for (int i = 0; i < 4; ++i) o[g][4 * c + t][i] = span_mark(o[g][4 * c + t][i], count[i]);
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int g = 0; g < QG; ++g)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          o[g][4 * c] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr[i][c].x, p[g][i], o[g][4 * c], 0, 0, 0);
          o[g][4 * c + 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr[i][c].y, p[g][i], o[g][4 * c + 1], 0, 0, 0);
          o[g][4 * c + 2] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr[i][c].z, p[g][i], o[g][4 * c + 2], 0, 0, 0);
          o[g][4 * c + 3] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr[i][c].w, p[g][i], o[g][4 * c + 3], 0, 0, 0);
        }
    load_v(next);
    place.ask(places, span_step(steps, rows, min(s + 2 * kSpWaves, steps.total - 1)));
  }
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    l[g] += __shfl_xor(l[g], 16);
    l[g] += __shfl_xor(l[g], 32);
    if (len[g] == 0) {
      m[g] = kNegBig;
      l[g] = 0.f;
#pragma unroll
      for (int c = 0; c < 8; ++c) o[g][c] = pf_f32x4_t{};
    }
    const int r = 16 * g + l16;
    if (c4 == 0) sm.ml[wave][r] = make_float2(m[g], l[g]);
    // o[4 c + t][i] is column 64 c + 4 (4 c4 + i) + t
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(&sm.o[wave][r][64 * c + 16 * c4 + 4 * i]) = make_float4(o[g][4 * c][i], o[g][4 * c + 1][i], o[g][4 * c + 2][i], o[g][4 * c + 3][i]);
  }
  span_store<F32, false>(a, sm, tile, r0, live);
}

// ---- parts joined ---------------------------------------------------------------------------------------------------
// 32 lanes take a query row, 16 bytes of each of its parts; GROUPS of them share a row's parts, four each at a time.  A launch: 2 to 5 us.
template <typename T, int GROUPS, bool DEALT>
__global__ __launch_bounds__(256) void span_merge_kernel(SpanArgs a) {
  constexpr int U = 4;
  __shared__ __align__(16) float s_o[GROUPS > 1 ? GROUPS : 1][kD];
  __shared__ float2 s_ml[GROUPS];
  const int lane = threadIdx.x & 31, grp = threadIdx.x >> 5;
  const int r = GROUPS > 1 ? (int)blockIdx.x : (int)blockIdx.x * 8 + grp;
  if (GROUPS == 1 && r >= a.B * a.m * a.Hq) return;
  int nsplit = a.nsplit;
  long long between = kPartStride;
  const float* partial = a.partial + (long long)r * nsplit * kPartStride;
  if constexpr (DEALT) {
    const int per = a.m * a.Hq, b = r / per, j = (r - b * per) / a.Hq, head = r - b * per - j * a.Hq, h = head >> (31 - __builtin_clz(a.G));
    const int row = j * a.G + (head & (a.G - 1)), tile = row >> (31 - __builtin_clz(a.rows));
    const int2 dealt = a.dealt[span_tile_index(a, b, tile)];
    nsplit = dealt.y;
    if (nsplit == 1) return;  // (written already)
    between = (long long)a.Hkv * a.rows * kPartStride;
    partial = a.partial + dealt.x * between + ((long long)h * a.rows + (row & (a.rows - 1))) * kPartStride;
  }
  typename T::store_t* out = static_cast<typename T::store_t*>(a.out) + (long long)r * kD;
  float m = kNegBig, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i0 = GROUPS > 1 ? grp : 0; i0 < nsplit; i0 += GROUPS * U) {
    float2 ml[U];
    float4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * GROUPS;
      const float* p = partial + (i < nsplit ? i : i0) * between;
      ml[u] = *reinterpret_cast<const float2*>(p + kD);
      x[u] = *reinterpret_cast<const float4*>(p + 4 * lane);
      if (i >= nsplit) ml[u] = make_float2(kNegBig, 0.f);
    }
    float mn = m;
#pragma unroll
    for (int u = 0; u < U; ++u) mn = fmaxf(mn, ml[u].x);
    const float c = fast_exp2(m - mn);
    m = mn;
    l *= c;
    o = make_float4(o.x * c, o.y * c, o.z * c, o.w * c);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float f = fast_exp2(ml[u].x - mn);
      if (ml[u].y != 0.f) {  // (a part without rows has no outputs)
        l = fmaf(ml[u].y, f, l);
        o = make_float4(fmaf(x[u].x, f, o.x), fmaf(x[u].y, f, o.y), fmaf(x[u].z, f, o.z), fmaf(x[u].w, f, o.w));
      }
    }
  }
  if constexpr (GROUPS > 1) {
    *reinterpret_cast<float4*>(&s_o[grp][4 * lane]) = o;
    if (lane == 0) s_ml[grp] = make_float2(m, l);
    __syncthreads();
    if (grp != 0) return;
    float mn = kNegBig;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) mn = fmaxf(mn, s_ml[g].x);
    l = 0.f;
    o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      const float f = fast_exp2(s_ml[g].x - mn);
      const float4 x = *reinterpret_cast<const float4*>(&s_o[g][4 * lane]);
      l = fmaf(s_ml[g].y, f, l);
      o = make_float4(fmaf(x.x, f, o.x), fmaf(x.y, f, o.y), fmaf(x.z, f, o.z), fmaf(x.w, f, o.w));
    }
  }
  const float inv = l == 0.f ? 0.f : 1.0f / l;  // (a token without rows: zeros)
  if constexpr (T::EPC == 8)
    *reinterpret_cast<uint2*>(out + 4 * lane) = make_uint2(BF16::round2(o.x * inv, o.y * inv), BF16::round2(o.z * inv, o.w * inv));
  else
    *reinterpret_cast<float4*>(out + 4 * lane) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
}

// ---- the launch -----------------------------------------------------------------------------------------------------
// Parts of a tile's rows, of at least 128: as many as make whole rounds of the blocks that are resident together, since one block more than a round
// costs another (up to a few rounds; 3 % of a round for the parts that more of them write and the merge reads).  us with the fewest that fill a round / so:
// 13 sequences of 32/8 bf16 heads with 4000 rows 49.2 / 42.3, 5 of 24 51.8 / 45.9, in 4 bits 24.3 / 21.4, 700 tokens of 32/8 behind 8192 rows 207 / 175; but
// where lengths leave some of the blocks without rows, 5 of 24 fp32 heads up to 2311 in 4 bits 17.4 / 18.4.  Never fewer for more rows.
static int span_splits(long long blocks, long long slots, long long most) {
  if (blocks >= 2 * slots) return 1;
  const double share = (double)slots / (double)blocks;
  double best = 1e30;
  int n = 1;
  for (int rounds = 1; rounds <= 3; ++rounds) {
    double parts = floor(rounds * share);
    if (parts > sqrt(rounds * share / 0.03)) parts = floor(sqrt(rounds * share / 0.03));  // (where one more costs what it gains)
    if (parts > (double)most) parts = (double)most;
    if (parts < 1.0) continue;
    const double cost = rounds / parts + 0.03 * (parts - 1.0) / share;
    if (cost < best) {
      best = cost;
      n = (int)parts;
    }
  }
  return n;
}

// Which kernel and how many blocks.  Tiles through LDS from 65 query rows of a KV head on (in 4 bits from 81), and from 33 on where more than 33 MB
// are read, us 16 rows at a time / so: 1 x 64 tokens of 8/8 heads, window 512 9.3 / 13.5, 2 x 8 of 64/8, window 1000 13.7 / 16.5, 4000 (33 MB) 19.3 / 19.9,
// 8 x 16 of 32/8 up to 8192 rows 93.2 / 54.8; with 32 query rows 8 x 4 of 64/8, window 1000 15.9 / 18.6, 2000 22.4 / 24.2, 8192 60.1 / 57.5; in 4 bits, 8192
// rows, 4 x 20 tokens of 32/8 (80 query rows) 54.0 / 52.9, of lengths from a quarter on 45.1 / 52.3, 4 x 32 (128) of such 72.8 / 54.7, 4 x 64 132 / 92.8.
SpanPlan span_plan(const Shape& s, int m, int window, int sinks, bool bits4, bool short_rows) {
  SpanPlan p{};
  p.rows = 16;
  const long long M = (long long)m * s.G;
  const long long tokens_read = window > 0 ? (long long)window + m - 1 + sinks : s.S, most_read = tokens_read < s.S ? tokens_read : s.S;
  const double bytes = (double)s.B * s.Hkv * most_read * (2 * kD * s.elem_bytes);
  const bool lds = s.dtype == 1 && (M > (bits4 ? 80 : 64) || (!bits4 && M > 32 && bytes > 33e6 && !short_rows));
  if (lds)
    p.rows = M <= 64 ? 64 : M <= 128 ? 128 : 256;
  else if (bits4)
    p.rows = M <= 4 ? 4 : M <= 8 ? 8 : 16;
  else if (s.dtype == 0 && M > 16)
    p.rows = 32;
  p.tiles = (int)((M + p.rows - 1) / p.rows);
  // a tile's rows at most: its tokens' windows and the sinks
  const long long tokens = p.rows < M ? (p.rows + s.G - 1) / s.G + 1 : m, most = (long long)window + tokens - 1 + sinks;
  const long long read = window > 0 && most < s.S ? most : s.S, blocks = (long long)s.B * p.tiles * s.Hkv;
  // as many parts as fill the blocks that are resident together, by the kernels' registers
  const long long slots = (lds ? 1LL : bits4 ? span_q4_waves(s.dtype == 1, p.rows) : s.dtype == 0 && p.rows == 16 ? 3LL : 2LL) * device_cus();
  // From 90 MB of rows on, of which none is read twice, values are loaded past the caches (row_loads in api.hip).  us through / past: 64
  // sequences of 64/8 heads with 4100 rows each 180 / 163, 16 of 32/8 with 16384 186 / 166, 13 with 4000 51.4 / 47.8, with 1500 (80 MB) 21.3 / 21.6;
  // fp32, 16 of 24 heads with 1000 rows 74.5 / 68.1, 5 with 703 (86 MB) 22.7 / 23.4.
  const bool large = (double)blocks * read * (bits4 ? 2.0 * (kQ4RowBytes + kQ4ScaleBytes) : 2.0 * kD * s.elem_bytes) >= kPastBytes;
  p.past = p.tiles == 1 && large;
  p.nsplit = span_splits(blocks, slots, (read + 127) / 128);
  if (p.rows == 256 && blocks >= slots && blocks <= 8 * slots) {
    p.nsplit = 1;
    p.halves = (int)slots;
  }
  p.run = (int)((read + p.nsplit - 1) / p.nsplit);
  p.parts = p.nsplit > 1 ? (size_t)s.B * m * s.G * s.Hkv * p.nsplit : 0;
  // Runs are dealt by the lengths where a round of blocks holds two and more of each tile and the call is long enough for what it costs, about 1 us: us
  // by the longest length / so, with lengths from a quarter of it on: in 4 bits, 16 sequences of 32/8 bf16 heads up to 16384 rows 53.1 / 44.5, 40 up to 3000
  // 31.8 / 26.3, of 8 fp32 heads 38.3 / 30.1, 8 of 64/8 up to 4000 (41 MB) 17.0 / 16.6, up to 2000 13.0 / 14.0, 4 of 32/8 up to 4096 (21 MB) 12.8 / 13.2; in bf16, 16 of
  // 32/8 up to 16384 129 / 124, 5 up to 8000 29.0 / 28.0; in fp32 none gained, 8 of 8 up to 2000 25.8 / 26.6.
  const bool deals = bits4 ? !lds && (double)blocks * read * 2.0 * (kQ4RowBytes + kQ4ScaleBytes) >= 33e6 : s.dtype == 1 && p.rows == 16 && p.past;
  const long long tiles = (long long)s.B * p.tiles, all = tiles * ((read + 127) / 128), round = slots / s.Hkv, cap = round < all ? round : all;
  if (tiles > 1 && tiles <= 64) {
    if (deals && cap >= 2 * tiles) p.cap = (int)cap;
    p.dealt = (size_t)tiles;
    const size_t parts = (size_t)cap * s.Hkv * p.rows;
    if (p.parts < parts) p.parts = parts;
  }
  return p;
}

hipError_t launch_span_q4(const Shape& s, const SpanArgs& a, unsigned blocks, bool past, hipStream_t st);

template <typename T, bool DEALT>
static void launch_span_merge(const SpanArgs& a, int runs, hipStream_t st) {
  const unsigned rows = (unsigned)(a.B * a.m * a.Hq);
  if (runs <= 4 * a.B * a.tiles)
    hipLaunchKernelGGL((span_merge_kernel<T, 1, DEALT>), dim3((rows + 7) / 8), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((span_merge_kernel<T, 8, DEALT>), dim3(rows), dim3(256), 0, st, a);
}
template <typename T>
static void launch_span_merge(const SpanArgs& a, int runs, hipStream_t st) {
  if (a.dealt != nullptr)
    launch_span_merge<T, true>(a, runs, st);
  else
    launch_span_merge<T, false>(a, runs, st);
}

hipError_t launch_span(const Shape& s, SpanArgs a, const SpanPlan& plan, hipStream_t st) {
  const bool bits4 = a.cache.k_scales != nullptr;
  if (a.window == 0) {
    a.window = 0x7fffffff;
    a.sinks = 0;
  }
  a.rows = plan.rows;
  a.tiles = plan.tiles;
  a.nsplit = plan.nsplit;
  a.run = plan.run;
  a.cap = plan.cap;
  a.halves = plan.halves;
  const int tiles = a.B * a.tiles, runs = a.dealt != nullptr ? a.cap : tiles * a.nsplit;
  a.halves_all = a.halves > 0 && a.window == 0x7fffffff && runs * a.Hkv < 2 * a.halves;  // (only tiles that see all rows differ that much)
  const unsigned blocks = (unsigned)((long long)runs * a.Hkv) + (a.halves_all ? runs * a.Hkv : a.halves / 2);
  const dim3 grid(blocks), block(64 * kSpWaves);
  hipError_t e = hipSuccess;
  if (bits4)
    e = launch_span_q4(s, a, blocks, plan.past, st);
  else if (s.dtype == 0 && plan.rows == 16 && plan.past)
    hipLaunchKernelGGL((span_f32_kernel<1, true>), grid, block, 0, st, a);
  else if (s.dtype == 0 && plan.rows == 16)
    hipLaunchKernelGGL((span_f32_kernel<1, false>), grid, block, 0, st, a);
  else if (s.dtype == 0)
    hipLaunchKernelGGL((span_f32_kernel<2, false>), grid, block, 0, st, a);
  else if (plan.rows == 16 && a.dealt != nullptr)
    hipLaunchKernelGGL((span_rows_kernel<true, true>), grid, block, 0, st, a);
  else if (plan.rows == 16 && plan.past)
    hipLaunchKernelGGL((span_rows_kernel<true, false>), grid, block, 0, st, a);
  else if (plan.rows == 16)
    hipLaunchKernelGGL((span_rows_kernel<false, false>), grid, block, 0, st, a);
  else if (plan.rows == 64)
    e = launch_span_tiles<8, 2, false>(a, blocks, st);
  else if (plan.rows == 128)
    e = launch_span_tiles<8, 4, false>(a, blocks, st);
  else if (a.halves == 0)
    e = launch_span_tiles<8, 8, false>(a, blocks, st);
  else
    e = launch_span_tiles<8, 8, false, true>(a, blocks, st);
  if (e == hipSuccess) e = hipGetLastError();
  if (e != hipSuccess || (a.dealt == nullptr && a.nsplit == 1)) return e;
  if (s.dtype == 1)
    launch_span_merge<BF16>(a, runs, st);
  else
    launch_span_merge<F32>(a, runs, st);
  return hipGetLastError();
}

}  // namespace loki
