// Attention over a cache held whole in 4 bits (cache_impl.h), contiguous or on pages (Section 2, Eq. 1 of arXiv 2406.02542), each token over
// the last rows of its sequence and the first few (span_impl.h).
//
// A value is lowest + step n with one (step, lowest) for a row's group g of 32 columns, so
//   logit[row] = sum over g of 16 step_g[row] sum over c in g of q[c] n[row, c] / 16 + lowest_g[row] sum over c in g of q[c]
//   out[c]     = sum over rows of (16 p step_g)[row] n[row, c] / 16 + sum over rows of (p lowest_g)[row]          for c in g
// and the codes go to the matrix cores as they are: the bits 0x3f80 | n << 3 are the bf16 number 1 + n / 16, exactly, a shift and a bit
// select for two of them.  The ones' share is taken off in advance (the first product begins with minus the group's sum of q) or
// at the end (sum over rows of 16 p step_g).
#include "span_impl.h"

namespace loki {

constexpr int kQ4Waves = 4;

// Codes g of a word's halves as two bf16 numbers 1 + n / 16.  The constants are kept in registers: one instruction takes both then.
struct Q4Pair {
  uint32_t mask = 0x00780078u, one = 0x3f803f80u;
  __device__ __forceinline__ Q4Pair() { asm("" : "+v"(mask), "+s"(one)); }
  __device__ __forceinline__ uint32_t operator()(uint32_t x, int g) const { return ((g == 0 ? x << 3 : x >> (4 * g - 3)) & mask) | one; }
};

template <bool STREAM>
__device__ __forceinline__ uint32_t load4_hint(const void* p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(static_cast<const uint32_t*>(p));
  return *static_cast<const uint32_t*>(p);
}

// x0, x1 as TERMS pairs of bf16 numbers that add up to them.
template <int TERMS>
__device__ __forceinline__ void q4_terms(float x0, float x1, uint32_t (&w)[TERMS]) {
#pragma unroll
  for (int t = 0; t < TERMS; ++t) {
    w[t] = BF16::round2(x0, x1);
    x0 -= __uint_as_float(w[t] << 16);  // exact in fp32
    x1 -= __uint_as_float(w[t] & 0xffff0000u);
  }
}

// Up to 4 NS query rows, as most calls with one token have.  Lane n = 4 r + g of the matrix cores' 16 columns is row r in group g, NS sets of them:
//   first product   column n holds q[r] in the columns of group g and zeros elsewhere, so that the four products add up to each lane's own
//                   group's sum, which takes one step and one lowest for a row; the four lanes of a query add theirs (DPP)
//   second          column n holds p step_g, so a lane forms its own group's only; it keeps the two output tiles of its group
// which leaves a quarter of the scaling and of the splitting into terms that whole columns for a query would ask of every lane: 24
// vector instructions a row of keys and values for all 64 lanes against 40 of the kernel below.
template <typename T, int NS, bool STREAM>
__global__ __launch_bounds__(64 * kQ4Waves, T::EPC == 8 && NS == 1 ? 3 : 2) void span_q4_few_kernel(SpanArgs a) {
  constexpr int KEYS = 32, QT = T::EPC == 8 ? 1 : 3, PT = T::EPC == 8 ? 2 : 3, ROWS = 4 * NS;
  __shared__ __align__(16) SpanMerge<ROWS, kQ4Waves> sm;
  const SpanTile tile = span_tile<KEYS>(a);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), r16 = lane & 15, kgrp = lane >> 4;
  const int g = r16 & 3, hd = r16 >> 2;
  const int M = a.m * a.G, r0 = tile.tile * ROWS, live = min(ROWS, M - r0), lg = 31 - __builtin_clz(a.G);
  const SpanRows rows = tile.rows;
  const SpanSteps<KEYS> steps(rows);
  if (tile.s0 >= tile.s1 && tile.part > 0) return span_none(a, tile, live);  // (uniform for the block)
  const int s1 = tile.s1;
  const RowPlaces places(a.cache, tile.b, tile.h, a.Hkv);
  const Q4Pair q4_pair;

  const char *kb = static_cast<const char*>(a.cache.k), *vb = static_cast<const char*>(a.cache.v);
  const char *ks = static_cast<const char*>(a.cache.k_scales), *vs = static_cast<const char*>(a.cache.v_scales);
  const int k_row = 4 * (r16 & 3) + (r16 >> 2);  // (see the head of this file)
  const unsigned k_at = k_row * kQ4RowBytes + 16 * kgrp, v_at = kgrp * kQ4RowBytes + 4 * r16, s_at = kgrp * kQ4ScaleBytes + 4 * g;
  uint4 kraw[2];
  uint32_t ksc[8], vsc[8], vraw[8];
  SpanPlaces<2> place;
  auto load = [&](const SpanStep& st, auto values) __attribute__((always_inline)) {
    constexpr bool V = decltype(values)::value;
    const char *codes = V ? vb : kb, *scales = V ? vs : ks;
    uint32_t(&sc)[8] = V ? vsc : ksc;
    span_loads<KEYS>(st, [&](auto whole) __attribute__((always_inline)) {
      constexpr bool W = decltype(whole)::value;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const char *c = codes + place.at[t] * kQ4RowBytes, *x = scales + place.at[t] * kQ4ScaleBytes;
        if constexpr (!V) kraw[t] = load16_hint<STREAM>(W ? c + k_at : c + span_near(st, t, k_row) * kQ4RowBytes + 16 * kgrp);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = W ? 0 : span_near(st, t, 4 * i + kgrp);
          sc[4 * t + i] = *reinterpret_cast<const uint32_t*>(W ? x + s_at + 4 * i * kQ4ScaleBytes : x + row * kQ4ScaleBytes + 4 * g);
          if constexpr (V) vraw[4 * t + i] = load4_hint<STREAM>(W ? c + v_at + 4 * i * kQ4RowBytes : c + row * kQ4RowBytes + 4 * r16);
        }
      }
    });
  };
  int s = tile.s0 + wave;
  if (s < s1) {  // (uniform for the wave)
    const SpanStep st = span_step(steps, rows, s);
    place.ask(places, st);
    place.settle(places, st);
    load(st, std::false_type{});
    load(st, std::true_type{});
    place.ask(places, span_step(steps, rows, min(s + kQ4Waves, steps.total - 1)));
  }

  int len[NS];
  am_bf16x8_t bq[NS][kQ4Groups][QT];
  float qsum[NS], m[NS], l[NS], low[NS], ones[NS];  // qsum: of the group's columns
  am_f32x4_t o[NS][8];
#pragma unroll
  for (int u = 0; u < NS; ++u) {
    const int r = 4 * u + hd;
    len[u] = r < live ? span_len(a, tile.b, (r0 + r) >> lg) : 0;
    const typename T::store_t* src =
        static_cast<const typename T::store_t*>(a.q) + span_place(a, tile.b, tile.h, r0 + min(r, live - 1)) * kD + 32 * g + 8 * kgrp;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; e += T::EPC) T::unpack(load16(src + e), *reinterpret_cast<float(*)[T::EPC]>(x + e));
    uint32_t w[4][QT];
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      q4_terms<QT>(x[2 * i], x[2 * i + 1], w[i]);
      sum += x[2 * i] + x[2 * i + 1];
    }
#pragma unroll
    for (int G = 0; G < kQ4Groups; ++G)
#pragma unroll
      for (int t = 0; t < QT; ++t)
        bq[u][G][t] = __builtin_bit_cast(am_bf16x8_t, G == g ? make_uint4(w[0][t], w[1][t], w[2][t], w[3][t]) : make_uint4(0, 0, 0, 0));
    sum += __shfl_xor(sum, 16);
    qsum[u] = sum + __shfl_xor(sum, 32);
    m[u] = kNegBig;
    l[u] = low[u] = ones[u] = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) o[u][c] = am_f32x4_t{};
  }

  for (; s < s1; s += kQ4Waves) {
    const SpanStep st = span_step(steps, rows, s), next = span_step(steps, rows, min(s + kQ4Waves, steps.total - 1));
    float x[NS][8];  // a sixteenth of the logits
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      am_f32x4_t acc[NS];
#pragma unroll
      for (int u = 0; u < NS; ++u) acc[u] = am_f32x4_t{-qsum[u], -qsum[u], -qsum[u], -qsum[u]};
#pragma unroll
      for (int G = 0; G < kQ4Groups; ++G) {
        const am_bf16x8_t ka = __builtin_bit_cast(am_bf16x8_t, make_uint4(q4_pair(kraw[t].x, G), q4_pair(kraw[t].y, G), q4_pair(kraw[t].z, G), q4_pair(kraw[t].w, G)));
#pragma unroll
        for (int u = 0; u < NS; ++u)
#pragma unroll
          for (int i = QT - 1; i >= 0; --i) acc[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, bq[u][G][i], acc[u], 0, 0, 0);
      }
#pragma unroll
      for (int u = 0; u < NS; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const cache_half2_t sc = __builtin_bit_cast(cache_half2_t, ksc[4 * t + i]);
          x[u][4 * t + i] = group_allreduce_sum<4>(fmaf((float)sc.x, acc[u][i], (float)sc.y * (qsum[u] * 0.0625f)));
        }
    }
    place.settle(places, next);
    load(next, std::false_type{});
    const bool full = span_full(a, rows, st, KEYS);
    float p[NS][8];
#pragma unroll
    for (int u = 0; u < NS; ++u) {
      if (!full) {  // (uniform)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!span_sees(a, st, len[u], st.at + 16 * (e / 4) + 4 * (e % 4) + kgrp)) x[u][e] = kUnseen;
      }
      float sum;
      auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) p[u][e] = fast_exp2(fmaf(x[u][e], 16.f * kSoftmaxScaleLog2, -m[u]));
        sum = ((p[u][0] + p[u][1]) + (p[u][2] + p[u][3])) + ((p[u][4] + p[u][5]) + (p[u][6] + p[u][7]));
      };
      weights();
      if (__ballot(!(sum <= kPfGrowth)) != 0ull) {
        float top = x[u][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = fmaxf(top, x[u][e]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32)) * (16.f * kSoftmaxScaleLog2);
        const float mn = fmaxf(m[u], top), corr = fast_exp2(m[u] - mn);
        m[u] = mn;
        l[u] *= corr;
        low[u] *= corr;
        ones[u] *= corr;
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[u][c][i] *= corr;
        weights();
      }
      l[u] += sum;
    }
    am_bf16x8_t b[NS][PT];
#pragma unroll
    for (int u = 0; u < NS; ++u) {
      uint32_t w[4][PT];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const cache_half2_t sc0 = __builtin_bit_cast(cache_half2_t, vsc[2 * i]), sc1 = __builtin_bit_cast(cache_half2_t, vsc[2 * i + 1]);
        const float p0 = p[u][2 * i], p1 = p[u][2 * i + 1], x0 = p0 * (float)sc0.x, x1 = p1 * (float)sc1.x;
        ones[u] += x0 + x1;
        low[u] = fmaf(p0, (float)sc0.y, fmaf(p1, (float)sc1.y, low[u]));
        q4_terms<PT>(x0, x1, w[i]);
      }
#pragma unroll
      for (int t = 0; t < PT; ++t) b[u][t] = __builtin_bit_cast(am_bf16x8_t, make_uint4(w[0][t], w[1][t], w[2][t], w[3][t]));
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      uint32_t y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = __builtin_amdgcn_perm(vraw[2 * i + 1], vraw[2 * i], c ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int G = 0; G < kQ4Groups; ++G) {
        const am_bf16x8_t av = __builtin_bit_cast(am_bf16x8_t, make_uint4(q4_pair(y[0], G), q4_pair(y[1], G), q4_pair(y[2], G), q4_pair(y[3], G)));
#pragma unroll
        for (int u = 0; u < NS; ++u)
#pragma unroll
          for (int t = PT - 1; t >= 0; --t) o[u][2 * G + c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, b[u][t], o[u][2 * G + c], 0, 0, 0);
      }
    }
    load(next, std::true_type{});
    place.ask(places, span_step(steps, rows, min(s + 2 * kQ4Waves, steps.total - 1)));
  }
#pragma unroll
  for (int u = 0; u < NS; ++u) {
    const int r = 4 * u + hd;
    l[u] += __shfl_xor(l[u], 16);
    l[u] += __shfl_xor(l[u], 32);
    if (len[u] == 0) l[u] = 0.f;  // (a padded token's lanes took whatever full steps gave)
    if (kgrp == 0 && g == 0) sm.ml[wave][r] = make_float2(m[u], l[u]);
    float base = low[u] - 16.f * ones[u];
    base += __shfl_xor(base, 16);
    base += __shfl_xor(base, 32);
    // o[2 g + c][i] is column 32 g + 2 (4 kgrp + i) + c
    float y[2][4];
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float mine = g < 2 ? (g == 0 ? o[u][c][i] : o[u][2 + c][i]) : (g == 2 ? o[u][4 + c][i] : o[u][6 + c][i]);
        y[c][i] = fmaf(16.f, mine, base);
      }
#pragma unroll
    for (int i = 0; i < 4; i += 2)
      *reinterpret_cast<float4*>(&sm.o[wave][r][32 * g + 8 * kgrp + 2 * i]) = make_float4(y[0][i], y[1][i], y[0][i + 1], y[1][i + 1]);
  }
  span_store<T>(a, sm, tile, r0, live);
}

// QG groups of 16 query rows.  bf16: q is one term, the weights two (2^-16 of each, as the library's other attention); fp32: three each.
template <typename T, int QG>
__global__ __launch_bounds__(64 * kQ4Waves, QG == 1 ? 2 : 1) void span_q4_kernel(SpanArgs a) {
  constexpr int KEYS = 32, QT = T::EPC == 8 ? 1 : 3, PT = T::EPC == 8 ? 2 : 3;
  __shared__ __align__(16) SpanMerge<16 * QG, kQ4Waves> sm;
  const SpanTile tile = span_tile<KEYS>(a);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), r16 = lane & 15, kgrp = lane >> 4;
  const int M = a.m * a.G, r0 = tile.tile * (16 * QG), live = min(16 * QG, M - r0), lg = 31 - __builtin_clz(a.G);
  const SpanRows rows = tile.rows;
  const SpanSteps<KEYS> steps(rows);
  if (tile.s0 >= tile.s1 && tile.part > 0) return span_none(a, tile, live);  // (uniform for the block)
  const int s1 = tile.s1;
  const RowPlaces places(a.cache, tile.b, tile.h, a.Hkv);
  const Q4Pair q4_pair;

  int len[QG];
  am_bf16x8_t bq[QG][kQ4Groups][QT];
  float qsum[QG][kQ4Groups];  // of a group's columns
  float m[QG], l[QG], low[QG][kQ4Groups], ones[QG][kQ4Groups];
  am_f32x4_t o[QG][8];
#pragma unroll
  for (int u = 0; u < QG; ++u) {
    const int r = 16 * u + r16;
    len[u] = r < live ? span_len(a, tile.b, (r0 + r) >> lg) : 0;
    const typename T::store_t* src = static_cast<const typename T::store_t*>(a.q) + span_place(a, tile.b, tile.h, r0 + min(r, live - 1)) * kD + 8 * kgrp;
#pragma unroll
    for (int g = 0; g < kQ4Groups; ++g) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; e += T::EPC) T::unpack(load16(src + 32 * g + e), *reinterpret_cast<float(*)[T::EPC]>(x + e));
      uint32_t w[4][QT];
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        q4_terms<QT>(x[2 * i], x[2 * i + 1], w[i]);
        sum += x[2 * i] + x[2 * i + 1];
      }
#pragma unroll
      for (int t = 0; t < QT; ++t) bq[u][g][t] = __builtin_bit_cast(am_bf16x8_t, make_uint4(w[0][t], w[1][t], w[2][t], w[3][t]));
      sum += __shfl_xor(sum, 16);
      qsum[u][g] = sum + __shfl_xor(sum, 32);
      low[u][g] = ones[u][g] = 0.f;
    }
    m[u] = kNegBig;
    l[u] = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) o[u][c] = am_f32x4_t{};
  }

  const char *kb = static_cast<const char*>(a.cache.k), *vb = static_cast<const char*>(a.cache.v);
  const char *ks = static_cast<const char*>(a.cache.k_scales), *vs = static_cast<const char*>(a.cache.v_scales);
  const int k_row = 4 * (r16 & 3) + (r16 >> 2);
  const unsigned k_at = k_row * kQ4RowBytes + 16 * kgrp, v_at = kgrp * kQ4RowBytes + 4 * r16, s_at = kgrp * kQ4ScaleBytes;
  uint4 kraw[2], ksc[8], vsc[8];
  uint32_t vraw[8];
  SpanPlaces<2> place;
  auto load = [&](const SpanStep& st, auto values) __attribute__((always_inline)) {
    constexpr bool V = decltype(values)::value;
    const char *codes = V ? vb : kb, *scales = V ? vs : ks;
    uint4(&sc)[8] = V ? vsc : ksc;
    span_loads<KEYS>(st, [&](auto whole) __attribute__((always_inline)) {
      constexpr bool W = decltype(whole)::value;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const char *c = codes + place.at[t] * kQ4RowBytes, *x = scales + place.at[t] * kQ4ScaleBytes;
        if constexpr (!V) kraw[t] = load16(W ? c + k_at : c + span_near(st, t, k_row) * kQ4RowBytes + 16 * kgrp);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = W ? 0 : span_near(st, t, 4 * i + kgrp);
          sc[4 * t + i] = load16(W ? x + s_at + 4 * i * kQ4ScaleBytes : x + row * kQ4ScaleBytes);
          if constexpr (V) vraw[4 * t + i] = *reinterpret_cast<const uint32_t*>(W ? c + v_at + 4 * i * kQ4RowBytes : c + row * kQ4RowBytes + 4 * r16);
        }
      }
    });
  };
  int s = tile.s0 + wave;
  if (s < s1) {  // (uniform for the wave)
    const SpanStep st = span_step(steps, rows, s);
    place.ask(places, st);
    place.settle(places, st);
    load(st, std::false_type{});
    load(st, std::true_type{});
    place.ask(places, span_step(steps, rows, min(s + kQ4Waves, steps.total - 1)));
  }
  for (; s < s1; s += kQ4Waves) {
    const SpanStep st = span_step(steps, rows, s), next = span_step(steps, rows, min(s + kQ4Waves, steps.total - 1));
    float x[QG][8];
#pragma unroll
    for (int u = 0; u < QG; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[u][e] = 0.f;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int g = 0; g < kQ4Groups; ++g) {
        const am_bf16x8_t ka = __builtin_bit_cast(am_bf16x8_t, make_uint4(q4_pair(kraw[t].x, g), q4_pair(kraw[t].y, g), q4_pair(kraw[t].z, g), q4_pair(kraw[t].w, g)));
#pragma unroll
        for (int u = 0; u < QG; ++u) {
          am_f32x4_t acc = {-qsum[u][g], -qsum[u][g], -qsum[u][g], -qsum[u][g]};
#pragma unroll
          for (int i = QT - 1; i >= 0; --i) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, bq[u][g][i], acc, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const cache_half2_t sc = __builtin_bit_cast(cache_half2_t, am_word(ksc[4 * t + i], g));
            x[u][4 * t + i] = fmaf(acc[i], 16.f * (float)sc.x, fmaf(qsum[u][g], (float)sc.y, x[u][4 * t + i]));
          }
        }
      }
    const bool full = span_full(a, rows, st, KEYS);
    float p[QG][8];
#pragma unroll
    for (int u = 0; u < QG; ++u) {
      uint32_t seen = 0xffu;
      if (!full) {  // (uniform)
        seen = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) seen |= (span_sees(a, st, len[u], st.at + 16 * (e / 4) + 4 * (e % 4) + kgrp) ? 1u : 0u) << e;
      }
      float sum;
      auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) p[u][e] = seen >> e & 1u ? fast_exp2(fmaf(x[u][e], kSoftmaxScaleLog2, -m[u])) : 0.f;
        sum = ((p[u][0] + p[u][1]) + (p[u][2] + p[u][3])) + ((p[u][4] + p[u][5]) + (p[u][6] + p[u][7]));
      };
      weights();
      if (__ballot(!(sum <= kPfGrowth)) != 0ull) {
        float top = kNegBig;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, seen >> e & 1u ? x[u][e] * kSoftmaxScaleLog2 : kNegBig);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float mn = fmaxf(m[u], top), corr = fast_exp2(m[u] - mn);
        m[u] = mn;
        l[u] *= corr;
#pragma unroll
        for (int g = 0; g < kQ4Groups; ++g) {
          low[u][g] *= corr;
          ones[u][g] *= corr;
        }
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[u][c][i] *= corr;
        weights();
      }
      l[u] += sum;
    }
#pragma unroll
    for (int g = 0; g < kQ4Groups; ++g) {
      // tile c of group g: column 32 g + 2 m + c of lane m's word
      am_bf16x8_t av[2];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint32_t y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = q4_pair(__builtin_amdgcn_perm(vraw[2 * i + 1], vraw[2 * i], c ? 0x07060302u : 0x05040100u), g);
        av[c] = __builtin_bit_cast(am_bf16x8_t, make_uint4(y[0], y[1], y[2], y[3]));
      }
#pragma unroll
      for (int u = 0; u < QG; ++u) {
        uint32_t w[4][PT];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const cache_half2_t s0 = __builtin_bit_cast(cache_half2_t, am_word(vsc[2 * i], g)), s1 = __builtin_bit_cast(cache_half2_t, am_word(vsc[2 * i + 1], g));
          const float p0 = p[u][2 * i], p1 = p[u][2 * i + 1], x0 = p0 * (float)s0.x, x1 = p1 * (float)s1.x;
          ones[u][g] += x0 + x1;
          low[u][g] = fmaf(p0, (float)s0.y, fmaf(p1, (float)s1.y, low[u][g]));
          q4_terms<PT>(x0, x1, w[i]);
        }
#pragma unroll
        for (int t = PT - 1; t >= 0; --t) {
          const am_bf16x8_t b = __builtin_bit_cast(am_bf16x8_t, make_uint4(w[0][t], w[1][t], w[2][t], w[3][t]));
#pragma unroll
          for (int c = 0; c < 2; ++c) o[u][2 * g + c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av[c], b, o[u][2 * g + c], 0, 0, 0);
        }
      }
    }
    place.settle(places, next);
    load(next, std::false_type{});
    load(next, std::true_type{});
    place.ask(places, span_step(steps, rows, min(s + 2 * kQ4Waves, steps.total - 1)));
  }
#pragma unroll
  for (int u = 0; u < QG; ++u) {
    const int r = 16 * u + r16;
    l[u] += __shfl_xor(l[u], 16);
    l[u] += __shfl_xor(l[u], 32);
    if (len[u] == 0) l[u] = 0.f;  // (a padded token's lanes took whatever full steps gave)
    if (kgrp == 0) sm.ml[wave][r] = make_float2(m[u], l[u]);
    // o[2 g + c][i] is column 32 g + 2 (4 kgrp + i) + c
#pragma unroll
    for (int g = 0; g < kQ4Groups; ++g) {
      float base = low[u][g] - 16.f * ones[u][g];
      base += __shfl_xor(base, 16);
      base += __shfl_xor(base, 32);
#pragma unroll
      for (int i = 0; i < 4; i += 2)
        *reinterpret_cast<float4*>(&sm.o[wave][r][32 * g + 8 * kgrp + 2 * i]) =
            make_float4(fmaf(16.f, o[u][2 * g][i], base), fmaf(16.f, o[u][2 * g + 1][i], base), fmaf(16.f, o[u][2 * g][i + 1], base), fmaf(16.f, o[u][2 * g + 1][i + 1], base));
    }
  }
  span_store<T>(a, sm, tile, r0, live);
}

template <typename T>
static hipError_t launch_span_q4_t(const SpanArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)((long long)a.B * a.Hkv * a.tiles * a.nsplit)), block(64 * kQ4Waves);
  const bool past = a.tiles == 1 && (double)a.B * a.Hkv * a.nsplit * a.run * (2 * (kQ4RowBytes + kQ4ScaleBytes)) >= kPastBytes;
  if (a.rows == 4 && past)
    hipLaunchKernelGGL((span_q4_few_kernel<T, 1, true>), grid, block, 0, st, a);
  else if (a.rows == 4)
    hipLaunchKernelGGL((span_q4_few_kernel<T, 1, false>), grid, block, 0, st, a);
  else if (T::EPC == 8 && a.rows == 8 && past)  // (fp32: its three terms for two sets do not fit in the registers of two waves)
    hipLaunchKernelGGL((span_q4_few_kernel<BF16, 2, true>), grid, block, 0, st, a);
  else if (T::EPC == 8 && a.rows == 8)
    hipLaunchKernelGGL((span_q4_few_kernel<BF16, 2, false>), grid, block, 0, st, a);
  else if (a.rows == 16)
    hipLaunchKernelGGL((span_q4_kernel<T, 1>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((span_q4_kernel<T, 2>), grid, block, 0, st, a);
  return hipGetLastError();
}

hipError_t launch_span_q4(const Shape& s, const SpanArgs& a, hipStream_t st) {
  return s.dtype == 0 ? launch_span_q4_t<F32>(a, st) : launch_span_q4_t<BF16>(a, st);
}

}  // namespace loki
