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

// (step, lowest) of N neighbouring groups of a row.
template <int N>
struct alignas(4 * N) Q4Scales {
  uint32_t w[N];
  __device__ __forceinline__ cache_half2_t at(int n) const { return __builtin_bit_cast(cache_half2_t, w[n]); }
};

// Waves on a SIMD that the registers are to leave room for.
template <typename T, int CG, int QG>
constexpr int q4_waves() {
  return span_q4_waves(T::EPC == 8, CG == 1 ? 16 * QG : 16 / CG);
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

// A lane's column of the matrix cores' 16 is query row n / CG in CG ways: with the NS = 4 / CG groups n % CG * NS ..  Up to 4 query rows take
// CG = 4, up to 8 two, else one; QG: 16-column sets of rows.
//   first product   for group g, column n holds q in the columns of g if g is among its own, else zeros, so the products of the CG groups that share
//                   a place s = g % NS add up to each lane's own; the lanes of a query add theirs (DPP)
//   second          for group g, column n holds p step_g if g is its own, else zeros: the outputs of CG groups share an accumulator too
// so a lane scales and splits into terms only what its own groups ask: vector instructions for 32 rows of keys and values of which 136 unpack
// codes: CG = 4 280, 2 340, 1 450.
// bf16: q is one term, the weights two (2^-16 of each, as the library's other attention); fp32: three each.
template <typename T, int CG, int QG, bool STREAM>
__global__ __launch_bounds__(64 * kQ4Waves, (q4_waves<T, CG, QG>())) void span_q4_kernel(SpanArgs a) {
  constexpr int KEYS = 32, QT = T::EPC == 8 ? 1 : 3, PT = T::EPC == 8 ? 2 : 3, NS = kQ4Groups / CG, PER = 16 / CG, ROWS = PER * QG;
  __shared__ __align__(16) SpanMerge<ROWS, kQ4Waves> sm;
  const SpanTile tile = span_tile<KEYS>(a);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), r16 = lane & 15, kgrp = lane >> 4;
  const int gl = r16 % CG, g0 = gl * NS, col = r16 / CG;
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
  const unsigned k_at = k_row * kQ4RowBytes + 16 * kgrp, v_at = kgrp * kQ4RowBytes + 4 * r16, s_at = kgrp * kQ4ScaleBytes + 4 * g0;
  uint4 kraw[2];
  Q4Scales<NS> ksc[8], vsc[8];  // of the lane's groups
  uint32_t vraw[8];
  SpanPlaces<2> place;
  auto load = [&](const SpanStep& st, auto values) __attribute__((always_inline)) {
    constexpr bool V = decltype(values)::value;
    const char *codes = V ? vb : kb, *scales = V ? vs : ks;
    Q4Scales<NS>(&sc)[8] = V ? vsc : ksc;
    span_loads<KEYS>(st, [&](auto whole) __attribute__((always_inline)) {
      constexpr bool W = decltype(whole)::value;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const char *c = codes + place.at[t] * kQ4RowBytes, *x = scales + place.at[t] * kQ4ScaleBytes;
        if constexpr (!V) kraw[t] = load16_hint<STREAM>(W ? c + k_at : c + span_near(st, t, k_row) * kQ4RowBytes + 16 * kgrp);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = W ? 0 : span_near(st, t, 4 * i + kgrp);
          sc[4 * t + i] = *reinterpret_cast<const Q4Scales<NS>*>(W ? x + s_at + 4 * i * kQ4ScaleBytes : x + row * kQ4ScaleBytes + 4 * g0);
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

  int len[QG];
  uint32_t own[CG];  // all ones where the lane's groups are the g-th's
#pragma unroll
  for (int i = 0; i < CG; ++i) own[i] = gl == i ? ~0u : 0u;
  am_bf16x8_t bq[QG][kQ4Groups][QT];
  float qsum[QG][NS];  // of a group's columns
  float m[QG], l[QG], low[QG][NS], ones[QG][NS];
  am_f32x4_t o[QG][NS][2];
#pragma unroll
  for (int u = 0; u < QG; ++u) {
    const int r = PER * u + col;
    len[u] = r < live ? span_len(a, tile.b, (r0 + r) >> lg) : 0;
    const typename T::store_t* src =
        static_cast<const typename T::store_t*>(a.q) + span_place(a, tile.b, tile.h, r0 + min(r, live - 1)) * kD + 32 * g0 + 8 * kgrp;
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; e += T::EPC) T::unpack(load16(src + 32 * n + e), *reinterpret_cast<float(*)[T::EPC]>(x + e));
      uint32_t w[4][QT];
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        q4_terms<QT>(x[2 * i], x[2 * i + 1], w[i]);
        sum += x[2 * i] + x[2 * i + 1];
      }
#pragma unroll
      for (int i = 0; i < CG; ++i)
#pragma unroll
        for (int t = 0; t < QT; ++t)
          bq[u][i * NS + n][t] = __builtin_bit_cast(am_bf16x8_t, make_uint4(w[0][t] & own[i], w[1][t] & own[i], w[2][t] & own[i], w[3][t] & own[i]));
      sum += __shfl_xor(sum, 16);
      qsum[u][n] = sum + __shfl_xor(sum, 32);
      low[u][n] = ones[u][n] = 0.f;
      o[u][n][0] = o[u][n][1] = am_f32x4_t{};
    }
    m[u] = kNegBig;
    l[u] = 0.f;
  }

  for (; s < s1; s += kQ4Waves) {
    const SpanStep st = span_step(steps, rows, s), next = span_step(steps, rows, min(s + kQ4Waves, steps.total - 1));
    float x[QG][8];  // a sixteenth of the logits
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      am_f32x4_t acc[QG][NS];
#pragma unroll
      for (int u = 0; u < QG; ++u)
#pragma unroll
        for (int n = 0; n < NS; ++n) acc[u][n] = am_f32x4_t{-qsum[u][n], -qsum[u][n], -qsum[u][n], -qsum[u][n]};
#pragma unroll
      for (int g = 0; g < kQ4Groups; ++g) {
        const am_bf16x8_t ka = __builtin_bit_cast(am_bf16x8_t, make_uint4(q4_pair(kraw[t].x, g), q4_pair(kraw[t].y, g), q4_pair(kraw[t].z, g), q4_pair(kraw[t].w, g)));
#pragma unroll
        for (int u = 0; u < QG; ++u)
#pragma unroll
          for (int i = QT - 1; i >= 0; --i) acc[u][g % NS] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, bq[u][g][i], acc[u][g % NS], 0, 0, 0);
      }
#pragma unroll
      for (int u = 0; u < QG; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float sum = 0.f;
#pragma unroll
          for (int n = 0; n < NS; ++n) {
            const cache_half2_t sc = ksc[4 * t + i].at(n);
            const float low_part = n == 0 ? (float)sc.y * (qsum[u][n] * 0.0625f) : fmaf((float)sc.y, qsum[u][n] * 0.0625f, sum);
            sum = fmaf((float)sc.x, acc[u][n][i], low_part);
          }
          x[u][4 * t + i] = group_allreduce_sum<CG>(sum);
        }
    }
    place.settle(places, next);
    load(next, std::false_type{});
    const bool full = span_full(a, rows, st, KEYS);
    float p[QG][8];
#pragma unroll
    for (int u = 0; u < QG; ++u) {
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
#pragma unroll
        for (int n = 0; n < NS; ++n) {
          low[u][n] *= corr;
          ones[u][n] *= corr;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            o[u][n][0][i] *= corr;
            o[u][n][1][i] *= corr;
          }
        }
        weights();
      }
      l[u] += sum;
    }
    uint32_t y[2][4];  // the rows' words, two to a register: columns 2 m, and 2 m + 1, of all groups
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) y[c][i] = __builtin_amdgcn_perm(vraw[2 * i + 1], vraw[2 * i], c ? 0x07060302u : 0x05040100u);
#pragma unroll
    for (int u = 0; u < QG; ++u)
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        uint32_t w[4][PT];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const cache_half2_t sc0 = vsc[2 * i].at(n), sc1 = vsc[2 * i + 1].at(n);
          const float p0 = p[u][2 * i], p1 = p[u][2 * i + 1], x0 = p0 * (float)sc0.x, x1 = p1 * (float)sc1.x;
          ones[u][n] += x0 + x1;
          low[u][n] = fmaf(p0, (float)sc0.y, fmaf(p1, (float)sc1.y, low[u][n]));
          q4_terms<PT>(x0, x1, w[i]);
        }
#pragma unroll
        for (int k = 0; k < CG; ++k) {
          const int g = k * NS + n;
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const am_bf16x8_t av = __builtin_bit_cast(am_bf16x8_t, make_uint4(q4_pair(y[c][0], g), q4_pair(y[c][1], g), q4_pair(y[c][2], g), q4_pair(y[c][3], g)));
#pragma unroll
            for (int t = PT - 1; t >= 0; --t) {
              const uint4 b = CG == 1 ? make_uint4(w[0][t], w[1][t], w[2][t], w[3][t])
                                      : make_uint4(w[0][t] & own[k], w[1][t] & own[k], w[2][t] & own[k], w[3][t] & own[k]);
              o[u][n][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, __builtin_bit_cast(am_bf16x8_t, b), o[u][n][c], 0, 0, 0);
            }
          }
        }
      }
    load(next, std::true_type{});
    place.ask(places, span_step(steps, rows, min(s + 2 * kQ4Waves, steps.total - 1)));
  }
#pragma unroll
  for (int u = 0; u < QG; ++u) {
    const int r = PER * u + col;
    l[u] += __shfl_xor(l[u], 16);
    l[u] += __shfl_xor(l[u], 32);
    if (len[u] == 0) l[u] = 0.f;  // (a padded token's lanes took whatever full steps gave)
    if (kgrp == 0 && gl == 0) sm.ml[wave][r] = make_float2(m[u], l[u]);
    // o[n][c][i] is column 32 (g0 + n) + 2 (4 kgrp + i) + c
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      float base = low[u][n] - 16.f * ones[u][n];
      base += __shfl_xor(base, 16);
      base += __shfl_xor(base, 32);
#pragma unroll
      for (int i = 0; i < 4; i += 2)
        *reinterpret_cast<float4*>(&sm.o[wave][r][32 * (g0 + n) + 8 * kgrp + 2 * i]) =
            make_float4(fmaf(16.f, o[u][n][0][i], base), fmaf(16.f, o[u][n][1][i], base), fmaf(16.f, o[u][n][0][i + 1], base), fmaf(16.f, o[u][n][1][i + 1], base));
    }
  }
  span_store<T>(a, sm, tile, r0, live);
}

template <typename T>
static hipError_t launch_span_q4_t(const SpanArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)((long long)a.B * a.Hkv * a.tiles * a.nsplit)), block(64 * kQ4Waves);
  const bool past = a.tiles == 1 && (double)a.B * a.Hkv * a.nsplit * a.run * (2 * (kQ4RowBytes + kQ4ScaleBytes)) >= kPastBytes;
  if (a.rows == 4 && past)
    hipLaunchKernelGGL((span_q4_kernel<T, 4, 1, true>), grid, block, 0, st, a);
  else if (a.rows == 4)
    hipLaunchKernelGGL((span_q4_kernel<T, 4, 1, false>), grid, block, 0, st, a);
  else if (a.rows == 8 && past)
    hipLaunchKernelGGL((span_q4_kernel<T, 2, 1, true>), grid, block, 0, st, a);
  else if (a.rows == 8)
    hipLaunchKernelGGL((span_q4_kernel<T, 2, 1, false>), grid, block, 0, st, a);
  else if (a.rows == 16)
    hipLaunchKernelGGL((span_q4_kernel<T, 1, 1, false>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((span_q4_kernel<T, 1, 2, false>), grid, block, 0, st, a);
  return hipGetLastError();
}

hipError_t launch_span_q4(const Shape& s, const SpanArgs& a, hipStream_t st) {
  return s.dtype == 0 ? launch_span_q4_t<F32>(a, st) : launch_span_q4_t<BF16>(a, st);
}

}  // namespace loki
