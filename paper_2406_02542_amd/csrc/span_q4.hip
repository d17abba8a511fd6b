// Attention over a cache held whole in 4 bits (cache_impl.h), contiguous or on pages (Section 2, Eq. 1 of arXiv 2406.02542), each token over
// the last rows of its sequence and the first few (span_impl.h).
//
// A value is lowest + step n with one (step, lowest) for a row's group g of 32 columns, so
//   logit[row] = sum over g of 16 step_g[row] sum over c in g of q[c] n[row, c] / 16 + lowest_g[row] sum over c in g of q[c]
//   out[c]     = sum over rows of (16 p step_g)[row] n[row, c] / 16 + sum over rows of (p lowest_g)[row]          for c in g
// and the codes go to the matrix cores as they are: the bits 0x3f80 | n << 3 are the bf16 number 1 + n / 16, exactly, a shift and a bit
// select for two of them.  The ones' share is taken off in advance (the first product begins with minus the group's sum of q) or
// at the end (the product of the same terms with ones).  In fp32 sums stay as small as their results, or they would lose bits: from each number
// 1 + 7.5 / 16, a code's middle, is taken off, at every step, and lowest + 7.5 step takes the place of lowest: 5 sequences of 24
// heads up to 2311 rows, relative error 6e-7 for 1.4e-6, 17.6 us for 17.0.
#include "span_tiles_impl.h"

namespace loki {

constexpr int kQ4Waves = 4;

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

// p times a row's step, from its half of the scales' word (which v_fma_mix_f32 takes as it is, and the compiler converts first).
__device__ __forceinline__ float q4_times_step(float p, uint32_t scales) {
  float x;
  asm("v_fma_mix_f32 %0, %1, %2, 0 op_sel_hi:[0,1,0]" : "=v"(x) : "v"(p), "v"(scales));
  return x;
}

// A lane's column of the matrix cores' 16 is query row n / CG in CG ways: with the NS = 4 / CG groups n % CG * NS ..  Up to 4 query rows take
// CG = 4, up to 8 two, more one, 16 at a time.
//   first product   for group g, column n holds q in the columns of g if g is among its own, else zeros, so the products of the CG groups that share
//                   a place s = g % NS add up to each lane's own; the lanes of a query add theirs (DPP)
//   second          for group g, column n holds p step_g if g is its own, else zeros: the outputs of CG groups share an accumulator too
// so a lane scales and splits into terms only what its own groups ask: vector instructions for 32 rows of keys and values, of which 136 unpack
// codes: CG = 4 308, 2 356, 1 409.  The scales go through the wave's own part of LDS: a load takes them for all of a step's rows, and no
// lane holds 16 (CG = 4) to 64 registers of them while it waits; us in registers / LDS (before runs were dealt by the lengths): 64 sequences of 64/8 heads with 4096 rows
// (CG = 2) 78.3, 72.5, 16 of 64/8 with 8000 and two tokens (1) 65.6, 48.4, 16 of 32/8 with 16384 (4) 65.0, 63.5.  (16 rows' products for two groups
// of queries at a time, which unpack codes half as often, leave a SIMD one wave: 50.6 us where these took 43.9.)
// bf16: q is one term, the weights two (2^-16 of each, as the library's other attention); fp32: three each.
// Vector instructions bound it: 16 sequences of 32/8 heads up to 16384 rows (210 to 240 MB) 43 to 48 us, 72 % of the SIMDs' cycles beside 5.6 TB/s of memory, all
// of 16384 60 us; four tokens of 8 of 64/8 up to 8192 35 to 38 us, 62 %; 5 of 24 fp32 heads up to 2311 17 us, 51 %; one of 32/8 over 8192 10 us, of which the
// merge 3.
template <typename T, int CG, bool STREAM, bool DEALT>
__global__ __launch_bounds__(64 * kQ4Waves, span_q4_waves(T::EPC == 8, 16 / CG)) void span_q4_kernel(SpanArgs a) {
  constexpr bool MID = T::EPC == 4;
  constexpr float kOff = MID ? 1.46875f : 1.f;  // taken off each number 1 + n / 16
  constexpr int KEYS = 32, QT = T::EPC == 8 ? 1 : 3, PT = T::EPC == 8 ? 2 : 3, NS = kQ4Groups / CG, ROWS = 16 / CG;
  __shared__ __align__(16) SpanMerge<ROWS, kQ4Waves> sm;
  __shared__ uint4 s_scales[kQ4Waves][2 * KEYS];  // of a step's keys, and values
  const SpanTile tile = span_tile<KEYS, DEALT>(a);
  if (tile.h < 0) return;  // (uniform for the block)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), r16 = lane & 15, kgrp = lane >> 4;
  const int gl = r16 % CG, g0 = gl * NS, r = r16 / CG;
  const int M = a.m * a.G, r0 = tile.tile * ROWS, live = min(ROWS, M - r0), lg = 31 - __builtin_clz(a.G);
  const SpanRows rows = tile.rows;
  const SpanSteps<KEYS> steps(rows);
  if (tile.s0 >= tile.s1 && tile.part > 0) return span_none<DEALT>(a, tile, live);  // (uniform for the block)
  const int s1 = tile.s1;
  const RowPlaces places(a.cache, tile.b, tile.h, a.Hkv);
  const Q4Pair q4_pair;

  const char *kb = static_cast<const char*>(a.cache.k), *vb = static_cast<const char*>(a.cache.v);
  const char *ks = static_cast<const char*>(a.cache.k_scales), *vs = static_cast<const char*>(a.cache.v_scales);
  const int k_row = 4 * (r16 & 3) + (r16 >> 2);  // (see the head of this file)
  const unsigned k_at = k_row * kQ4RowBytes + 16 * kgrp, v_at = kgrp * kQ4RowBytes + 4 * r16, s_at = (lane & 15) * kQ4ScaleBytes;
  uint4 kraw[2], sraw;  // sraw: this lane's row's scales, a half of the wave for the keys', the other for the values'
  uint32_t vraw[8];
  SpanPlaces<2> place;
  auto load_k = [&](const SpanStep& st) __attribute__((always_inline)) {
    const long long at = lane & 16 ? place.at[1] : place.at[0];
    const char* x = (lane < 32 ? ks : vs) + at * kQ4ScaleBytes;
    span_loads<KEYS>(st, [&](auto whole) __attribute__((always_inline)) {
      constexpr bool W = decltype(whole)::value;
      sraw = load16(W ? x + s_at : x + span_near(st, lane >> 4 & 1, lane & 15) * kQ4ScaleBytes);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const char* c = kb + place.at[t] * kQ4RowBytes;
        kraw[t] = load16_hint<STREAM>(W ? c + k_at : c + span_near(st, t, k_row) * kQ4RowBytes + 16 * kgrp);
      }
    });
  };
  auto load_v = [&](const SpanStep& st) __attribute__((always_inline)) {
    span_loads<KEYS>(st, [&](auto whole) __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const char* c = vb + place.at[t] * kQ4RowBytes;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          vraw[4 * t + i] = load4_hint<STREAM>(decltype(whole)::value ? c + v_at + 4 * i * kQ4RowBytes : c + span_near(st, t, 4 * i + kgrp) * kQ4RowBytes + 4 * r16);
      }
    });
  };
  // (step, lowest) of the lane's groups, of the row whose weight is its e-th (a wave's LDS operations keep their order)
  const uint32_t* s_mine = reinterpret_cast<const uint32_t*>(&s_scales[wave][kgrp]) + g0;
  auto scales = [&](int values, int e) __attribute__((always_inline)) {
    return *reinterpret_cast<const Q4Scales<NS>*>(s_mine + (values * KEYS + 16 * (e / 4) + 4 * (e % 4)) * kQ4Groups);
  };
  int s = tile.s0 + wave;
  if (s < s1) {  // (uniform for the wave)
    const SpanStep st = span_step(steps, rows, s);
    place.ask(places, st);
    place.settle(places, st);
    load_k(st);
    load_v(st);
    place.ask(places, span_step(steps, rows, min(s + kQ4Waves, steps.total - 1)));
  }

  const int len = r < live ? span_len(a, tile.b, (r0 + r) >> lg) : 0;
  uint32_t own[CG];  // all ones where the lane's groups are the i-th's
#pragma unroll
  for (int i = 0; i < CG; ++i) own[i] = gl == i ? ~0u : 0u;
  am_bf16x8_t bq[kQ4Groups][QT];
  float qsum[NS], qoff[NS], low[NS];  // qsum: of a group's columns; qoff: what the first product begins with
  float m = kNegBig, l = 0.f;
  am_f32x4_t o[NS][2], ones[NS];  // ones: the sum of the numbers that multiply codes, in every element
  const am_bf16x8_t one = __builtin_bit_cast(am_bf16x8_t, make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u));
  const typename T::store_t* src =
      static_cast<const typename T::store_t*>(a.q) + span_place(a, tile.b, tile.h, r0 + min(r, live - 1)) * kD + 32 * g0 + 8 * kgrp;
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; e += T::EPC) T::unpack(span_query(load16(src + 32 * n + e), len), *reinterpret_cast<float(*)[T::EPC]>(x + e));
    uint32_t w[4][QT];
    std::conditional_t<MID, double, float> sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      q4_terms<QT>(x[2 * i], x[2 * i + 1], w[i]);
      sum += x[2 * i];
      sum += x[2 * i + 1];
    }
#pragma unroll
    for (int i = 0; i < CG; ++i)
#pragma unroll
      for (int t = 0; t < QT; ++t)
        bq[i * NS + n][t] = __builtin_bit_cast(am_bf16x8_t, make_uint4(w[0][t] & own[i], w[1][t] & own[i], w[2][t] & own[i], w[3][t] & own[i]));
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    qsum[n] = (float)sum;
    qoff[n] = (float)(-kOff * sum);
    low[n] = 0.f;
    o[n][0] = o[n][1] = ones[n] = am_f32x4_t{};
  }

  // The waves of a SIMD, of different blocks, are to end together: those that are behind go first.  (The oldest go first otherwise, and a SIMD is left
  // to the last one: blocks of equal work took 34 to 65 us where these take 49 to 61.)  us without / so: 16 sequences of 32/8 heads
  // with 16384 rows 64.1 / 60.9, four tokens of 8 of 64/8 44.3 / 42.4 (each in equal parts).
  const int quarter = (s1 - s) >> 2, marks[3] = {s + quarter, s + 2 * quarter, s + 3 * quarter};
  __builtin_amdgcn_s_setprio(3);
  for (; s < s1; s += kQ4Waves) {
    if (s >= marks[2])
      __builtin_amdgcn_s_setprio(0);
    else if (s >= marks[1])
      __builtin_amdgcn_s_setprio(1);
    else if (s >= marks[0])
      __builtin_amdgcn_s_setprio(2);
    const SpanStep st = span_step(steps, rows, s), next = span_step(steps, rows, min(s + kQ4Waves, steps.total - 1));
    s_scales[wave][lane] = sraw;
    __builtin_amdgcn_wave_barrier();
    float x[8];  // a sixteenth of the logits
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      am_f32x4_t acc[NS];
#pragma unroll
      for (int n = 0; n < NS; ++n) acc[n] = am_f32x4_t{qoff[n], qoff[n], qoff[n], qoff[n]};
#pragma unroll
      for (int g = 0; g < kQ4Groups; ++g) {
        const am_bf16x8_t ka = __builtin_bit_cast(am_bf16x8_t, make_uint4(q4_pair(kraw[t].x, g), q4_pair(kraw[t].y, g), q4_pair(kraw[t].z, g), q4_pair(kraw[t].w, g)));
#pragma unroll
        for (int i = 0; i < QT; ++i) acc[g % NS] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, bq[g][i], acc[g % NS], 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const Q4Scales<NS> row = scales(0, 4 * t + i);
        float sum = 0.f;
#pragma unroll
        for (int n = 0; n < NS; ++n) {
          const cache_half2_t sc = row.at(n);
          const float base = MID ? fmaf((float)sc.x, 7.5f, (float)sc.y) : (float)sc.y;
          const float lowest = n == 0 ? base * (qsum[n] * 0.0625f) : fmaf(base, qsum[n] * 0.0625f, sum);
          sum = fmaf((float)sc.x, acc[n][i], lowest);
        }
        x[4 * t + i] = group_allreduce_sum<CG>(sum);
      }
    }
    place.settle(places, next);
    load_k(next);
    const bool full = span_full(a, rows, st, KEYS);
    if (!full) {  // (uniform)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (!span_sees(a, st, len, st.at + 16 * (e / 4) + 4 * (e % 4) + kgrp)) x[e] = kUnseen;
    }
    float p[8], sum;
    auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = fast_exp2(fmaf(x[e], 16.f * kSoftmaxScaleLog2, -m));
      sum = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    };
    weights();
    if (__ballot(!(sum <= kPfGrowth)) != 0ull) {
      float top = x[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) top = fmaxf(top, x[e]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32)) * (16.f * kSoftmaxScaleLog2);
      const float mn = fmaxf(m, top), corr = fast_exp2(m - mn);
      m = mn;
      l *= corr;
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        low[n] *= corr;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          o[n][0][i] *= corr;
          o[n][1][i] *= corr;
          if constexpr (!MID) ones[n][i] *= corr;
        }
      }
      weights();
    }
    l += sum;
    uint32_t y[2][4];  // the rows' words, two to a register: columns 2 m, and 2 m + 1, of all groups
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) y[c][i] = __builtin_amdgcn_perm(vraw[2 * i + 1], vraw[2 * i], c ? 0x07060302u : 0x05040100u);
    Q4Scales<NS> sc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) sc[e] = scales(1, e);
    if (!full) {  // (a row that the token does not see may hold no numbers)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (!span_sees(a, st, len, st.at + 16 * (e / 4) + 4 * (e % 4) + kgrp)) sc[e] = Q4Scales<NS>{};
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      uint32_t w[4][PT];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p0 = p[2 * i], p1 = p[2 * i + 1];
        const cache_half2_t s0 = sc[2 * i].at(n), s1 = sc[2 * i + 1].at(n);
        if constexpr (MID)
          low[n] = fmaf(p0, fmaf((float)s0.x, 7.5f, (float)s0.y), fmaf(p1, fmaf((float)s1.x, 7.5f, (float)s1.y), low[n]));
        else
          low[n] = fmaf(p0, (float)s0.y, fmaf(p1, (float)s1.y, low[n]));
        q4_terms<PT>(q4_times_step(p0, sc[2 * i].w[n]), q4_times_step(p1, sc[2 * i + 1].w[n]), w[i]);
      }
      if constexpr (MID) ones[n] = am_f32x4_t{};
#pragma unroll
      for (int t = PT - 1; t >= 0; --t)
        ones[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(one, __builtin_bit_cast(am_bf16x8_t, make_uint4(w[0][t], w[1][t], w[2][t], w[3][t])), ones[n], 0, 0, 0);
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
            o[n][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, __builtin_bit_cast(am_bf16x8_t, b), o[n][c], 0, 0, 0);
          }
        }
      }
      if constexpr (MID) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          o[n][0][i] = fmaf(-kOff, ones[n][i], o[n][0][i]);
          o[n][1][i] = fmaf(-kOff, ones[n][i], o[n][1][i]);
        }
      }
    }
    load_v(next);
    place.ask(places, span_step(steps, rows, min(s + 2 * kQ4Waves, steps.total - 1)));
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (len == 0) {  // (a padded token's lanes took whatever full steps gave, a maximum too)
    m = kNegBig;
    l = 0.f;
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      o[n][0] = o[n][1] = ones[n] = am_f32x4_t{};
      low[n] = 0.f;
    }
  }
  if (kgrp == 0 && gl == 0) sm.ml[wave][r] = make_float2(m, l);
  // o[n][c][i] is column 32 (g0 + n) + 2 (4 kgrp + i) + c
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    float base = low[n];
    base += __shfl_xor(base, 16);
    base += __shfl_xor(base, 32);
    float y[2][4];
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) y[c][i] = fmaf(16.f, MID ? o[n][c][i] : o[n][c][i] - ones[n][i], base);
#pragma unroll
    for (int i = 0; i < 4; i += 2)
      *reinterpret_cast<float4*>(&sm.o[wave][r][32 * (g0 + n) + 8 * kgrp + 2 * i]) = make_float4(y[0][i], y[1][i], y[0][i + 1], y[1][i + 1]);
  }
  span_store<T, DEALT>(a, sm, tile, r0, live);
}

template <typename T>
static hipError_t launch_span_q4_t(const SpanArgs& a, unsigned blocks, bool past, hipStream_t st) {
  const dim3 grid(blocks), block(64 * kQ4Waves);
  if (T::EPC == 8 && a.rows == 128) return launch_span_tiles<8, 4, true>(a, blocks, st);
  if (T::EPC == 8 && a.rows == 256) return a.halves == 0 ? launch_span_tiles<8, 8, true>(a, blocks, st) : launch_span_tiles<8, 8, true, true>(a, blocks, st);
#define LOKI_SPAN_Q4(CG, STREAM)                                                            \
  if (a.dealt != nullptr)                                                                   \
    hipLaunchKernelGGL((span_q4_kernel<T, CG, STREAM, true>), grid, block, 0, st, a);       \
  else                                                                                      \
    hipLaunchKernelGGL((span_q4_kernel<T, CG, STREAM, false>), grid, block, 0, st, a)
  if (a.rows == 4 && past) {
    LOKI_SPAN_Q4(4, true);
  } else if (a.rows == 4) {
    LOKI_SPAN_Q4(4, false);
  } else if (a.rows == 8 && past) {
    LOKI_SPAN_Q4(2, true);
  } else if (a.rows == 8) {
    LOKI_SPAN_Q4(2, false);
  } else {
    LOKI_SPAN_Q4(1, false);
  }
#undef LOKI_SPAN_Q4
  return hipGetLastError();
}

hipError_t launch_span_q4(const Shape& s, const SpanArgs& a, unsigned blocks, bool past, hipStream_t st) {
  return s.dtype == 0 ? launch_span_q4_t<F32>(a, blocks, past, st) : launch_span_q4_t<BF16>(a, blocks, past, st);
}

}  // namespace loki
