// Attention over a cache held whole, contiguous or on pages (Section 2, Eq. 1 of arXiv 2406.02542), each token over the last rows of its
// sequence and the first few (span_impl.h): one token of every sequence, several, or chunks of prompts.
//
// Up to 16 query rows of a KV head (span_rows_kernel, span_f32_kernel): memory bounds it, a wave takes steps of rows straight from
// registers, a block's waves take steps in turn.  More, in bf16 (span_tiles_kernel): the matrix cores bound it, tiles of keys and
// values go through LDS for all of the block's query rows.
#include "span_impl.h"

namespace loki {

constexpr int kSpWaves = 4;

// ---- bf16, up to 16 query rows ------------------------------------------------------------------------------------
// A wave takes steps of 32 rows:
//   S[row, query] = K Q^T           v_mfma_f32_16x16x32_bf16, A = 16 bytes of a row for each lane (row, c), two tiles of 16 rows
//   O^T[column, query] += V^T P^T   lane (m, c) loads 16 bytes, columns 8 m .., of the 8 rows whose weights its own column of P has, and pairs
//                                   rows up (v_perm_b32); the weights in two bf16 terms, 2^-16 of each (as the library's other attention)
// so a query's maximum, sum and outputs are its own lanes'.  The reference of the exponentials follows the maximum only when a
// lane's weights of a step sum up to more than 2^8.
template <bool STREAM>
__global__ __launch_bounds__(64 * kSpWaves) void span_rows_kernel(SpanArgs a) {
  constexpr int KEYS = 32;
  __shared__ __align__(16) SpanMerge<16, kSpWaves> sm;
  const SpanTile tile = span_tile<KEYS>(a);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), r16 = lane & 15, kgrp = lane >> 4;
  const int M = a.m * a.G, r0 = tile.tile * 16, live = min(16, M - r0), lg = 31 - __builtin_clz(a.G);
  const SpanRows rows = tile.rows;
  const SpanSteps<KEYS> steps(rows);
  if (tile.s0 >= tile.s1 && tile.part > 0) return span_none(a, tile, live);  // (uniform for the block)
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
  if (len == 0) l = 0.f;  // (a padded token's lanes took whatever full steps gave)
  if (kgrp == 0) sm.ml[wave][r16] = make_float2(m, l);
  // o[c][i] is column 8 (4 kgrp + i) + c
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float4* dst = reinterpret_cast<float4*>(&sm.o[wave][r16][8 * (4 * kgrp + i)]);
    dst[0] = make_float4(o[0][i], o[1][i], o[2][i], o[3][i]);
    dst[1] = make_float4(o[4][i], o[5][i], o[6][i], o[7][i]);
  }
  span_store<BF16>(a, sm, tile, r0, live);
}

// ---- fp32 -----------------------------------------------------------------------------------------------------------
// The products of parts_impl.h's attend_f32, v_mfma_f32_16x16x4_f32, straight from registers, for QG groups of 16 query rows; steps of 16 rows.
template <int QG, bool STREAM>
__global__ __launch_bounds__(64 * kSpWaves, 2) void span_f32_kernel(SpanArgs a) {
  constexpr int KEYS = 16;
  __shared__ __align__(16) SpanMerge<16 * QG, kSpWaves> sm;
  const SpanTile tile = span_tile<KEYS>(a);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l16 = lane & 15, c4 = lane >> 4;
  const int M = a.m * a.G, r0 = tile.tile * (16 * QG), live = min(16 * QG, M - r0), lg = 31 - __builtin_clz(a.G);
  const SpanRows rows = tile.rows;
  const SpanSteps<KEYS> steps(rows);
  if (tile.s0 >= tile.s1 && tile.part > 0) return span_none(a, tile, live);  // (uniform for the block)
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
    if (len[g] == 0) l[g] = 0.f;
    const int r = 16 * g + l16;
    if (c4 == 0) sm.ml[wave][r] = make_float2(m[g], l[g]);
    // o[4 c + t][i] is column 64 c + 4 (4 c4 + i) + t
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(&sm.o[wave][r][64 * c + 16 * c4 + 4 * i]) = make_float4(o[g][4 * c][i], o[g][4 * c + 1][i], o[g][4 * c + 2][i], o[g][4 * c + 3][i]);
  }
  span_store<F32>(a, sm, tile, r0, live);
}

// ---- bf16, more query rows: tiles through LDS -------------------------------------------------------------------------
// The products of shared.hip's prefix kernel: a wave holds 32 query rows and takes steps of 32 keys, S^T = K Q^T and O^T += V^T P^T by
// v_mfma_f32_32x32x16_bf16, the weights in two bf16 terms as they come out of the first product.  Tiles of KT keys and values go through LDS
// once for the block's waves, WQ of which hold different queries and WK = WAVES / WQ different keys of the tile; the next tile is loaded into
// registers while this one is used.  What is masked is decided for a wave's step as a whole: nothing to see, everything, or each on its own.
typedef short sp_s16x4_t __attribute__((ext_vector_type(4)));
typedef float sp_f32x16_t __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) sp_s16x4_t sp_lds_s16x4_t;

template <int WAVES, int WQ>
constexpr int span_tile_keys() {
  return WAVES / WQ == 4 ? 128 : 64;
}
// Two pairs of tiles; at the end, where waves have other keys of the same queries, what half of them hand over, or the outputs.
template <int WAVES, int WQ>
constexpr int span_lds_bytes() {
  const int tiles = 4 * span_tile_keys<WAVES, WQ>() * 256, merge = WQ == WAVES ? 0 : WAVES * 32 * 8 + WAVES / 2 * 64 * 256;
  return tiles > merge ? tiles : merge;
}

template <int WAVES, int WQ>
__global__ __launch_bounds__(64 * WAVES, WAVES == 4 ? 1 : 2) void span_tiles_kernel(SpanArgs a) {
  extern __shared__ __align__(16) char smem[];  // [2][K tile, V tile]
  constexpr int kThreads = 64 * WAVES, WK = WAVES / WQ, KT = span_tile_keys<WAVES, WQ>(), kSteps = KT / (32 * WK), kChunks = KT * 16 / kThreads;
  constexpr int kTileBytes = KT * 256;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, half = lane >> 5, l16 = lane & 15;
  const int wq = wave % WQ, wk = wave / WQ;
  const SpanTile tile = span_tile<KT>(a);
  const int M = a.m * a.G, r0 = tile.tile * (32 * WQ), live = min(32 * WQ, M - r0), lg = 31 - __builtin_clz(a.G);
  const SpanRows rows = tile.rows;
  const SpanSteps<KT> steps(rows);
  if (tile.s0 >= tile.s1 && tile.part > 0) return span_none(a, tile, live);  // (uniform for the block)
  const int s0 = tile.s0, s1 = tile.s1;
  const RowPlaces places(a.cache, tile.b, tile.h, a.Hkv);
  // this wave's queries, and its lane's
  const int q0 = wq * 32, mine = min(32, live - q0), row = q0 + l32;
  SpanRows own{0, 0, 0, 0};
  if (mine > 0) own = span_rows(a, tile.b, (r0 + q0) >> lg, (r0 + q0 + mine - 1) >> lg);
  const int len = row < live ? span_len(a, tile.b, (r0 + row) >> lg) : 0;

  am_bf16x8_t q[8];
  {
    const uint16_t* src = static_cast<const uint16_t*>(a.q) + span_place(a, tile.b, tile.h, r0 + min(row, live - 1)) * kD + 8 * half;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) q[ks] = __builtin_bit_cast(am_bf16x8_t, load16(src + 16 * ks));
  }
  const uint16_t* kb = static_cast<const uint16_t*>(a.cache.k) + l16 * 8;
  const uint16_t* vb = static_cast<const uint16_t*>(a.cache.v) + l16 * 8;
  uint4 kst[kChunks], vst[kChunks];
  auto load = [&](int s) __attribute__((always_inline)) {  // (a wave's four rows of a chunk lie in one page)
    const SpanStep st = span_step(steps, rows, s);
#pragma unroll
    for (int j = 0; j < kChunks; ++j) {
      const int first = st.at + 4 * wave + kThreads / 16 * j;
      const long long off = (places(min(max(first, st.lo), st.hi - 1)) + min(max(first + (lane >> 4), st.lo), st.hi - 1)) * kD;
      kst[j] = load16(kb + off);
      vst[j] = load16(vb + off);
    }
  };
  auto store = [&](int b) __attribute__((always_inline)) {
    char* base = smem + b * 2 * kTileBytes;
#pragma unroll
    for (int j = 0; j < kChunks; ++j) {
      const int at = tid + kThreads * j, r = at >> 4, c = at & 15;
      *reinterpret_cast<uint4*>(base + r * 256 + ((c ^ (r & 15)) * 16)) = kst[j];
      *reinterpret_cast<uint4*>(base + kTileBytes + r * 256 + ((c ^ ((r & 3) << 2)) * 16)) = vst[j];
    }
  };

  float m = kNegBig, l = 0.f;
  sp_f32x16_t o[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) o[c] = sp_f32x16_t{};
  const int k_at = l32 * 256 + ((half ^ l16) * 16);
  const int v_row = 4 * half + (l16 >> 2);
  const int v_at = kTileBytes + v_row * 256 + (((((lane >> 4) & 1) * 2 + ((l16 & 3) >> 1)) ^ ((v_row & 3) << 2)) * 16) + (l16 & 1) * 8;

  // 32 keys of the tile in buffer `base`, rows st.at ..; full: all of them are seen by all of the wave's queries
  auto step = [&](const char* base, const SpanStep& st, bool full) __attribute__((always_inline)) {
    am_bf16x8_t ka[8], va[2][4];
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) ka[ks] = __builtin_bit_cast(am_bf16x8_t, *reinterpret_cast<const uint4*>(base + (k_at ^ (ks * 32))));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const char* at = base + (v_at ^ (c * 64)) + ks * 4096;
        const sp_s16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((sp_lds_s16x4_t*)(at));
        const sp_s16x4_t y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((sp_lds_s16x4_t*)(at + 2048));
        va[ks][c] = __builtin_bit_cast(am_bf16x8_t, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
      }
    sp_f32x16_t s = sp_f32x16_t{};
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[ks], q[ks], s, 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
    if (!full) {  // (uniform)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (!span_sees(a, st, len, st.at + 8 * (i >> 2) + 4 * half + (i & 3))) s[i] = kUnseen;
    }
    float p[16], sum;
    auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] = fast_exp2(fmaf(s[i], kSoftmaxScaleLog2, -m));
      float odd = p[1];
      sum = p[0];
#pragma unroll
      for (int i = 2; i < 16; i += 2) {
        sum += p[i];
        odd += p[i + 1];
      }
      sum += odd;
    };
    weights();
    if (__ballot(!(sum <= kPfGrowth)) != 0ull) {
      float top = s[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
      top = fmaxf(top, __shfl_xor(top, 32)) * kSoftmaxScaleLog2;
      const float mn = fmaxf(m, top), corr = fast_exp2(m - mn);
      m = mn;
      l *= corr;
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[c][i] *= corr;
      weights();
    }
    l += sum;
    uint32_t w[2][8];  // the weights' two terms
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[0][i] = BF16::round2(p[2 * i], p[2 * i + 1]);
      w[1][i] = BF16::round2(p[2 * i] - __uint_as_float(w[0][i] << 16), p[2 * i + 1] - __uint_as_float(w[0][i] & 0xffff0000u));
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int c = 0; c < 4; ++c)
          o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              va[ks][c], __builtin_bit_cast(am_bf16x8_t, make_uint4(w[t][4 * ks], w[t][4 * ks + 1], w[t][4 * ks + 2], w[t][4 * ks + 3])), o[c], 0, 0, 0);
  };

  if (s0 < s1) {
    load(s0);
    store(0);
    __syncthreads();
    for (int t = s0; t < s1; ++t) {
      if (t + 1 < s1) load(t + 1);
      const char* base = smem + ((t - s0) & 1) * 2 * kTileBytes;
      const SpanStep whole = span_step(steps, rows, t);
#pragma unroll 1
      for (int s = 0; s < kSteps; ++s) {
        const int key = (s * WK + wk) * 32;
        const SpanStep st{whole.at + key, whole.lo, whole.hi};
        // (all uniform for the wave)
        if (st.at >= min(st.hi, own.hi) || st.at + 32 <= st.lo || (st.at + 32 <= own.lo && st.at >= a.sinks)) continue;
        step(base + key * 256, st, span_full(a, own, st, 32));
      }
      if (t + 1 < s1) store((t + 1 - s0) & 1);
      __syncthreads();
    }
  }

  // both halves of a query's keys; then the waves that had other keys of the same queries
  l += __shfl_xor(l, 32);
  if constexpr (WK > 1) {
    float2* ml = reinterpret_cast<float2*>(smem);                   // [wave][32] (max, sum)
    float4* ob = reinterpret_cast<float4*>(smem + WAVES * 32 * 8);  // [wave of the upper half][4][4][lane]
    if (half == 0) ml[wave * 32 + l32] = make_float2(m, l);
    __syncthreads();
    float mn = kNegBig, ls = 0.f;
#pragma unroll
    for (int w = 0; w < WK; ++w) mn = fmaxf(mn, ml[(w * WQ + wq) * 32 + l32].x);
#pragma unroll
    for (int w = 0; w < WK; ++w) {
      const float2 x = ml[(w * WQ + wq) * 32 + l32];
      ls = fmaf(x.y, fast_exp2(x.x - mn), ls);
    }
    const float f = fast_exp2(m - mn);
    m = mn;
    l = ls;
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[c][i] *= f;
#pragma unroll
    for (int n = WK / 2; n >= 1; n /= 2) {
      if (wk >= n && wk < 2 * n) {
        float4* dst = ob + ((wk - n) * WQ + wq) * 16 * 64;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            dst[(c * 4 + i) * 64 + lane] = make_float4(o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]);
      }
      __syncthreads();
      if (wk < n) {
        const float4* src = ob + (wk * WQ + wq) * 16 * 64;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 x = src[(c * 4 + i) * 64 + lane];
            o[c][4 * i] += x.x;
            o[c][4 * i + 1] += x.y;
            o[c][4 * i + 2] += x.z;
            o[c][4 * i + 3] += x.w;
          }
      }
      __syncthreads();
    }
    if (wk != 0) return;
  }
  if (len == 0) l = 0.f;  // (a padded token's lanes took whatever full steps gave)
  const float inv = l > 0.f ? 1.0f / l : 0.f;  // (a token without rows: zeros)
  const bool parts = a.nsplit > 1;
  // a lane has four columns of one query at a time: through LDS, so that a store takes four half rows
  char* at = smem + wave * 8192;  // [32 queries][64 columns], 16-byte chunks exchanged as the keys'
#pragma unroll
  for (int pass = 0; pass < 2; ++pass) {
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const sp_f32x16_t& x = o[2 * pass + c];
        const float f = parts ? 1.0f : inv;
        *reinterpret_cast<float4*>(at + l32 * 256 + (((8 * c + 2 * i + half) ^ l16) * 16)) = make_float4(x[4 * i] * f, x[4 * i + 1] * f, x[4 * i + 2] * f, x[4 * i + 3] * f);
      }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int r = 4 * j + (lane >> 4);
      const float4 x = *reinterpret_cast<const float4*>(at + r * 256 + ((l16 ^ (r & 15)) * 16));
      if (q0 + r < live) {
        if (parts)
          *reinterpret_cast<float4*>(span_part(a, tile, q0 + r) + 64 * pass + 4 * l16) = x;
        else
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + span_place(a, tile.b, tile.h, r0 + q0 + r) * kD + 64 * pass + 4 * l16) = make_uint2(BF16::round2(x.x, x.y), BF16::round2(x.z, x.w));
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
  if (parts && half == 0 && row < live)
    *reinterpret_cast<float2*>(span_part(a, tile, row) + kD) = make_float2(m, l);
}

template <int WAVES, int WQ>
static hipError_t launch_tiles(const SpanArgs& a, dim3 grid, hipStream_t st) {
  static std::atomic<unsigned long long> raised{0};
  constexpr int bytes = span_lds_bytes<WAVES, WQ>();
  const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(&span_tiles_kernel<WAVES, WQ>), bytes, raised);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((span_tiles_kernel<WAVES, WQ>), grid, dim3(64 * WAVES), bytes, st, a);
  return hipGetLastError();
}

// ---- parts joined ---------------------------------------------------------------------------------------------------
// 32 lanes take a query row, 16 bytes of each of its parts; GROUPS of them share a row's parts, four each at a time.
template <typename T, int GROUPS>
__global__ __launch_bounds__(256) void span_merge_kernel(const float* __restrict__ partials, typename T::store_t* __restrict__ out,
                                                         long long rows, int nsplit) {
  constexpr int U = 4;
  __shared__ __align__(16) float s_o[GROUPS > 1 ? GROUPS : 1][kD];
  __shared__ float2 s_ml[GROUPS];
  const int lane = threadIdx.x & 31, grp = threadIdx.x >> 5;
  const long long r = GROUPS > 1 ? (long long)blockIdx.x : (long long)blockIdx.x * 8 + grp;
  if (GROUPS == 1 && r >= rows) return;
  const float* partial = partials + r * nsplit * kPartStride;
  float m = kNegBig, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i0 = GROUPS > 1 ? grp : 0; i0 < nsplit; i0 += GROUPS * U) {
    float2 ml[U];
    float4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * GROUPS;
      const float* p = partial + (long long)(i < nsplit ? i : i0) * kPartStride;
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
      if (ml[u].y > 0.f) {  // (a part without rows has no outputs)
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
  const float inv = l > 0.f ? 1.0f / l : 0.f;  // (a token without rows: zeros)
  if constexpr (T::EPC == 8)
    *reinterpret_cast<uint2*>(out + r * kD + 4 * lane) = make_uint2(BF16::round2(o.x * inv, o.y * inv), BF16::round2(o.z * inv, o.w * inv));
  else
    *reinterpret_cast<float4*>(out + r * kD + 4 * lane) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
}

// ---- the launch -----------------------------------------------------------------------------------------------------
SpanPlan span_plan(const Shape& s, int m, int window, int sinks, bool bits4) {
  SpanPlan p{16, 0, 1, 0};
  const long long M = (long long)m * s.G;
  const bool lds = s.dtype == 1 && !bits4 && M > 16;
  if (lds)
    p.rows = M <= 32 ? 32 : M <= 64 ? 64 : M <= 128 ? 128 : 256;
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
  const int least = lds ? 256 : 128;
  long long n = (slots + blocks - 1) / blocks;
  if (n > (read + least - 1) / least) n = (read + least - 1) / least;
  p.nsplit = n < 1 ? 1 : (int)n;
  p.run = (int)((read + p.nsplit - 1) / p.nsplit);
  return p;
}

hipError_t launch_span_q4(const Shape& s, const SpanArgs& a, hipStream_t st);

template <typename T>
static void launch_span_merge(const SpanArgs& a, hipStream_t st) {
  const long long rows = (long long)a.B * a.m * a.Hq;
  auto* out = static_cast<typename T::store_t*>(a.out);
  if (a.nsplit <= 4)
    hipLaunchKernelGGL((span_merge_kernel<T, 1>), dim3((unsigned)((rows + 7) / 8)), dim3(256), 0, st, a.partial, out, rows, a.nsplit);
  else
    hipLaunchKernelGGL((span_merge_kernel<T, 8>), dim3((unsigned)rows), dim3(256), 0, st, a.partial, out, rows, a.nsplit);
}

hipError_t launch_span(const Shape& s, SpanArgs a, hipStream_t st) {
  const bool bits4 = a.cache.k_scales != nullptr;
  const SpanPlan plan = span_plan(s, a.m, a.window, a.sinks, bits4);
  if (a.window == 0) {
    a.window = 0x7fffffff;
    a.sinks = 0;
  }
  a.rows = plan.rows;
  a.tiles = plan.tiles;
  a.nsplit = plan.nsplit;
  a.run = plan.run;
  const dim3 grid((unsigned)((long long)a.B * a.Hkv * a.tiles * a.nsplit)), block(64 * kSpWaves);
  hipError_t e = hipSuccess;
  // From 90 MB of rows on, of which none is read twice, values are loaded past the caches (row_loads in api.hip).  us through / past: 64
  // sequences of 64/8 heads with 4100 rows each 180 / 163, 16 of 32/8 with 16384 186 / 166, 13 with 4000 51.4 / 47.8, with 1500 (80 MB) 21.3 / 21.6;
  // fp32, 16 of 24 heads with 1000 rows 74.5 / 68.1, 5 with 703 (86 MB) 22.7 / 23.4.
  const bool past = plan.tiles == 1 && (double)a.B * a.Hkv * plan.nsplit * plan.run * (2 * kD * s.elem_bytes) >= kPastBytes;
  if (bits4)
    e = launch_span_q4(s, a, st);
  else if (s.dtype == 0 && plan.rows == 16 && past)
    hipLaunchKernelGGL((span_f32_kernel<1, true>), grid, block, 0, st, a);
  else if (s.dtype == 0 && plan.rows == 16)
    hipLaunchKernelGGL((span_f32_kernel<1, false>), grid, block, 0, st, a);
  else if (s.dtype == 0)
    hipLaunchKernelGGL((span_f32_kernel<2, false>), grid, block, 0, st, a);
  else if (plan.rows == 16 && past)
    hipLaunchKernelGGL((span_rows_kernel<true>), grid, block, 0, st, a);
  else if (plan.rows == 16)
    hipLaunchKernelGGL((span_rows_kernel<false>), grid, block, 0, st, a);
  else if (plan.rows == 32)
    e = launch_tiles<4, 1>(a, grid, st);
  else if (plan.rows == 64)
    e = launch_tiles<8, 2>(a, grid, st);
  else if (plan.rows == 128)
    e = launch_tiles<8, 4>(a, grid, st);
  else
    e = launch_tiles<8, 8>(a, grid, st);
  if (e == hipSuccess) e = hipGetLastError();
  if (e != hipSuccess || a.nsplit == 1) return e;
  if (s.dtype == 1)
    launch_span_merge<BF16>(a, st);
  else
    launch_span_merge<F32>(a, st);
  return hipGetLastError();
}

}  // namespace loki
