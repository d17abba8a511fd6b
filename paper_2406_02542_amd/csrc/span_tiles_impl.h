// Attention over a whole cache for many query rows of a KV head, bf16 queries: tiles of keys and values through LDS (span.hip: rows in the
// storage type; span_q4.hip: in 4 bits).
//
// The products of shared.hip's prefix kernel: a wave holds 32 query rows and takes steps of 32 keys, S^T = K Q^T and O^T += V^T P^T by
// v_mfma_f32_32x32x16_bf16, the weights in two bf16 terms as they come out of the first product.  Tiles of KT keys and values go through LDS
// once for the block's waves, WQ of which hold different queries and WK = WAVES / WQ different keys of the tile; the next tile is loaded into
// registers while this one is used.  What is masked is decided for a wave's step as a whole: nothing to see, everything, or each on its own.
// In 4 bits a tile is unpacked on its way into LDS, once for all of the block's queries, into two bf16 terms a value, and meets them in two and
// three products where the storage type's takes one and two.
// The matrix cores bound it: 2 x 2048 tokens of 32/8 heads, window 4096 (275 GFLOP) 385 us, 0.71 PFLOP/s, 1.07 with the weights' second term (a library product of
// 8192 cubed 1.14); in 4 bits 4 x 64 tokens of 32/8 behind 8192 rows 93 us, 0.37.
#pragma once

#include "span_impl.h"

namespace loki {

// Codes g of a word's halves as two bf16 numbers 1 + n / 16.  The constants are kept in registers: one instruction takes both then.
struct Q4Pair {
  uint32_t mask = 0x00780078u, one = 0x3f803f80u;
  __device__ __forceinline__ Q4Pair() { asm("" : "+v"(mask), "+s"(one)); }
  __device__ __forceinline__ uint32_t operator()(uint32_t x, int g) const { return ((g == 0 ? x << 3 : x >> (4 * g - 3)) & mask) | one; }
};

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

typedef short sp_s16x4_t __attribute__((ext_vector_type(4)));
typedef float sp_f32x16_t __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) sp_s16x4_t sp_lds_s16x4_t;

template <int WAVES, int WQ>
constexpr int span_tile_keys() {
  return WAVES / WQ == 4 ? 128 : 64;
}
// (step, lowest) of a row's groups and a chunk of its words, 4 c .., of keys or of values: columns 32 g + 8 c .. of every group, each value in two
// bf16 terms (2^-17 of it), 16 bytes a group for each.
struct SpanQ4Chunk {
  uint4 words, scales;
  __device__ __forceinline__ void operator()(const Q4Pair& pair, int g, uint4& hi, uint4& lo) const {
    const cache_half2_t sc = __builtin_bit_cast(cache_half2_t, am_word(scales, g));
    const float step = 16.f * (float)sc.x, base = (float)sc.y - step;
    uint32_t w[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t n = pair(am_word(words, i), g);  // numbers 1 + n / 16
      q4_terms<2>(fmaf(step, __uint_as_float(n << 16), base), fmaf(step, __uint_as_float(n & 0xffff0000u), base), w[i]);
    }
    hi = make_uint4(w[0][0], w[1][0], w[2][0], w[3][0]);
    lo = make_uint4(w[0][1], w[1][1], w[2][1], w[3][1]);
  }
};
// Two pairs of tiles; at the end, where waves have other keys of the same queries, what half of them hand over, or the outputs.
template <int WAVES, int WQ, bool BITS4>
constexpr int span_lds_bytes() {
  const int tiles = (BITS4 ? 8 : 4) * span_tile_keys<WAVES, WQ>() * 256, merge = WAVES * 32 * 8 + WAVES / 2 * 64 * 256;
  return tiles > merge ? tiles : merge;
}

template <int WAVES, int WQ, bool BITS4, bool HALVES>
__global__ __launch_bounds__(64 * WAVES, 2) void span_tiles_kernel(SpanArgs a) {
  extern __shared__ __align__(16) char smem[];  // [2][K tile, V tile], in 4 bits [2][K tile's terms, V tile's terms]
  constexpr int kThreads = 64 * WAVES, WK = WAVES / WQ, KT = span_tile_keys<WAVES, WQ>(), kSteps = KT / (32 * WK);
  constexpr int kChunks = BITS4 ? KT * 8 / kThreads : KT * 16 / kThreads;  // of a thread, of keys and of values (4 bits: of either)
  constexpr int kTileBytes = KT * 256, kBufferBytes = (BITS4 ? 4 : 2) * kTileBytes, kValues = kBufferBytes / 2;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, half = lane >> 5, l16 = lane & 15;
  SpanTile tile;
  if constexpr (HALVES) {
    tile = span_tile_halves(a);
    if (tile.h < 0) return;  // (uniform for the block)
  } else {
    tile = span_tile<KT, false>(a);
  }
  // half of a tile: as WQ / 2 waves of queries, and two of keys
  const bool half_tile = HALVES && tile.half != 0;
  const int wq = half_tile ? wave % (WQ / 2) : wave % WQ, wk = half_tile ? wave / (WQ / 2) : wave / WQ;
  const int M = a.m * a.G, r0 = tile.tile * (32 * WQ) + (tile.half == 2 ? 16 * WQ : 0), lg = 31 - __builtin_clz(a.G);
  const int live = min(half_tile ? 16 * WQ : 32 * WQ, M - r0);
  const SpanRows rows = tile.rows;
  const SpanSteps<KT> steps(rows);
  if (tile.s0 >= tile.s1 && tile.part > 0) return span_none<false>(a, tile, live);  // (uniform for the block)
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
    for (int ks = 0; ks < 8; ++ks) q[ks] = __builtin_bit_cast(am_bf16x8_t, span_query(load16(src + 16 * ks), len));
  }
  uint4 kst[BITS4 ? 1 : kChunks], vst[BITS4 ? 1 : kChunks];
  SpanQ4Chunk cst[BITS4 ? kChunks : 1];
  const Q4Pair pair;
  // A thread's chunk j: of row `row` of the tile; in 4 bits chunk c of the row's four, of keys or of values.
  struct At {
    int row, c;
    bool values;
  };
  auto chunk_at = [&](int j) __attribute__((always_inline)) {
    const int at = tid + kThreads * j;
    return BITS4 ? At{at >> 2 & (KT - 1), at & 3, at >= 4 * KT} : At{at >> 4, at & 15, false};
  };
  auto load = [&](int s) __attribute__((always_inline)) {  // (a wave's rows of a chunk, 4 or 16, lie in one page)
    const SpanStep st = span_step(steps, rows, s);
#pragma unroll
    for (int j = 0; j < kChunks; ++j) {
      const At at = chunk_at(j);
      const int first = st.at + __builtin_amdgcn_readfirstlane(at.row);
      const long long row = places(min(max(first, st.lo), st.hi - 1)) + min(max(st.at + at.row, st.lo), st.hi - 1);
      if constexpr (BITS4) {
        const bool values = __builtin_amdgcn_readfirstlane(at.values);
        cst[j].words = load16(static_cast<const char*>(values ? a.cache.v : a.cache.k) + row * kQ4RowBytes + 16 * at.c);
        cst[j].scales = load16(static_cast<const char*>(values ? a.cache.v_scales : a.cache.k_scales) + row * kQ4ScaleBytes);
      } else {
        kst[j] = load16(static_cast<const uint16_t*>(a.cache.k) + row * kD + at.c * 8);
        vst[j] = load16(static_cast<const uint16_t*>(a.cache.v) + row * kD + at.c * 8);
      }
    }
  };
  auto store = [&](int b) __attribute__((always_inline)) {
    char* base = smem + b * kBufferBytes;
#pragma unroll
    for (int j = 0; j < kChunks; ++j) {
      const At at = chunk_at(j);
      if constexpr (BITS4) {
        char* row = base + (at.values ? kValues : 0) + at.row * 256;
        const int turn = at.values ? (at.row & 3) << 2 : at.row & 15;
#pragma unroll
        for (int g = 0; g < kQ4Groups; ++g) {
          uint4 hi, lo;
          cst[j](pair, g, hi, lo);
          const int c = ((4 * g + at.c) ^ turn) * 16;
          *reinterpret_cast<uint4*>(row + c) = hi;
          *reinterpret_cast<uint4*>(row + kTileBytes + c) = lo;
        }
      } else {
        *reinterpret_cast<uint4*>(base + at.row * 256 + ((at.c ^ (at.row & 15)) * 16)) = kst[j];
        *reinterpret_cast<uint4*>(base + kValues + at.row * 256 + ((at.c ^ ((at.row & 3) << 2)) * 16)) = vst[j];
      }
    }
  };

  float m = kNegBig, l = 0.f;
  sp_f32x16_t o[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) o[c] = sp_f32x16_t{};
  const int k_at = l32 * 256 + ((half ^ l16) * 16);
  const int v_row = 4 * half + (l16 >> 2);
  const int v_at = kValues + v_row * 256 + (((((lane >> 4) & 1) * 2 + ((l16 & 3) >> 1)) ^ ((v_row & 3) << 2)) * 16) + (l16 & 1) * 8;

  // 32 keys of the tile in buffer `base`, rows st.at ..; full: all of them are seen by all of the wave's queries
  auto step = [&](const char* base, const SpanStep& st, bool full) __attribute__((always_inline)) {
    am_bf16x8_t ka[8], va[2][4];
    auto values = [&](int term) __attribute__((always_inline)) {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const char* at = base + (v_at ^ (c * 64)) + ks * 4096 + term * kTileBytes;
          const sp_s16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((sp_lds_s16x4_t*)(at));
          const sp_s16x4_t y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((sp_lds_s16x4_t*)(at + 2048));
          va[ks][c] = __builtin_bit_cast(am_bf16x8_t, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    };
    sp_f32x16_t s = sp_f32x16_t{};
    if constexpr (BITS4) {
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) ka[ks] = __builtin_bit_cast(am_bf16x8_t, *reinterpret_cast<const uint4*>(base + kTileBytes + (k_at ^ (ks * 32))));
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[ks], q[ks], s, 0, 0, 0);
    }
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) ka[ks] = __builtin_bit_cast(am_bf16x8_t, *reinterpret_cast<const uint4*>(base + (k_at ^ (ks * 32))));
    __builtin_amdgcn_sched_barrier(0);
    values(0);
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[ks], q[ks], s, 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
    // whether any of the values in registers is no finite number (span_mark)
    auto odd = [&]() __attribute__((always_inline)) {
      uint32_t x = 0;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int w = 0; w < 4; ++w) x |= bf16_not_finite(am_word(__builtin_bit_cast(uint4, va[ks][c]), w));
      return __ballot(x != 0) != 0ull;
    };
    if (!full) {  // (uniform)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (!span_sees(a, st, len, st.at + 8 * (i >> 2) + 4 * half + (i & 3))) s[i] = kUnseen;
      if (odd()) {
        uint32_t ones[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float x = s[2 * i], y = s[2 * i + 1];
          asm volatile("" : "+v"(x), "+v"(y));  // (else the masks of all of them stay in scalar registers, which there are too few of)
          ones[i] = (x != kUnseen ? 0x3f80u : 0u) | (y != kUnseen ? 0x3f800000u : 0u);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          sp_f32x16_t count = sp_f32x16_t{};
#pragma unroll
          for (int ks = 0; ks < 2; ++ks) {
            uint4 x = __builtin_bit_cast(uint4, va[ks][c]);
            asm volatile("" : "+v"(x.x), "+v"(x.y), "+v"(x.z), "+v"(x.w));  // (else what was found above is kept, in as many registers)
            const uint4 bad = make_uint4(bf16_marks(x.x), bf16_marks(x.y), bf16_marks(x.z), bf16_marks(x.w));
            count = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                __builtin_bit_cast(am_bf16x8_t, bad),
                __builtin_bit_cast(am_bf16x8_t, make_uint4(ones[4 * ks], ones[4 * ks + 1], ones[4 * ks + 2], ones[4 * ks + 3])), count, 0, 0, 0);
            va[ks][c] = __builtin_bit_cast(am_bf16x8_t, make_uint4(bf16_finite(x.x), bf16_finite(x.y), bf16_finite(x.z), bf16_finite(x.w)));
            __builtin_amdgcn_sched_barrier(0);
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) o[c][i] = span_mark(o[c][i], count[i]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
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
    if constexpr (BITS4) {  // (the two second terms' product is 2^-18 of the first two's)
      values(1);
      if (!full && odd()) {
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const uint4 x = __builtin_bit_cast(uint4, va[ks][c]);
            va[ks][c] = __builtin_bit_cast(am_bf16x8_t, make_uint4(bf16_finite(x.x), bf16_finite(x.y), bf16_finite(x.z), bf16_finite(x.w)));
          }
      }
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int c = 0; c < 4; ++c)
          o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              va[ks][c], __builtin_bit_cast(am_bf16x8_t, make_uint4(w[0][4 * ks], w[0][4 * ks + 1], w[0][4 * ks + 2], w[0][4 * ks + 3])), o[c], 0, 0, 0);
    }
  };

  if (s0 < s1) {
    load(s0);
    store(0);
    __syncthreads();
    for (int t = s0; t < s1; ++t) {
      if (t + 1 < s1) load(t + 1);
      const char* base = smem + ((t - s0) & 1) * kBufferBytes;
      const SpanStep whole = span_step(steps, rows, t);
#pragma unroll 1
      for (int s = 0; s < (half_tile ? kSteps / 2 : kSteps); ++s) {
        const int key = half_tile ? (2 * s + wk) * 32 : (s * WK + wk) * 32;
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
  if (len == 0) {  // (a padded token's lanes took whatever full steps gave, a maximum too)
    m = kNegBig;
    l = 0.f;
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] = sp_f32x16_t{};
  }
  if ((HALVES && half_tile) || WK > 1) {  // (uniform)
    constexpr int Q = HALVES ? WQ / 2 : WQ, K = WAVES / Q;
    float2* ml = reinterpret_cast<float2*>(smem);                   // [wave][32] (max, sum)
    float4* ob = reinterpret_cast<float4*>(smem + WAVES * 32 * 8);  // [wave of the upper half][4][4][lane]
    if (half == 0) ml[wave * 32 + l32] = make_float2(m, l);
    __syncthreads();
    float mn = kNegBig, ls = 0.f;
#pragma unroll
    for (int w = 0; w < K; ++w) mn = fmaxf(mn, ml[(w * Q + wq) * 32 + l32].x);
#pragma unroll
    for (int w = 0; w < K; ++w) {
      const float2 x = ml[(w * Q + wq) * 32 + l32];
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
    for (int n = K / 2; n >= 1; n /= 2) {
      if (wk >= n && wk < 2 * n) {
        float4* dst = ob + ((wk - n) * Q + wq) * 16 * 64;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            dst[(c * 4 + i) * 64 + lane] = make_float4(o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]);
      }
      __syncthreads();
      if (wk < n) {
        const float4* src = ob + (wk * Q + wq) * 16 * 64;
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
  const float inv = l == 0.f ? 0.f : 1.0f / l;  // (a token without rows: zeros)
  const bool parts = tile.parts > 1;
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
          *reinterpret_cast<float4*>(span_part<false>(a, tile, q0 + r) + 64 * pass + 4 * l16) = x;
        else
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + span_place(a, tile.b, tile.h, r0 + q0 + r) * kD + 64 * pass + 4 * l16) = make_uint2(BF16::round2(x.x, x.y), BF16::round2(x.z, x.w));
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
  if (parts && half == 0 && row < live)
    *reinterpret_cast<float2*>(span_part<false>(a, tile, row) + kD) = make_float2(m, l);
}

template <int WAVES, int WQ, bool BITS4, bool HALVES = false>
static hipError_t launch_span_tiles(const SpanArgs& a, unsigned blocks, hipStream_t st) {
  static std::atomic<unsigned long long> raised{0};
  constexpr int bytes = span_lds_bytes<WAVES, WQ, BITS4>();
  const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(&span_tiles_kernel<WAVES, WQ, BITS4, HALVES>), bytes, raised);
  if (e != hipSuccess) return e;
  const dim3 grid(blocks);
  hipLaunchKernelGGL((span_tiles_kernel<WAVES, WQ, BITS4, HALVES>), grid, dim3(64 * WAVES), bytes, st, a);
  return hipGetLastError();
}

}  // namespace loki
