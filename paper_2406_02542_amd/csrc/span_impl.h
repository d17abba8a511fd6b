// What the attention kernels over a whole cache share (span.hip, span_q4.hip): which rows a tile of query rows reads, which of them a
// token sees, and where a tile's results go.
//
// A tile is ROWS consecutive query rows r = j G + g (token j, query head g of the KV head) of one sequence and KV head.  A token that sees
// L rows sees row s < L where s < sinks or s >= L - window.  The tile reads [0, nsink) and [lo, hi): lo goes by its shortest token, hi by
// its longest; tokens with L = 0 (padding) are not asked.  Rows are taken in steps of 32 or 16 that begin at multiples of 16, so that
// 16 rows lie in one page; rows outside the two ranges are never loaded (the range's last or first row is, again).
#pragma once

#include "cache_impl.h"
#include "parts_impl.h"

namespace loki {

constexpr float kUnseen = -3.0e38f;  // a logit that no maximum follows and whose weight is 0 whatever the maximum is

__device__ __forceinline__ int span_len(const SpanArgs& a, int b, int j) {
  if (a.lens == nullptr) return max(0, a.S_max - (a.m - 1 - j));
  return min(max(a.lens[(long long)b * a.m + j], 0), a.S_max);
}

struct SpanRows {
  int lo, hi, nsink;  // of the tile
  int len_min;        // the shortest token's rows (not 0), hi the longest's
};
// Of tokens j0 .. j1 of sequence b; every wave for itself.
__device__ __forceinline__ SpanRows span_rows(const SpanArgs& a, int b, int j0, int j1) {
  int most = 0, least = 0;  // least: S_max less the shortest
  const int lane = threadIdx.x & 63;
  for (int j = j0 + lane; j - lane <= j1; j += 64) {
    const int len = j <= j1 ? span_len(a, b, j) : 0;
    most = max(most, len);
    least = max(least, len > 0 ? a.S_max - len : 0);
  }
  SpanRows r;
  r.hi = wave_max_i32(most);
  r.len_min = a.S_max - wave_max_i32(least);
  r.lo = r.hi > 0 ? max(0, r.len_min - a.window) : 0;
  r.nsink = min(a.sinks, r.lo);
  return r;
}

// Steps of a tile: those of the sinks, then those of the window.
template <int KEYS>
struct SpanSteps {
  int sinks, base, total;
  __device__ __forceinline__ explicit SpanSteps(const SpanRows& r) {
    sinks = (r.nsink + KEYS - 1) / KEYS;
    base = r.lo & ~15;
    total = sinks + (r.hi - base + KEYS - 1) / KEYS;
  }
};
struct SpanStep {
  int at, lo, hi;  // rows at .., of which [lo, hi) are there
};
template <int KEYS>
__device__ __forceinline__ SpanStep span_step(const SpanSteps<KEYS>& n, const SpanRows& r, int s) {
  return s < n.sinks ? SpanStep{s * KEYS, 0, r.nsink} : SpanStep{n.base + (s - n.sinks) * KEYS, r.lo, r.hi};
}

// The places of a step's TILES tiles of 16 rows (the range's first or last row's, where a tile lies outside): asked for a step ahead,
// settled when the step's rows are loaded.
template <int TILES>
struct SpanPlaces {
  int row[TILES], entry[TILES];
  long long at[TILES];  // of the tile's first row, which may lie outside
  __device__ __forceinline__ void ask(const RowPlaces& places, const SpanStep& st) {
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      row[t] = min(max(st.at + 16 * t, st.lo), st.hi - 1);
      entry[t] = places.entry(row[t]);
    }
  }
  __device__ __forceinline__ void settle(const RowPlaces& places, const SpanStep& st) {
#pragma unroll
    for (int t = 0; t < TILES; ++t) at[t] = places.place(row[t], entry[t]) + st.at + 16 * t;
  }
};
// Row `i` of tile t of a step from the tile's first: itself, or the range's last or first.
__device__ __forceinline__ int span_near(const SpanStep& st, int t, int i) {
  const int first = st.at + 16 * t;
  return min(max(first + i, st.lo), st.hi - 1) - first;
}
// f(whole): whether the step's rows are all there, so that they lie at fixed distances.  (The empty statements keep the compiler from taking
// the loads of both branches together, for which it would carry an address for each in registers.)
template <int KEYS, typename F>
__device__ __forceinline__ void span_loads(const SpanStep& st, F f) {
  if (st.at >= st.lo && st.at + KEYS <= st.hi) {  // (uniform)
    f(std::true_type{});
    asm volatile("" ::: "memory");
  } else {
    f(std::false_type{});
    asm volatile("" ::: "memory");
  }
}

// Whether a token that sees `len` rows sees row s of a step.
__device__ __forceinline__ bool span_sees(const SpanArgs& a, const SpanStep& st, int len, int s) {
  return s >= st.lo && s < min(st.hi, len) && (s >= len - a.window || s < a.sinks);
}
// Whether every token of the tile sees all of the step's `keys` rows.
__device__ __forceinline__ bool span_full(const SpanArgs& a, const SpanRows& r, const SpanStep& st, int keys) {
  return st.at >= st.lo && st.at + keys <= min(st.hi, r.len_min) && (st.at >= r.hi - a.window || st.at + keys <= a.sinks);
}

// A row that a token does not see may hold anything, and a product with a weight of zero is no zero where it holds no finite number.  So in
// steps that are masked such values are cleared, and which of them a token sees is a product of its own, of ones: a column's count, and where
// it is not zero the output is no number.
__device__ __forceinline__ float span_mark(float o, float count) { return count > 0.f ? __builtin_nanf("") : o; }
// The halves of x that are no finite bf16 number (all ones as exponents, which one more carries into the sign's place): in bits 0 and 16;
// as ones; and x with zeros for them.
__device__ __forceinline__ uint32_t bf16_not_finite(uint32_t x) { return ((x & 0x7f807f80u) + 0x00800080u) >> 15 & 0x00010001u; }
__device__ __forceinline__ uint32_t bf16_marks(uint32_t x) { return bf16_not_finite(x) * 0x3f80u; }
__device__ __forceinline__ uint32_t bf16_finite(uint32_t x) { return x & ~(bf16_not_finite(x) * 0xffffu); }
__device__ __forceinline__ uint32_t f32_not_finite(float x) { return ((__float_as_uint(x) & 0x7f800000u) + 0x00800000u) >> 31; }

// What a block does: steps [s0, s1) of a tile, part `part` of its nsplit.
struct SpanTile {
  int b, h, tile, part, s0, s1;
  SpanRows rows;
};

// Query row r of a sequence: its place among the rows of q, of out and of the parts.
__device__ __forceinline__ long long span_place(const SpanArgs& a, int b, int h, int r) {
  const int j = r >> (31 - __builtin_clz(a.G));
  return ((long long)b * a.m + j) * a.Hq + h * a.G + (r & (a.G - 1));
}
// Where query row r of the tile has this block's part.
__device__ __forceinline__ float* span_part(const SpanArgs& a, const SpanTile& t, int r) {
  return a.partial + (span_place(a, t.b, t.h, t.tile * a.rows + r) * a.nsplit + t.part) * kPartStride;
}

// This block's tile and its share of the tile's steps: runs of equal length, so that blocks have equal work whatever the lengths and short
// sequences fewer of them (more rows than expected, of tokens that do not lie next to each other, make a tile's runs longer).  us with the
// rows of each sequence in equal parts and so: 16 sequences of 32/8 bf16 heads up to 16384 rows 144, 136; 5 of 24 fp32 heads up to 2311 in
// 4 bits 19.1, 16.8.
template <int KEYS>
__device__ __forceinline__ SpanTile span_tile(const SpanArgs& a) {
  SpanTile t;
  int x = blockIdx.x;
  t.h = x % a.Hkv;  // (a run's heads next to each other)
  x /= a.Hkv;
  t.part = x % a.nsplit;
  x /= a.nsplit;
  t.b = x / a.tiles;
  t.tile = a.tiles - 1 - (x - t.b * a.tiles);  // (the last tokens see the most)
  const int r0 = t.tile * a.rows, lg = 31 - __builtin_clz(a.G), last = min(r0 + a.rows, a.m * a.G) - 1;
  t.rows = span_rows(a, t.b, r0 >> lg, last >> lg);
  const SpanSteps<KEYS> n(t.rows);
  const int each = max((a.run + KEYS - 1) / KEYS, (n.total + a.nsplit - 1) / a.nsplit);
  t.s0 = t.part * each;
  t.s1 = min(n.total, t.s0 + each);
  return t;
}

// A run that no row is left for: its parts say so, which the merge goes by.
__device__ __forceinline__ void span_none(const SpanArgs& a, const SpanTile& t, int live) {
  for (int r = threadIdx.x; r < live; r += blockDim.x) *reinterpret_cast<float2*>(span_part(a, t, r) + kD) = make_float2(kNegBig, 0.f);
}

// A wave's state after its steps, for 16 query rows: lane (row r16, kgrp) holds maximum m and sum l of its row (l its own share of the
// rows), columns col(c, i) of the row's output in o[c][i].
template <int ROWS, int WAVES>
struct SpanMerge {
  float2 ml[WAVES][ROWS];
  float o[WAVES][ROWS][kD];
};

// The waves' results joined: `live` query rows of the tile, out or as parts.  Begins with a barrier.
template <typename T, int ROWS, int WAVES>
__device__ __forceinline__ void span_store(const SpanArgs& a, const SpanMerge<ROWS, WAVES>& sm, const SpanTile& tile, int r0, int live) {
  __syncthreads();
  for (int i = threadIdx.x; i < live * (kD / 4); i += 64 * WAVES) {
    const int r = i / (kD / 4), c = i % (kD / 4) * 4;
    float mn = kNegBig, ls = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) mn = fmaxf(mn, sm.ml[w][r].x);
    float4 os = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float f = fast_exp2(sm.ml[w][r].x - mn);
      const float4 x = *reinterpret_cast<const float4*>(&sm.o[w][r][c]);
      ls = fmaf(sm.ml[w][r].y, f, ls);
      os = make_float4(fmaf(x.x, f, os.x), fmaf(x.y, f, os.y), fmaf(x.z, f, os.z), fmaf(x.w, f, os.w));
    }
    if (a.nsplit > 1) {
      float* p = span_part(a, tile, r);
      *reinterpret_cast<float4*>(p + c) = os;
      if (c == 0) *reinterpret_cast<float2*>(p + kD) = make_float2(mn, ls);
    } else {
      const long long place = span_place(a, tile.b, tile.h, r0 + r);
      const float inv = ls == 0.f ? 0.f : 1.0f / ls;  // (a token without rows: zeros)
      if constexpr (T::EPC == 8)
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + place * kD + c) =
            make_uint2(BF16::round2(os.x * inv, os.y * inv), BF16::round2(os.z * inv, os.w * inv));
      else
        *reinterpret_cast<float4*>(static_cast<float*>(a.out) + place * kD + c) = make_float4(os.x * inv, os.y * inv, os.z * inv, os.w * inv);
    }
  }
}

}  // namespace loki
