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

struct SpanTile {
  int b, h, tile, split;
};
__device__ __forceinline__ SpanTile span_tile(const SpanArgs& a) {
  int x = blockIdx.x;
  const int h = x % a.Hkv;
  x /= a.Hkv;
  const int split = x % a.nsplit;
  x /= a.nsplit;
  return {x / a.tiles, h, x % a.tiles, split};
}

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

// Whether a token that sees `len` rows sees row s of a step.
__device__ __forceinline__ bool span_sees(const SpanArgs& a, const SpanStep& st, int len, int s) {
  return s >= st.lo && s < min(st.hi, len) && (s >= len - a.window || s < a.sinks);
}
// Whether every token of the tile sees all of the step's `keys` rows.
__device__ __forceinline__ bool span_full(const SpanArgs& a, const SpanRows& r, const SpanStep& st, int keys) {
  return st.at >= st.lo && st.at + keys <= min(st.hi, r.len_min) && (st.at >= r.hi - a.window || st.at + keys <= a.sinks);
}

// The steps of this block's run: the same number for every tile, so that blocks have equal work whatever the lengths; a tile has as many
// runs as its rows fill (more rows than expected, of tokens that do not lie next to each other, make its runs longer).
template <int KEYS>
struct SpanRun {
  int s0, s1;
  __device__ __forceinline__ SpanRun(const SpanArgs& a, const SpanSteps<KEYS>& n, int split) {
    const int each = max((a.run + KEYS - 1) / KEYS, (n.total + a.nsplit - 1) / a.nsplit);
    s0 = split * each;
    s1 = min(n.total, s0 + each);
  }
};

// Query row r of a sequence: its place among the rows of q, of out and of the parts.
__device__ __forceinline__ long long span_place(const SpanArgs& a, int b, int h, int r) {
  const int j = r >> (31 - __builtin_clz(a.G));
  return ((long long)b * a.m + j) * a.Hq + h * a.G + (r & (a.G - 1));
}

// A run that no row is left for: its parts say so, which the merge asks for in front of their outputs.
__device__ __forceinline__ void span_none(const SpanArgs& a, const SpanTile& tile, int r0, int live) {
  for (int r = threadIdx.x; r < live; r += blockDim.x)
    *reinterpret_cast<float2*>(a.partial + (span_place(a, tile.b, tile.h, r0 + r) * a.nsplit + tile.split) * kPartStride + kD) = make_float2(kNegBig, 0.f);
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
    const long long place = span_place(a, tile.b, tile.h, r0 + r);
    if (a.nsplit > 1) {
      float* p = a.partial + (place * a.nsplit + tile.split) * kPartStride;
      *reinterpret_cast<float4*>(p + c) = os;
      if (c == 0) *reinterpret_cast<float2*>(p + kD) = make_float2(mn, ls);
    } else {
      const float inv = ls > 0.f ? 1.0f / ls : 0.f;  // (a token without rows: zeros)
      if constexpr (T::EPC == 8)
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + place * kD + c) =
            make_uint2(BF16::round2(os.x * inv, os.y * inv), BF16::round2(os.z * inv, os.w * inv));
      else
        *reinterpret_cast<float4*>(static_cast<float*>(a.out) + place * kD + c) = make_float4(os.x * inv, os.y * inv, os.z * inv, os.w * inv);
    }
  }
}

}  // namespace loki
