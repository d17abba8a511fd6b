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
// Of tokens that see from `least` to `most` rows.
__device__ __forceinline__ SpanRows span_rows_of(const SpanArgs& a, int least, int most) {
  SpanRows r;
  r.hi = most;
  r.len_min = least;
  r.lo = most > 0 ? max(0, least - a.window) : 0;
  r.nsink = min(a.sinks, r.lo);
  return r;
}
// Of tokens j0 .. j1 of sequence b; every wave for itself.
__device__ __forceinline__ SpanRows span_rows(const SpanArgs& a, int b, int j0, int j1) {
  int most = 0, least = 0;  // least: S_max less the shortest
  const int lane = threadIdx.x & 63;
  for (int j = j0 + lane; j - lane <= j1; j += 64) {
    const int len = j <= j1 ? span_len(a, b, j) : 0;
    most = max(most, len);
    least = max(least, len > 0 ? a.S_max - len : 0);
  }
  const int hi = wave_max_i32(most);
  return span_rows_of(a, a.S_max - wave_max_i32(least), hi);
}

// 16 bytes of the query of a token that sees `len` rows.  A padded token's lanes take part in steps that all others see whole: with zeros, so that no
// reference of the exponentials, which a wave moves for all of its lanes at once, goes by what such a query holds.
__device__ __forceinline__ uint4 span_query(uint4 x, int len) {
  return len == 0 ? make_uint4(0, 0, 0, 0) : x;
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

// What a block does: steps [s0, s1) of a tile, run `part` of its `parts`.
struct SpanTile {
  int b, h, tile, part, parts, s0, s1;  // h < 0: nothing
  int slot;  // the run's number
  int half;  // 0, or of a tile's rows the first (1) or the second (2) half
  SpanRows rows;
};

// Query row r of a sequence: its place among the rows of q, of out and of the parts.
__device__ __forceinline__ long long span_place(const SpanArgs& a, int b, int h, int r) {
  const int j = r >> (31 - __builtin_clz(a.G));
  return ((long long)b * a.m + j) * a.Hq + h * a.G + (r & (a.G - 1));
}
// Where query row r of the tile has this block's part.
template <bool DEALT>
__device__ __forceinline__ float* span_part(const SpanArgs& a, const SpanTile& t, int r) {
  const long long at = DEALT ? ((long long)t.slot * a.Hkv + t.h) * a.rows + r : span_place(a, t.b, t.h, t.tile * a.rows + r) * a.nsplit + t.part;
  return a.partial + at * kPartStride;
}

// Tiles in the order in which blocks take them, the last tokens first, which see the most: sequence by sequence, so that neighbours read the same
// rows; where tokens see all rows and tiles are not cut, so that blocks differ in length, the last of every sequence, then the ones before.  us sequence
// by sequence / so: prompts with nothing before them, 4 x 1024 tokens of 32/8 bf16 heads 86.6 / 66.3, 16 x 512 111 / 97, 8 x 512 of 16/8 fp32 heads 134 / 114;
// 4 x 1024 up to 4096 rows 356 / 336; with a window 4096, 16 x 100 of 64/8 156 / 161.
__device__ __forceinline__ bool span_longest_first(const SpanArgs& a) { return a.window == 0x7fffffff && a.nsplit == 1; }
__device__ __forceinline__ void span_tile_at(const SpanArgs& a, int t, int& b, int& tile) {
  const int n = span_longest_first(a) ? a.B : a.tiles, x = t / n, y = t - x * n;
  b = span_longest_first(a) ? y : x;
  tile = a.tiles - 1 - (span_longest_first(a) ? x : y);
}
__device__ __forceinline__ int span_tile_index(const SpanArgs& a, int b, int tile) {
  return span_longest_first(a) ? (a.tiles - 1 - tile) * a.B + b : b * a.tiles + a.tiles - 1 - tile;
}
// Of 64 tiles t0 .. those whose first token sees rows, and those that there are; `len`: of the lane's tile, the rows that token reads.
__device__ __forceinline__ unsigned long long span_there(const SpanArgs& a, int t0, unsigned long long& tiles, int& len) {
  const int at = t0 + (int)(threadIdx.x & 63), all = a.B * a.tiles;
  int b, tile;
  span_tile_at(a, min(at, all - 1), b, tile);
  tiles = __ballot(at < all);
  len = at < all ? min(span_len(a, b, tile * a.rows >> (31 - __builtin_clz(a.G))), a.window) : 0;
  return __ballot(len > 0);
}
// Blocks of tiles without parts, of which a CU holds one: whole rounds of tiles, and what is left, if it is no more than half a round, in halves of
// their query rows, which take a little more than half the time (tiles of that few rows do so anyway).  All are halved where the longest would take longer
// than all together otherwise.  Tiles of padded tokens come last.  us without / so: 16 chunks of up to 100 tokens of 64/8 heads, window 2048 186 / 156, 4 of
// up to 700 of 32/8, window 4096 303 / 288, 2 of up to 2048 (of three pairs of lengths one leaves that little) 358 / 336; 2048 tokens of 32/32, all halved, 88 / 73.
__device__ __forceinline__ SpanTile span_tile_halves(const SpanArgs& a) {
  SpanTile t{};
  const int all = a.B * a.tiles, lg = 31 - __builtin_clz(a.G);
  unsigned long long tiles;
  int there = 0, longest = 0, len;
  float total = 0.f;
  for (int t0 = 0; t0 < all; t0 += 64) {
    there += __popcll(span_there(a, t0, tiles, len));
    longest = max(longest, len);
    total += (float)len;
  }
  const int blocks = there * a.Hkv, whole = blocks / a.halves * a.halves, rest = blocks - whole;
  const bool cut = 2 * rest <= a.halves;
  const bool cut_all = a.halves_all && wave_sum_f32(total) * (float)a.Hkv * 1.14f < 0.95f * (float)wave_max_i32(longest) * (float)a.halves;
  const int busy = cut_all ? 2 * blocks : cut ? whole + 2 * rest : blocks;
  int x = blockIdx.x;
  const bool padded = x >= busy;
  if (padded) {
    x -= busy;
  } else if (cut_all) {
    const int y = x / a.Hkv;  // (heads next to each other)
    t.half = 1 + (y & 1);
    x -= (y + 1) / 2 * a.Hkv;
  } else if (cut && x >= whole) {
    t.half = x < whole + rest ? 1 : 2;
    x -= t.half == 2 ? rest : 0;
  }
  int n = x / a.Hkv, at = -1;  // the n-th of those tiles
  t.h = x - n * a.Hkv;
  for (int t0 = 0; t0 < all; t0 += 64) {
    unsigned long long mask = span_there(a, t0, tiles, len);
    if (padded) mask = tiles & ~mask;
    const int c = __popcll(mask);
    if (at < 0 && n < c) {
      const int lane = threadIdx.x & 63;
      at = t0 + __builtin_ctzll(__ballot((mask >> lane & 1ull) != 0ull && __popcll(mask & ((1ull << lane) - 1)) == n));
    }
    n -= c;
  }
  if (at < 0) t.h = -1;
  span_tile_at(a, max(at, 0), t.b, t.tile);
  t.parts = 1;
  if (t.half == 0 && a.m * a.G - t.tile * a.rows <= a.rows / 2) t.half = 1;
  const int r0 = t.tile * a.rows + (t.half == 2 ? a.rows / 2 : 0), last = min(r0 + (t.half != 0 ? a.rows / 2 : a.rows), a.m * a.G) - 1;
  if (r0 > last) t.h = -1;  // (the second half of what has no such rows)
  t.rows = span_rows(a, t.b, min(r0, last) >> lg, last >> lg);
  t.s1 = SpanSteps<64>(t.rows).total;
  for (int* x : {&t.b, &t.h, &t.tile, &t.half, &t.s1, &t.rows.lo, &t.rows.hi, &t.rows.nsink, &t.rows.len_min})
    *x = __builtin_amdgcn_readfirstlane(*x);  // (uniform, which the compiler does not see)
  return t;
}

// This block's run.  Without lengths, and for one or many tiles, a tile is cut into nsplit runs of `run` rows, as the longest length asks for (more rows
// than expected, of tokens that do not lie next to each other, make a tile's runs longer).  Else the blocks deal the runs, each for itself, since lengths
// are on the device only: all runs are of about one length, the least of a few with which they fit the blocks that are resident together, so that sequences
// of all lengths keep every CU as busy as equal ones would.  A tile's lane takes as many as its length asks for, and where they begin is the
// sum of the lanes before (figures at span_plan).
template <int KEYS, bool DEALT>
__device__ __forceinline__ SpanTile span_tile(const SpanArgs& a) {
  SpanTile t;
  const int i = blockIdx.x / a.Hkv, lg = 31 - __builtin_clz(a.G);
  t.h = blockIdx.x - i * a.Hkv;  // (a run's heads next to each other)
  t.slot = i;
  t.half = 0;
  bool known = false;
  int each = 0;
  if constexpr (!DEALT) {
    const int at = i / a.nsplit;
    t.parts = a.nsplit;
    t.part = i - at * a.nsplit;
    span_tile_at(a, at, t.b, t.tile);
    each = (a.run + KEYS - 1) / KEYS;
  } else {
    constexpr int kUnit = 4;  // steps of a run: a multiple of the waves that take them in turn, and at least 128 rows
    const int lane = threadIdx.x & 63, all = a.B * a.tiles;  // (up to 64)
    int b, tile, n = 0, most, least;
    span_tile_at(a, min(lane, all - 1), b, tile);
    const int r0 = tile * a.rows, j0 = r0 >> lg, j1 = (min(r0 + a.rows, a.m * a.G) - 1) >> lg;
    most = least = span_len(a, b, j0);
    known = a.rows <= 8 << lg;  // (else by the tile's first and last token and some between)
    if (a.m > 1) {
      least = least > 0 ? least : 0x7fffffff;
#pragma unroll
      for (int u = 1; u < 8; ++u) {
        const int len = span_len(a, b, u == 7 ? j1 : min(j0 + u, j1));
        most = max(most, len);
        least = min(least, len > 0 ? len : 0x7fffffff);
      }
      least = min(least, most);
    }
    if (lane < all) n = SpanSteps<KEYS>(span_rows_of(a, least, most)).total;
    const float longest = (float)wave_max_i32(n), total = wave_sum_f32((float)n);
    // a run's length, from the least that may do to one that does
    const float low = total * __builtin_amdgcn_rcpf((float)a.cap), high = fminf(total * __builtin_amdgcn_rcpf((float)(a.cap - all)), longest);
    uint32_t c[4], incl[2];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float run = fmaxf(ceilf(fmaf(high - low, (float)k / 3.f, low) * (1.0f / kUnit)) * kUnit, 128.f / KEYS);
      c[k] = lane < all ? (uint32_t)fmaxf(ceilf(fmaf((float)n, __builtin_amdgcn_rcpf(run), -1e-4f)), 1.f) : 0u;
    }
    incl[0] = wave_inclusive_scan_u32(c[0] | c[1] << 16);
    incl[1] = wave_inclusive_scan_u32(c[2] | c[3] << 16);
    uint32_t mine = lane < all ? 1u : 0u, sum = min(lane + 1, all);  // (a run each)
#pragma unroll
    for (int k = 3; k >= 0; --k) {
      const uint32_t x = incl[k / 2] >> (16 * (k % 2)) & 0xffffu;
      if (__builtin_amdgcn_readlane((int)x, 63) <= a.cap) {
        mine = c[k];
        sum = x;
      }
    }
    const int found = __popcll(__ballot((int)sum <= i)), at = min(found, all - 1);
    if (found >= all) t.h = -1;
    t.parts = __builtin_amdgcn_readlane((int)mine, at);
    t.part = i - __builtin_amdgcn_readlane((int)(sum - mine), at);
    t.b = __builtin_amdgcn_readlane(b, at);
    t.tile = __builtin_amdgcn_readlane(tile, at);
    t.rows = span_rows_of(a, __builtin_amdgcn_readlane(least, at), __builtin_amdgcn_readlane(most, at));
    if (t.h == 0 && t.part == 0 && threadIdx.x == 0) a.dealt[at] = make_int2(i, t.parts);
  }
  if (!known) {
    const int r0 = t.tile * a.rows, last = min(r0 + a.rows, a.m * a.G) - 1;
    t.rows = span_rows(a, t.b, r0 >> lg, last >> lg);
  }
  const SpanSteps<KEYS> n(t.rows);
  each = max(each, (n.total + t.parts - 1) / t.parts);
  t.s0 = min(n.total, t.part * each);
  t.s1 = min(n.total, t.s0 + each);
  for (int* x : {&t.b, &t.h, &t.tile, &t.part, &t.parts, &t.slot, &t.s0, &t.s1, &t.rows.lo, &t.rows.hi, &t.rows.nsink, &t.rows.len_min})
    *x = __builtin_amdgcn_readfirstlane(*x);  // (uniform, which the compiler does not see)
  return t;
}

// A run that no row is left for: its parts say so, which the merge goes by.
template <bool DEALT>
__device__ __forceinline__ void span_none(const SpanArgs& a, const SpanTile& t, int live) {
  for (int r = threadIdx.x; r < live; r += blockDim.x) *reinterpret_cast<float2*>(span_part<DEALT>(a, t, r) + kD) = make_float2(kNegBig, 0.f);
}

// A wave's state after its steps, for 16 query rows: lane (row r16, kgrp) holds maximum m and sum l of its row (l its own share of the
// rows), columns col(c, i) of the row's output in o[c][i].
template <int ROWS, int WAVES>
struct SpanMerge {
  float2 ml[WAVES][ROWS];
  float o[WAVES][ROWS][kD];
};

// The waves' results joined: `live` query rows of the tile, out or as parts.  Begins with a barrier.
template <typename T, bool DEALT, int ROWS, int WAVES>
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
    if (tile.parts > 1) {
      float* p = span_part<DEALT>(a, tile, r);
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
