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
// The sequence and the run of it that run x of a KV head is; b = B: none.
struct RunAt {
  int b, i, len;
};
__device__ __forceinline__ RunAt find_run(const Ragged& rg, int B, int S_max, int run, int x) {
  if (rg.seq_lens == nullptr) {
    const int each = (S_max + run - 1) / run, b = x / each;
    return {min(b, B), x - b * each, S_max};
  }
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < B; b0 += 64) {
    const int len = b0 + lane < B ? part_rows_held(rg, b0 + lane, S_max) : 0, runs = (len + run - 1) / run;
    const int incl = (int)wave_inclusive_scan_u32((uint32_t)runs);
    const unsigned long long behind = __ballot(incl > x);
    if (behind != 0ull) {
      const int at = __ffsll((long long)behind) - 1;
      const int before = __builtin_amdgcn_readlane(incl, at) - __builtin_amdgcn_readlane(runs, at);
      return {b0 + at, x - before, __builtin_amdgcn_readlane(len, at)};
    }
    x -= __builtin_amdgcn_readlane(incl, 63);
  }
  return {B, 0, 0};
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

template <typename T, int NH>
constexpr bool parts_mfma() {  // four heads and more on a bf16 cache: matrix cores (as attend_mfma_applies)
  return T::EPC == 8 && NH >= 4;
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
// On the matrix cores a wave keeps those of some steps in LDS and stores them together, whole lines: memory operations are
// waited for in their order, so a store of every step is waited for with the next rows.  16 sequences of 32/8 heads up to
// 16384 rows: the launch 142 us with a store in every step, 136, 130 and 131 for runs of 4, 16 and 32 steps; 118 with the stores left out.
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

// One run by a block of WAVES waves: part `x` of the X that each query head of KV head h has.
template <typename T, int NH, bool LOGITS, bool STREAM, int WAVES>
__device__ __forceinline__ void parts_body(MergeSmem<WAVES, NH>& s_merge, float* kept, const RunAt& at, int run, int h, int x, int X,
                                           const void* __restrict__ k, const void* __restrict__ v, const void* __restrict__ qv,
                                           float* __restrict__ partial, float* __restrict__ logits, size_t pitch, int Hkv, int S_cap) {
  using ST = typename T::store_t;
  constexpr bool MFMA = parts_mfma<T, NH>();
  const int tid = threadIdx.x, unit = at.b * Hkv + h;
  const int r0 = at.i * run, r1 = min(at.len, r0 + run);
  const size_t head0 = (size_t)unit * NH;
  const ST* q = static_cast<const ST*>(qv) + head0 * kD;
  float* lg = logits + head0 * pitch;
  if constexpr (MFMA) {
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
    for (int i = tid; i < NH * kD; i += (64 * WAVES)) {
    const int g = i / kD, col = i % kD;
    float mn, ls, os;
    attend_merged<WAVES, NH>(s_merge, g, col, mn, ls, os);
    float* pr = partial + ((size_t)(h * NH + g) * X + x) * kPartStride;
    pr[col] = os;
    if (col == 0) {
      pr[kD] = mn;
      pr[kD + 1] = ls;
    }
  }
}

}  // namespace loki
