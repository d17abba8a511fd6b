// Dense attention over a cache (Section 2, Eq. 1 of arXiv 2406.02542) that also adds every row's softmax weight to
// the row's running total, which is what an eviction by accumulated weight goes by (evict.hip).
//
// A weight is 2^(logit - M) / L with the maximum and the sum of the whole sequence, so it can be formed only when
// all rows have been seen.  Two launches: (1) parts_kernel: runs of rows, the keys and values read once; each
// run leaves (max, sum, output) per head and, for the weights, its rows' logits: 4 bytes per row and head beside the
// 512 (bf16) of the row.  (2) weigh_merge_kernel: every block joins the runs' maxima and sums, then takes its
// share of the rows' totals or of the outputs.  Memory bounds both.
#include "attend_mfma_impl.h"

namespace loki {

constexpr int kPtThreads = 256;
constexpr int kPtWaves = kPtThreads / 64;
constexpr int kMgThreads = 256;
constexpr int kMgRows = 1024;  // rows of a merge block

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
// On the matrix cores a wave keeps those of some steps in LDS and stores them together, whole lines: memory
// operations are waited for in their order, so a store of every step is waited for with the next rows (16 sequences of 32/8
// heads up to 16384 rows: the launch 142 us with a store in every step, NNN so, 115 without the weights).
template <int NH>
constexpr int kept_steps() {
  return 64 / NH;
}
template <int NH>
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
      *reinterpret_cast<float4*>(p + g * pitch + base + s * (kPtWaves * kAmRows) + i % 8 * 4) = x;
    }
    __builtin_amdgcn_wave_barrier();
    n = 0;
  }
};

template <typename T, int NH, bool MFMA, bool LOGITS, bool STREAM>
__device__ __forceinline__ void parts_body(MergeSmem<kPtWaves, NH>& s_merge, float* kept, const RunAt& at, int run, const void* __restrict__ k,
                                           const void* __restrict__ v, const void* __restrict__ qv, float* __restrict__ partial,
                                           float* __restrict__ logits, size_t pitch, int Hkv, int S_cap) {
  using ST = typename T::store_t;
  const int tid = threadIdx.x, h = blockIdx.y, unit = at.b * Hkv + h;
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
      KeepLogits<NH> keep{lg, pitch, kept + (tid >> 6) * (kept_steps<NH>() * NH * kAmRows)};
      am_attend_rows<false, 4, 1, STREAM>(ad, bq, nullptr, r0, AmRoundRobin<kPtWaves>(r0, r1), st, [] {}, keep);
      keep.flush();
    } else
      am_attend_rows<false, 4, 1, STREAM>(ad, bq, nullptr, r0, AmRoundRobin<kPtWaves>(r0, r1), st, [] {});
    am_publish<NH, kPtWaves>(st, s_merge);
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
      attend_rows<T, NH, kPtWaves * RPW, false, false, false, false, STREAM>(acc, qr, ra, nullptr, nullptr, gid, r0, r1,
                                                                             StoreLogits{lg, pitch, c == 0});
    else
      attend_rows<T, NH, kPtWaves * RPW, false, false, false, false, STREAM>(acc, qr, ra, nullptr, nullptr, gid, r0, r1);
    attend_publish<T, NH, kPtWaves>(acc, s_merge);
  }
  // part blockIdx.x of query head h NH + g, of gridDim.x
  for (int i = tid; i < NH * kD; i += kPtThreads) {
    const int g = i / kD, col = i % kD;
    float mn, ls, os;
    attend_merged<kPtWaves, NH>(s_merge, g, col, mn, ls, os);
    float* pr = partial + ((size_t)(h * NH + g) * gridDim.x + blockIdx.x) * kPartStride;
    pr[col] = os;
    if (col == 0) {
      pr[kD] = mn;
      pr[kD + 1] = ls;
    }
  }
}

template <typename T, int NH, bool MFMA, bool LOGITS>
__global__ __launch_bounds__(kPtThreads) void parts_kernel(const void* __restrict__ k, const void* __restrict__ v,
                                                           const void* __restrict__ qv, float* __restrict__ partial,
                                                           float* __restrict__ logits, size_t pitch, int B, int Hkv, int S_cap,
                                                           int S_max, int nsplit, Ragged rg) {
  __shared__ __align__(16) MergeSmem<kPtWaves, NH> s_merge;
  __shared__ __align__(16) float s_kept[MFMA && LOGITS ? kPtWaves * kept_steps<NH>() * NH * kAmRows : 1];
  const Dealt d = deal_runs(rg, B, S_max, nsplit);
  const RunAt at = find_run(rg, B, S_max, d.run, blockIdx.x);
  if (at.b >= B) return;  // uniform for the block; the merge knows how many runs there are
  const int form_now = rg.loads.form == kByLengths ? form_of(rg.loads, {d.total, 0.f}) : rg.loads.form;
  with_form<kPastCaches>(form_now, [&](auto form) __attribute__((always_inline)) {
    parts_body<T, NH, MFMA, LOGITS, decltype(form)::value != kThroughCaches>(s_merge, s_kept, at, d.run, k, v, qv, partial, logits, pitch, Hkv, S_cap);
  });
}

// Parts of one head: the `live` runs of its sequence, and the prefix's that it has behind them.
struct PartList {
  const float *own, *prefix;
  int live, n;
  __device__ __forceinline__ const float* at(int i) const { return i < live ? own + (size_t)i * kPartStride : prefix + (size_t)(i - live) * kPartStride; }
};

// The outputs: a block joins the parts of one head.  32 lanes take a part's row, 16 bytes each, so a block's 8 lane
// groups go through the parts eight at a time with a running maximum of their own, and meet in LDS.
template <typename T>
__device__ __forceinline__ void merge_head(const PartList& pl, typename T::store_t* out) {
  constexpr int kGroups = kMgThreads / 32, U = 4;
  __shared__ __align__(16) float s_o[kGroups][kD];
  __shared__ float2 s_ml[kGroups];
  const int tid = threadIdx.x, lane = tid & 31, grp = tid >> 5;
  float m = kNegBig, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i0 = grp; i0 < pl.n; i0 += kGroups * U) {
    float2 ml[U];
    float4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool ok = i0 + u * kGroups < pl.n;
      const float* p = pl.at(ok ? i0 + u * kGroups : i0);
      ml[u] = *reinterpret_cast<const float2*>(p + kD);
      x[u] = *reinterpret_cast<const float4*>(p + 4 * lane);
      if (!ok) ml[u] = make_float2(kNegBig, 0.f);
    }
    float mn = m;
#pragma unroll
    for (int u = 0; u < U; ++u) mn = fmaxf(mn, ml[u].x);
    const float c = fast_exp2(m - mn);
    l *= c;
    o = make_float4(o.x * c, o.y * c, o.z * c, o.w * c);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float f = i0 + u * kGroups < pl.n ? fast_exp2(ml[u].x - mn) : 0.f;
      l = fmaf(ml[u].y, f, l);
      o = make_float4(fmaf(x[u].x, f, o.x), fmaf(x[u].y, f, o.y), fmaf(x[u].z, f, o.z), fmaf(x[u].w, f, o.w));
    }
    m = mn;
  }
  *reinterpret_cast<float4*>(&s_o[grp][4 * lane]) = o;
  if (lane == 0) s_ml[grp] = make_float2(m, l);
  __syncthreads();
  if (tid < kD) {
    float mn = kNegBig, ls = 0.f, os = 0.f;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) mn = fmaxf(mn, s_ml[g].x);
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const float f = fast_exp2(s_ml[g].x - mn);
      ls = fmaf(s_ml[g].y, f, ls);
      os = fmaf(s_o[g][tid], f, os);
    }
    T::store1(out + tid, ls > 0.f ? os / ls : 0.f);  // (no row at all: zeros)
  }
}

// blockIdx.x < row_blocks: totals of kMgRows rows; behind them one head's output each.
template <typename T, int NH>
__global__ __launch_bounds__(kMgThreads) void weigh_merge_kernel(const float* __restrict__ partial, const float* __restrict__ prefix,
                                                                 const float* __restrict__ logits, size_t pitch,
                                                                 const float* weights_in, float* weights_out,
                                                                 typename T::store_t* __restrict__ out, int B, int Hkv, int S_cap,
                                                                 int S_max, int nsplit, int shared, int row_blocks, Ragged rg) {
  __shared__ float s_max[NH], s_inv[NH];
  const int unit = blockIdx.y, b = unit / Hkv, h = unit - b * Hkv, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int run = deal_runs(rg, B, S_max, nsplit).run, len = part_rows_held(rg, b, S_max);
  const size_t head0 = (size_t)unit * NH, X = (size_t)nsplit * B;
  const float* own = partial + ((size_t)h * NH * X + first_run(rg, S_max, run, b)) * kPartStride;
  const int live = (len + run - 1) / run;
  auto parts = [&](int g) { return PartList{own + g * X * kPartStride, prefix + (head0 + g) * shared * kPartStride, live, live + shared}; };
  if ((int)blockIdx.x >= row_blocks) {
    const int g = (int)blockIdx.x - row_blocks;
    merge_head<T>(parts(g), out + (head0 + g) * kD);
    return;
  }
  const int r0 = (int)blockIdx.x * kMgRows;
  if (r0 >= len) return;  // uniform for the block
  // wave w joins the maxima and sums of heads w, w + 4, .. : a lane for every 64th part
  for (int g = wave; g < NH; g += kMgThreads / 64) {
    const PartList pl = parts(g);
    float m = kNegBig, l = 0.f;
    for (int i = lane; i < pl.n; i += 64) {
      const float2 ml = *reinterpret_cast<const float2*>(pl.at(i) + kD);
      const float mn = fmaxf(m, ml.x);
      l = l * fast_exp2(m - mn) + ml.y * fast_exp2(ml.x - mn);
      m = mn;
    }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const float m2 = __shfl_xor(m, off), l2 = __shfl_xor(l, off), mn = fmaxf(m, m2);
      l = l * fast_exp2(m - mn) + l2 * fast_exp2(m2 - mn);
      m = mn;
    }
    if (lane == 0) {
      s_max[g] = m;
      s_inv[g] = 1.0f / l;
    }
  }
  __syncthreads();
  const float* lg = logits + head0 * pitch;
  const size_t w0 = (size_t)unit * S_cap;
#pragma unroll
  for (int u = 0; u < kMgRows / kMgThreads; ++u) {
    const int r = r0 + u * kMgThreads + tid;
    if (r < len) {
      float w = weights_in != nullptr ? weights_in[w0 + r] : 0.f;
#pragma unroll
      for (int g = 0; g < NH; ++g) w = fmaf(fast_exp2(lg[g * pitch + r] - s_max[g]), s_inv[g], w);
      weights_out[w0 + r] = w;
    }
  }
}

// Runs of a sequence: about four blocks per CU in bf16, eight in fp32, of at least 64 rows.  us with 2, 4, 6, 8 and 12
// per CU: 16 sequences of 32/8 bf16 heads up to 16384 rows 162, 144, 147, 145, 148; 5 of 24 fp32 heads up to 2311 rows
// 43.5, 41.2, 38.4, 38.3, 38.8.
int weigh_splits(const Shape& s) {
  const int units = s.B * s.Hkv;
  int n = ((s.dtype == 1 ? 4 : 8) * device_cus() + units - 1) / units;
  const int most = (s.S + 63) / 64;
  if (n > most) n = most;
  return n < 1 ? 1 : n;
}

size_t weigh_logits_pitch(int S_max) { return ((size_t)S_max + 31) / 32 * 32; }

template <typename T, int NH, bool MFMA>
static hipError_t launch_parts_nh(const Shape& s, int nsplit, const void* q, const void* k, const void* v, float* partial,
                                  float* logits, hipStream_t st) {
  const dim3 grid(nsplit * s.B, s.Hkv), block(kPtThreads);
  const size_t pitch = weigh_logits_pitch(s.S);
  const Ragged rg = with_loads(s, kEveryRow);
  if (logits != nullptr)
    hipLaunchKernelGGL((parts_kernel<T, NH, MFMA, true>), grid, block, 0, st, k, v, q, partial, logits, pitch, s.B, s.Hkv, s.S_cap,
                       s.S, nsplit, rg);
  else
    hipLaunchKernelGGL((parts_kernel<T, NH, MFMA, false>), grid, block, 0, st, k, v, q, partial, logits, pitch, s.B, s.Hkv, s.S_cap,
                       s.S, nsplit, rg);
  return hipGetLastError();
}

hipError_t launch_parts(const Shape& s, int nsplit, const void* q, const void* k, const void* v, float* partial, float* logits,
                        hipStream_t st) {
#define LOKI_PARTS(T, NH, M) return launch_parts_nh<T, NH, M>(s, nsplit, q, k, v, partial, logits, st)
  if (s.dtype == 1) {
    switch (s.G) {
      case 1: LOKI_PARTS(BF16, 1, false);
      case 2: LOKI_PARTS(BF16, 2, false);
      case 4: LOKI_PARTS(BF16, 4, true);
      case 8: LOKI_PARTS(BF16, 8, true);
      default: return hipErrorInvalidValue;
    }
  }
  switch (s.G) {
    case 1: LOKI_PARTS(F32, 1, false);
    case 2: LOKI_PARTS(F32, 2, false);
    case 4: LOKI_PARTS(F32, 4, false);
    case 8: LOKI_PARTS(F32, 8, false);
    default: return hipErrorInvalidValue;
  }
#undef LOKI_PARTS
}

template <typename T>
static hipError_t launch_merge_t(const Shape& s, int nsplit, int shared, const float* partial, const float* prefix, const float* logits,
                                 const float* weights_in, float* weights_out, void* out, hipStream_t st) {
  const int row_blocks = weights_out != nullptr ? (s.S + kMgRows - 1) / kMgRows : 0;
  const dim3 grid(row_blocks + s.G, s.B * s.Hkv), block(kMgThreads);
  auto* o = static_cast<typename T::store_t*>(out);
#define LOKI_MERGE(NH)                                                                                                     \
  hipLaunchKernelGGL((weigh_merge_kernel<T, NH>), grid, block, 0, st, partial, prefix, logits, weigh_logits_pitch(s.S),    \
                     weights_in, weights_out, o, s.B, s.Hkv, s.S_cap, s.S, nsplit, shared, row_blocks, s.rg);               \
  break
  switch (s.G) {
    case 1: LOKI_MERGE(1);
    case 2: LOKI_MERGE(2);
    case 4: LOKI_MERGE(4);
    case 8: LOKI_MERGE(8);
    default: return hipErrorInvalidValue;
  }
#undef LOKI_MERGE
  return hipGetLastError();
}

hipError_t launch_weigh_merge(const Shape& s, int nsplit, int shared, const float* partial, const float* prefix,
                              const float* logits, const float* weights_in, float* weights_out, void* out, hipStream_t st) {
  return s.dtype == 0 ? launch_merge_t<F32>(s, nsplit, shared, partial, prefix, logits, weights_in, weights_out, out, st)
                      : launch_merge_t<BF16>(s, nsplit, shared, partial, prefix, logits, weights_in, weights_out, out, st);
}

}  // namespace loki
