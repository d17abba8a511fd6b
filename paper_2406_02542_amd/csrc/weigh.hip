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
// Rows of a part of a sequence of `len`: whole steps of 32, so that a step's logits are stored 16 bytes at a time.
__device__ __forceinline__ int part_run(int len, int nsplit) {
  nsplit = max(nsplit, 1);
  return max(32, ((len + nsplit - 1) / nsplit + 31) & ~31);
}

// The logits of the unit's heads, [head][pitch].
template <int NH>
struct StoreLogits {
  static constexpr bool kAny = true;
  float* p;  // of the unit's first head
  size_t pitch;
  bool writer;  // vector units: one lane of a row's group
  __device__ __forceinline__ void operator()(int g, int row, bool ok, float x) const {
    if (writer && ok) p[g * pitch + row] = x;
  }
  // (a step's rows past the last lie inside the pitch, which is a multiple of 32)
  __device__ __forceinline__ void operator()(int g, int row, const float4& x) const {
    if (g < NH) *reinterpret_cast<float4*>(p + g * pitch + row) = x;
  }
};

template <typename T, int NH, bool MFMA, bool LOGITS, bool STREAM>
__global__ __launch_bounds__(kPtThreads) void parts_kernel(const void* __restrict__ k, const void* __restrict__ v,
                                                           const void* __restrict__ qv, float* __restrict__ partial,
                                                           float* __restrict__ logits, size_t pitch, int Hkv, int S_cap, int S_max,
                                                           int nsplit, int nparts, Ragged rg) {
  using ST = typename T::store_t;
  __shared__ __align__(16) MergeSmem<kPtWaves, NH> s_merge;
  const int unit = blockIdx.y, split = blockIdx.x, tid = threadIdx.x;
  const int len = part_rows_held(rg, unit / Hkv, S_max), run = part_run(len, nsplit);
  const int r0 = split * run, r1 = min(len, r0 + run);
  if (r0 >= r1) return;  // uniform for the block; the merge knows how many parts there are
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
    if constexpr (LOGITS)
      am_attend_rows<false, 4, 1, STREAM>(ad, bq, nullptr, r0, AmRoundRobin<kPtWaves>(r0, r1), st, [] {}, StoreLogits<NH>{lg, pitch, true});
    else
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
                                                                             StoreLogits<NH>{lg, pitch, c == 0});
    else
      attend_rows<T, NH, kPtWaves * RPW, false, false, false, false, STREAM>(acc, qr, ra, nullptr, nullptr, gid, r0, r1);
    attend_publish<T, NH, kPtWaves>(acc, s_merge);
  }
  for (int i = tid; i < NH * kD; i += kPtThreads) {
    const int g = i / kD, col = i % kD;
    float mn, ls, os;
    attend_merged<kPtWaves, NH>(s_merge, g, col, mn, ls, os);
    float* pr = partial + ((head0 + g) * nparts + split) * kPartStride;
    pr[col] = os;
    if (col == 0) {
      pr[kD] = mn;
      pr[kD + 1] = ls;
    }
  }
}

// Parts of one head: its sequence's `live` ones, then `shared` that every head has behind the nsplit places.
struct PartList {
  const float* p;
  int live, nsplit, n;
  __device__ __forceinline__ const float* at(int i) const { return p + (size_t)(i < live ? i : nsplit + i - live) * kPartStride; }
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
__global__ __launch_bounds__(kMgThreads) void weigh_merge_kernel(const float* __restrict__ partial, const float* __restrict__ logits,
                                                                 size_t pitch, const float* weights_in, float* weights_out,
                                                                 typename T::store_t* __restrict__ out, int Hkv, int S_cap, int S_max,
                                                                 int nsplit, int shared, int row_blocks, Ragged rg) {
  __shared__ float s_max[NH], s_inv[NH];
  const int unit = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int len = part_rows_held(rg, unit / Hkv, S_max), run = part_run(len, nsplit);
  const int live = (len + run - 1) / run, nparts = nsplit + shared;
  const size_t head0 = (size_t)unit * NH;
  if ((int)blockIdx.x >= row_blocks) {
    const size_t head = head0 + blockIdx.x - row_blocks;
    merge_head<T>(PartList{partial + head * nparts * kPartStride, live, nsplit, live + shared}, out + head * kD);
    return;
  }
  const int r0 = (int)blockIdx.x * kMgRows;
  if (r0 >= len) return;  // uniform for the block
  // wave w joins the maxima and sums of heads w, w + 4, .. : a lane for every 64th part
  for (int g = wave; g < NH; g += kMgThreads / 64) {
    const PartList pl{partial + (head0 + g) * nparts * kPartStride, live, nsplit, live + shared};
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

// Parts of a sequence: about four blocks per CU, of at least 64 rows.
int weigh_splits(const Shape& s) {
  const int units = s.B * s.Hkv;
  int n = (4 * device_cus() + units - 1) / units;
  const int most = (s.S + 63) / 64;
  if (n > most) n = most;
  return n < 1 ? 1 : n;
}

size_t weigh_logits_pitch(int S_max) { return ((size_t)S_max + 31) / 32 * 32; }

template <typename T, int NH, bool MFMA>
static hipError_t launch_parts_nh(const Shape& s, int nsplit, int nparts, const void* q, const void* k, const void* v,
                                  float* partial, float* logits, hipStream_t st) {
  const dim3 grid(nsplit, s.B * s.Hkv), block(kPtThreads);
  const size_t pitch = weigh_logits_pitch(s.S);
  if (logits != nullptr)
    hipLaunchKernelGGL((parts_kernel<T, NH, MFMA, true, false>), grid, block, 0, st, k, v, q, partial, logits, pitch, s.Hkv,
                       s.S_cap, s.S, nsplit, nparts, s.rg);
  else
    hipLaunchKernelGGL((parts_kernel<T, NH, MFMA, false, false>), grid, block, 0, st, k, v, q, partial, logits, pitch, s.Hkv,
                       s.S_cap, s.S, nsplit, nparts, s.rg);
  return hipGetLastError();
}

hipError_t launch_parts(const Shape& s, int nsplit, int nparts, const void* q, const void* k, const void* v, float* partial,
                        float* logits, hipStream_t st) {
#define LOKI_PARTS(T, NH, M) return launch_parts_nh<T, NH, M>(s, nsplit, nparts, q, k, v, partial, logits, st)
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
static hipError_t launch_merge_t(const Shape& s, int nsplit, int shared, const float* partial, const float* logits,
                                 const float* weights_in, float* weights_out, void* out, hipStream_t st) {
  const int row_blocks = weights_out != nullptr ? (s.S + kMgRows - 1) / kMgRows : 0;
  const dim3 grid(row_blocks + s.G, s.B * s.Hkv), block(kMgThreads);
  auto* o = static_cast<typename T::store_t*>(out);
#define LOKI_MERGE(NH)                                                                                                     \
  hipLaunchKernelGGL((weigh_merge_kernel<T, NH>), grid, block, 0, st, partial, logits, weigh_logits_pitch(s.S), weights_in, \
                     weights_out, o, s.Hkv, s.S_cap, s.S, nsplit, shared, row_blocks, s.rg);                               \
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

hipError_t launch_weigh_merge(const Shape& s, int nsplit, int shared, const float* partial, const float* logits,
                              const float* weights_in, float* weights_out, void* out, hipStream_t st) {
  return s.dtype == 0 ? launch_merge_t<F32>(s, nsplit, shared, partial, logits, weights_in, weights_out, out, st)
                      : launch_merge_t<BF16>(s, nsplit, shared, partial, logits, weights_in, weights_out, out, st);
}

}  // namespace loki
