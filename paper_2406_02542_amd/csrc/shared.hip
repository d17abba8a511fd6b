// Attention of a whole batch over the prefix that its sequences share (Section 2, Eq. 1 of arXiv 2406.02542, the
// part of the rows that is the same for all): the prefix's keys and values are held once, and the B G query rows
// of a KV head meet each of them in one product.  A run of the prefix leaves (max, sum, output) per query row, which
// weigh_merge_kernel joins with the parts of the sequence's own rows.
#include "attend_mfma_impl.h"

namespace loki {

constexpr int kPfThreads = 256;
constexpr int kPfWaves = kPfThreads / 64;

// Row of q (and of the partial results) that query row r of KV head h is: r = b G + g.
__device__ __forceinline__ size_t prefix_head(int r, int h, int G, int Hq) {
  const int b = r / G;
  return (size_t)b * Hq + h * G + (r - b * G);
}

template <typename T, int NQ>
__global__ __launch_bounds__(kPfThreads) void prefix_kernel(const void* __restrict__ k, const void* __restrict__ v,
                                                            const void* __restrict__ qv, float* __restrict__ partial, int M, int G,
                                                            int Hq, int rows, int cap, int run, int first, int nparts) {
  using ST = typename T::store_t;
  __shared__ __align__(16) MergeSmem<kPfWaves, NQ> s_merge;
  const int split = blockIdx.x, q0 = blockIdx.y * NQ, h = blockIdx.z, tid = threadIdx.x;
  const int r0 = split * run, r1 = min(rows, r0 + run);
  const ST* q = static_cast<const ST*>(qv);
  if constexpr (T::EPC == 8) {
    const int lane = tid & 63, r16 = lane & 15, kgrp = lane >> 4;
    const bool there = q0 + r16 < M;
    am_bf16x8_t bq[4][1];
#pragma unroll
    for (int step = 0; step < 4; ++step) {
      uint4 raw = load16(q + prefix_head(there ? q0 + r16 : 0, h, G, Hq) * kD + 32 * step + 8 * kgrp);
      if (!there) raw = make_uint4(0, 0, 0, 0);
      bq[step][0] = __builtin_bit_cast(am_bf16x8_t, raw);
    }
    const AmAddr<4> ad = am_make_addr<4, false>(k, nullptr, v, (size_t)h, cap, kD);
    AmState st;
    st.init();
    am_attend_rows<false, 4, 1, false>(ad, bq, nullptr, r0, AmRoundRobin<kPfWaves>(r0, r1), st, [] {});
    am_publish<NQ, kPfWaves>(st, s_merge);
  } else {
    constexpr int EPC = T::EPC, LPRV = kD / EPC, RPW = 64 / LPRV;
    const int lane = tid & 63, wave = tid >> 6, c = lane % LPRV;
    float qr[NQ][EPC];
#pragma unroll
    for (int g = 0; g < NQ; ++g) T::unpack(load16(q + prefix_head(min(q0 + g, M - 1), h, G, Hq) * kD + c * EPC), qr[g]);
    const RowAddr ra = make_row_addr<T, false>(k, nullptr, v, (size_t)h, cap, kD, c);
    AttendAcc<T, NQ> acc;
    acc.init();
    attend_rows<T, NQ, kPfWaves * RPW, false, false>(acc, qr, ra, nullptr, nullptr, wave * RPW + lane / LPRV, r0, r1);
    attend_publish<T, NQ, kPfWaves>(acc, s_merge);
  }
  for (int i = tid; i < NQ * kD; i += kPfThreads) {
    const int g = i / kD, col = i % kD;
    if (q0 + g >= M) continue;
    float mn, ls, os;
    attend_merged<kPfWaves, NQ>(s_merge, g, col, mn, ls, os);
    float* pr = partial + (prefix_head(q0 + g, h, G, Hq) * nparts + first + split) * kPartStride;
    pr[col] = os;
    if (col == 0) {
      pr[kD] = mn;
      pr[kD + 1] = ls;
    }
  }
}

static int prefix_run(const Shape& s, int rows) {
  const int tiles = s.Hkv * ((s.B * s.G + 15) / 16);
  int n = (4 * device_cus() + tiles - 1) / tiles;
  const int run = (rows + n - 1) / n;
  return (run + 127) / 128 * 128;
}

int prefix_splits(const Shape& s, int prefix_rows) {
  if (prefix_rows < 1) return 0;
  const int run = prefix_run(s, prefix_rows);
  return (prefix_rows + run - 1) / run;
}

hipError_t launch_prefix(const Shape& s, int first, int splits, int nparts, const void* q, const void* k, const void* v, int rows,
                         int cap, float* partial, hipStream_t st) {
  const int M = s.B * s.G, run = prefix_run(s, rows);
  if (s.dtype == 0)
    hipLaunchKernelGGL((prefix_kernel<F32, 8>), dim3(splits, (M + 7) / 8, s.Hkv), dim3(kPfThreads), 0, st, k, v, q, partial, M, s.G,
                       s.Hq, rows, cap, run, first, nparts);
  else
    hipLaunchKernelGGL((prefix_kernel<BF16, 16>), dim3(splits, (M + 15) / 16, s.Hkv), dim3(kPfThreads), 0, st, k, v, q, partial, M,
                       s.G, s.Hq, rows, cap, run, first, nparts);
  return hipGetLastError();
}

}  // namespace loki
