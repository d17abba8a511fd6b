// Dense attention over a cache (Section 2, Eq. 1 of arXiv 2406.02542) that also adds every row's softmax weight to
// the row's running total, which is what an eviction by accumulated weight goes by (evict.hip).
//
// A weight is 2^(logit - M) / L with the maximum and the sum of the whole sequence, so it can be formed only when
// all rows have been seen.  Two launches: (1) parts_kernel: runs of rows, the keys and values read once; each
// run leaves (max, sum, output) per head and, for the weights, its rows' logits: 4 bytes per row and head beside the
// 512 (bf16) of the row.  (2) weigh_merge_kernel: every block joins the runs' maxima and sums, then takes its
// share of the rows' totals or of the outputs.  Memory bounds both.
#include "parts_impl.h"

namespace loki {

constexpr int kPtThreads = 256;
constexpr int kPtWaves = kPtThreads / 64;
constexpr int kMgThreads = 256;
constexpr int kMgRows = 1024;  // rows of a merge block

template <typename T, int NH, bool LOGITS>
__global__ __launch_bounds__(kPtThreads) void parts_kernel(const void* __restrict__ k, const void* __restrict__ v,
                                                           const void* __restrict__ qv, float* __restrict__ partial,
                                                           float* __restrict__ logits, size_t pitch, int B, int Hkv, int S_cap,
                                                           int S_max, int nsplit, Ragged rg) {
  __shared__ __align__(16) PartsSmem<T, NH, kPtWaves> s_merge;
  __shared__ __align__(16) float s_kept[LOGITS && T::EPC == 8 && parts_mfma<NH>() ? kPtWaves * kept_steps<NH>() * NH * kAmRows : 1];
  const Dealt d = deal_runs(rg, B, S_max, nsplit);
  const int x = blockIdx.x / Hkv, h = blockIdx.x - x * Hkv;  // (a run's heads next to each other: whole runs of all heads first)
  const RunAt at = find_run(rg, B, S_max, d.run, x);
  if (at.b >= B) return;  // uniform for the block; the merge knows how many runs there are
  const int form_now = rg.loads.form == kByLengths ? form_of(rg.loads, {d.total, 0.f}) : rg.loads.form;
  with_form<kPastCaches>(form_now, [&](auto form) __attribute__((always_inline)) {
    parts_body<T, NH, LOGITS, decltype(form)::value != kThroughCaches, kPtWaves>(s_merge, s_kept, at, d.run, h, nsplit * B,
                                                                               k, v, qv, partial, logits, pitch, Hkv, S_cap);
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
  // the rows' logits and totals are asked for before the runs' maxima and sums are joined
  const float* lg = logits + head0 * pitch;
  const size_t w0 = (size_t)unit * S_cap;
  constexpr int U = kMgRows / kMgThreads;
  float x[U][NH], w[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int r = min(r0 + u * kMgThreads + tid, len - 1);
    w[u] = weights_in != nullptr ? weights_in[w0 + r] : 0.f;
#pragma unroll
    for (int g = 0; g < NH; ++g) x[u][g] = lg[g * pitch + r];
  }
  // wave w joins heads w, w + 4, .. : a lane for every 64th part
  for (int g = wave; g < NH; g += kMgThreads / 64) {
    const PartList pl = parts(g);
    float m = kNegBig, l = 0.f;
    for (int i = lane; i < pl.n; i += 64) {
      const float2 ml = *reinterpret_cast<const float2*>(pl.at(i) + kD);
      const float mn = fmaxf(m, ml.x);
      l = l * fast_exp2(m - mn) + ml.y * fast_exp2(ml.x - mn);
      m = mn;
    }
    const float top = wave_max_f32(m);
    l = wave_sum_f32(l * fast_exp2(m - top));
    if (lane == 0) {
      s_max[g] = top;
      s_inv[g] = 1.0f / l;
    }
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int r = r0 + u * kMgThreads + tid;
#pragma unroll
    for (int g = 0; g < NH; ++g) w[u] = fmaf(fast_exp2(x[u][g] - s_max[g]), s_inv[g], w[u]);
    if (r < len) weights_out[w0 + r] = w[u];
  }
}

// Runs of a sequence, at most as many as leave each of a block's four waves a step of 32 rows (bf16 on the matrix cores) or 16 rows.
// Matrix cores: two blocks per CU, as many as are resident, where a sequence then has six runs and more, else four, which even
// out lengths better.  us with 2, 4, 8 per CU, bf16: one of 32/8 heads, 20000 rows 20.9, 25.0, 26.7, 10 of 32/4 up to 9000 28.9, 32.0, 40.1,
// 20 of 32/4 up to 5000 31.5, 34.5, 42.4, 16 of 32/8 up to 16384 149, 141, 142, 24 up to 7000 94.0, 90.7, 93.6, 50 up to 2500 80.5, 74.0, 75.9
// (but 64 of 64/8, all of 600 40.5, 44.5, 53.2); fp32: 13 of 32/8 up to 3000 48.7, 48.0, 50.5.
// Vector units: eight per CU in fp32 (5 sequences of 24 fp32 heads up to 2311 rows with 2, 4, 6, 8 and 12 per CU 43.5, 41.2, 38.4,
// 38.3, 38.8), four in bf16, where no count is best for all.  With 2, 3 and 4: 40 of 16 heads up to 2000 rows 81.4, 74.0, 74.1, 7 of 24 up to
// 3000 42.2, 38.4, 37.8; 16 of 32 with 4096 178, 182, 182, up to 4096 131, 134, 134; 4 of 32/16 with 4096 27.8, 30.0, 28.2, 9 up to 5000
// 56.4, 61.4, 59.3; 4 of 32 up to 4096 42.5, 45.5, 48.2; one of 32 with 8192 27.4, 27.5, 31.0, of 24 22.2, 22.2, 22.2.
int weigh_splits(const Shape& s) {
  const int units = s.B * s.Hkv, slots = 2 * device_cus();
  const bool mfma = s.G >= 4;
  const int blocks = !mfma ? (s.dtype == 1 ? 2 : 4) * slots : slots >= 6 * units ? slots : 2 * slots;
  const int rows = mfma && s.dtype == 1 ? 128 : 64, n = min((blocks + units - 1) / units, (s.S + rows - 1) / rows);
  return n < 1 ? 1 : n;
}

size_t weigh_logits_pitch(int S_max) { return ((size_t)S_max + 31) / 32 * 32; }

hipError_t launch_parts(const Shape& s, int nsplit, const void* q, const void* k, const void* v, float* partial, float* logits,
                        hipStream_t st) {
  const dim3 grid(nsplit * s.B * s.Hkv), block(kPtThreads);
  const Ragged rg = with_loads(s, kEveryRow);
#define LOKI_PARTS(T, NH)                                                                                               \
  if (logits != nullptr)                                                                                                \
    hipLaunchKernelGGL((parts_kernel<T, NH, true>), grid, block, 0, st, k, v, q, partial, logits, weigh_logits_pitch(s.S), \
                       s.B, s.Hkv, s.S_cap, s.S, nsplit, rg);                                                            \
  else                                                                                                                  \
    hipLaunchKernelGGL((parts_kernel<T, NH, false>), grid, block, 0, st, k, v, q, partial, logits, weigh_logits_pitch(s.S), \
                       s.B, s.Hkv, s.S_cap, s.S, nsplit, rg);                                                            \
  break
  switch (s.dtype == 1 ? s.G : -s.G) {
    case 1: LOKI_PARTS(BF16, 1);
    case 2: LOKI_PARTS(BF16, 2);
    case 4: LOKI_PARTS(BF16, 4);
    case 8: LOKI_PARTS(BF16, 8);
    case -1: LOKI_PARTS(F32, 1);
    case -2: LOKI_PARTS(F32, 2);
    case -4: LOKI_PARTS(F32, 4);
    case -8: LOKI_PARTS(F32, 8);
    default: return hipErrorInvalidValue;
  }
#undef LOKI_PARTS
  return hipGetLastError();
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
