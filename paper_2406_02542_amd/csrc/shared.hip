// Attention of a whole batch over the prefix that its sequences share (Section 2, Eq. 1 of arXiv 2406.02542, the
// part of the rows that is the same for all): the prefix's keys and values are held once, and the B G query rows
// of a KV head meet each of them in one product.  A run of the prefix leaves (max, sum, output) per query row, which
// weigh_merge_kernel joins with the parts of the sequence's own rows.
#include "attend_mfma_impl.h"

namespace loki {

constexpr int kPfThreads = 256;
constexpr int kPfWaves = kPfThreads / 64;

// Row of q (and of the partial results) that query row r of KV head h is: r = b G + g.
__device__ __forceinline__ size_t prefix_head(int r, int h, int G, int Hq) {  // (G is a power of two)
  return (size_t)(r >> (31 - __builtin_clz(G))) * Hq + h * G + (r & (G - 1));
}

// ---- fp32: matrix cores straight from registers ------------------------------------------------------------------
// A wave takes steps of 16 keys and holds QG groups of 16 query rows:
//   S^T[key, query] = K Q^T         v_mfma_f32_16x16x4_f32; lane (key, c) loads 16 bytes of its key's row at a time, columns
//                                   16 j + 4 c .. + 3, one for each of four products, and the queries the same columns
//   O^T[column, query] += V^T P^T   the weights as they come out of the first product are operand i's keys 4 c + i; lane (m, c)
//                                   loads 16 bytes of each of these rows, columns 4 m .. + 3 of either half
// A step's keys and values are in registers before it begins.  The block's waves take steps in turn and are joined in LDS.
typedef float pf_f32x4_t __attribute__((ext_vector_type(4)));
constexpr int kPfSteps = 16;       // keys of a step
constexpr float kPfGrowth = 256.0f;  // the reference of the exponentials follows the maximum when weights sum up to more

template <int QG>
__global__ __launch_bounds__(kPfThreads, QG == 1 ? 3 : QG == 2 ? 2 : 1) void prefix_f32_kernel(
    const float* __restrict__ k, const float* __restrict__ v, const float* __restrict__ qv, float* __restrict__ partial, int M, int G,
    int Hq, int rows, int cap, int run) {
  __shared__ __align__(16) float s_o[kPfWaves / 2][QG][32][64];
  __shared__ float2 s_ml[kPfWaves][QG][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, c4 = lane >> 4;
  const int split = blockIdx.x, h = blockIdx.z, q0 = blockIdx.y * (QG * 16);
  const int r0 = split * run, r1 = min(rows, r0 + run);
  const float* kh = k + (size_t)h * cap * kD + 4 * c4;
  const float* vh = v + (size_t)h * cap * kD + 4 * l16;

  float4 q[QG][8];
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    const float* src = qv + prefix_head(min(q0 + 16 * g + l16, M - 1), h, G, Hq) * kD + 4 * c4;
#pragma unroll
    for (int j = 0; j < 8; ++j) q[g][j] = *reinterpret_cast<const float4*>(src + 16 * j);
  }
  float m[QG], l[QG];
  pf_f32x4_t o[QG][8];
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    m[g] = kNegBig;
    l[g] = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) o[g][c] = pf_f32x4_t{};
  }
  float4 kr[8], vr[4][2];
  auto load_k = [&](int at) __attribute__((always_inline)) {  // (past the end: the last row again)
    const float* p = kh + (size_t)min(at + l16, r1 - 1) * kD;
#pragma unroll
    for (int j = 0; j < 8; ++j) kr[j] = *reinterpret_cast<const float4*>(p + 16 * j);
  };
  auto load_v = [&](int at) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float* p = vh + (size_t)min(at + 4 * c4 + i, r1 - 1) * kD;
      vr[i][0] = *reinterpret_cast<const float4*>(p);
      vr[i][1] = *reinterpret_cast<const float4*>(p + 64);
    }
  };
  int at = r0 + wave * kPfSteps;
  if (at < r1) {  // (uniform for the wave)
    load_k(at);
    load_v(at);
  }
  for (; at < r1; at += kPfWaves * kPfSteps) {
    pf_f32x4_t s[QG];
#pragma unroll
    for (int g = 0; g < QG; ++g) s[g] = pf_f32x4_t{};
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int g = 0; g < QG; ++g) {
        s[g] = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[j].x, q[g][j].x, s[g], 0, 0, 0);
        s[g] = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[j].y, q[g][j].y, s[g], 0, 0, 0);
        s[g] = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[j].z, q[g][j].z, s[g], 0, 0, 0);
        s[g] = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[j].w, q[g][j].w, s[g], 0, 0, 0);
      }
    load_k(at + kPfWaves * kPfSteps);
#pragma unroll
    for (int g = 0; g < QG; ++g) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[g][i] = at + 4 * c4 + i < r1 ? s[g][i] * kSoftmaxScaleLog2 : kNegBig;
      float p[4], sum;
      auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = fast_exp2(s[g][i] - m[g]);
        sum = (p[0] + p[1]) + (p[2] + p[3]);
      };
      weights();
      if (__ballot(!(sum <= kPfGrowth)) != 0ull) {
        float top = fmaxf(fmaxf(s[g][0], s[g][1]), fmaxf(s[g][2], s[g][3]));
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
#pragma unroll
      for (int i = 0; i < 4; ++i) s[g][i] = p[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int g = 0; g < QG; ++g)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          o[g][4 * c] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr[i][c].x, s[g][i], o[g][4 * c], 0, 0, 0);
          o[g][4 * c + 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr[i][c].y, s[g][i], o[g][4 * c + 1], 0, 0, 0);
          o[g][4 * c + 2] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr[i][c].z, s[g][i], o[g][4 * c + 2], 0, 0, 0);
          o[g][4 * c + 3] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr[i][c].w, s[g][i], o[g][4 * c + 3], 0, 0, 0);
        }
    load_v(at + kPfWaves * kPfSteps);
  }

  // the four waves' shares of the keys
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    l[g] += __shfl_xor(l[g], 16);
    l[g] += __shfl_xor(l[g], 32);
    if (c4 == 0) s_ml[wave][g][l16] = make_float2(m[g], l[g]);
  }
  __syncthreads();
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    float mn = kNegBig, ls = 0.f;
#pragma unroll
    for (int w = 0; w < kPfWaves; ++w) mn = fmaxf(mn, s_ml[w][g][l16].x);
#pragma unroll
    for (int w = 0; w < kPfWaves; ++w) ls = fmaf(s_ml[w][g][l16].y, fast_exp2(s_ml[w][g][l16].x - mn), ls);
    const float f = fast_exp2(m[g] - mn);
    m[g] = mn;
    l[g] = ls;
#pragma unroll
    for (int c = 0; c < 8; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[g][c][i] *= f;
  }
#pragma unroll
  for (int n = kPfWaves / 2; n >= 1; n /= 2) {
    if (wave >= n && wave < 2 * n) {
#pragma unroll
      for (int g = 0; g < QG; ++g)
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) s_o[wave - n][g][4 * c + i][lane] = o[g][c][i];
    }
    __syncthreads();
    if (wave < n) {
#pragma unroll
      for (int g = 0; g < QG; ++g)
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[g][c][i] += s_o[wave][g][4 * c + i][lane];
    }
    __syncthreads();
  }
  if (wave != 0) return;
  // o[4 c + t][i] is column 64 c + 4 (4 c4 + i) + t of query l16
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    const int r = q0 + 16 * g + l16;
    if (r >= M) continue;
    float* pr = partial + (prefix_head(r, h, G, Hq) * gridDim.x + split) * kPartStride;
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(pr + 64 * c + 16 * c4 + 4 * i) =
            make_float4(o[g][4 * c][i], o[g][4 * c + 1][i], o[g][4 * c + 2][i], o[g][4 * c + 3][i]);
    if (c4 == 0) *reinterpret_cast<float2*>(pr + kD) = make_float2(m[g], l[g]);
  }
}

// ---- bf16, more than 16 query rows per KV head: matrix cores on tiles that the block's waves share -------------
// A wave holds QG groups of 32 query rows (their columns as operands in registers, 32 a group, and their outputs, 64) and
// takes steps of 32 keys:
//   S^T[key, query] = K Q^T      v_mfma_f32_32x32x16_bf16, A = 16 bytes of a key row, B = the queries
//   weights                      a lane has 16 of the 32 keys of ONE query, so maximum, sum and the rescaling of its outputs
//                                are the lane's own but for one exchange with lane ^ 32
//   O^T[column, query] += V^T P^T    B = the weights as they come out of the first product: the order of the keys in a
//                                product is free, so A takes the same one, rows read column-wise by the transposing LDS load
// K and V tiles of KT keys go through LDS once for the block's four waves, WQ of which hold different queries and WK = 4 / WQ
// different keys of the tile; the next tile is loaded into registers while this one is used.  16-byte chunks are stored at
// places exchanged by the row's number, so that neither the key rows (stride 256 bytes) nor the four rows of a transposing
// load meet in a bank.
// The reference of the exponentials follows the running maximum only when that has grown by 2^8: the outputs (half of the
// registers) are rescaled a few times per run instead of in most steps, and weights up to 2^8 lose nothing in fp32.
typedef float pf_f32x16_t __attribute__((ext_vector_type(16)));
typedef short pf_s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) pf_s16x4_t pf_lds_s16x4_t;
typedef __bf16 pf_bf16x2_t __attribute__((ext_vector_type(2)));

template <int WAVES, int WQ>
constexpr int pf_tile_keys() {
  return WAVES / WQ == 4 ? 128 : 64;
}

// LDS: two pairs of tiles; at the end, where waves have other keys of the same queries, what half of them hand over.
template <int QG, int WAVES, int WQ>
constexpr int pf_lds_bytes() {
  const int tiles = 4 * pf_tile_keys<WAVES, WQ>() * 256, merge = WQ == WAVES ? 0 : WAVES * QG * 32 * 8 + WAVES / 2 * QG * 64 * 256;
  return tiles > merge ? tiles : merge;
}

template <int QG, int WAVES, int WQ>
__global__ __launch_bounds__(64 * WAVES, QG == 2 ? 1 : 2) void prefix_mfma_kernel(
    const uint16_t* __restrict__ k, const uint16_t* __restrict__ v, const uint16_t* __restrict__ qv, float* __restrict__ partial,
    int M, int G, int Hq, int rows, int cap, int run) {
  constexpr int kThreads = 64 * WAVES, WK = WAVES / WQ, KT = pf_tile_keys<WAVES, WQ>(), kSteps = KT / (32 * WK), kChunks = KT * 16 / kThreads;
  constexpr int kTileBytes = KT * 256;
  extern __shared__ __align__(16) char smem[];  // [2][K tile, V tile]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, half = lane >> 5, l16 = lane & 15;
  const int wq = wave % WQ, wk = wave / WQ;
  const int split = blockIdx.x, h = blockIdx.z;
  const int q0 = (blockIdx.y * WQ + wq) * (QG * 32);
  const int r0 = split * run, r1 = min(rows, r0 + run);
  const int tiles = (r1 - r0 + KT - 1) / KT;

  am_bf16x8_t q[QG][8];
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    const int r = min(q0 + 32 * g + l32, M - 1);
    const uint16_t* src = qv + prefix_head(r, h, G, Hq) * kD + 8 * half;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      q[g][ks] = __builtin_bit_cast(am_bf16x8_t, load16(src + 16 * ks));
      if constexpr (QG == 2) asm volatile("" : "+a"(q[g][ks]));  // in accumulation registers: the others are for the loads
    }
  }
  const uint16_t* kh = k + (size_t)h * cap * kD;
  const uint16_t* vh = v + (size_t)h * cap * kD;

  uint4 kst[kChunks], vst[kChunks];
  auto load = [&](int t) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < kChunks; ++j) {
      const int at = tid + kThreads * j;
      const size_t off = (size_t)min(r0 + t * KT + (at >> 4), r1 - 1) * kD + (at & 15) * 8;  // past the end: the last row again
      kst[j] = load16(kh + off);
      vst[j] = load16(vh + off);
    }
  };
  auto store = [&](int b) __attribute__((always_inline)) {
    char* base = smem + b * 2 * kTileBytes;
#pragma unroll
    for (int j = 0; j < kChunks; ++j) {
      const int at = tid + kThreads * j, row = at >> 4, c = at & 15;
      *reinterpret_cast<uint4*>(base + row * 256 + ((c ^ (row & 15)) * 16)) = kst[j];
      *reinterpret_cast<uint4*>(base + kTileBytes + row * 256 + ((c ^ ((row & 3) << 2)) * 16)) = vst[j];
    }
  };

  float m[QG], l[QG];
  pf_f32x16_t o[QG][4];
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    m[g] = kNegBig;
    l[g] = 0.f;
#pragma unroll
    for (int c = 0; c < 4; ++c) o[g][c] = pf_f32x16_t{};
  }
  const int k_at = l32 * 256 + ((half ^ (l32 & 15)) * 16);
  const int v_row = 4 * half + (l16 >> 2);
  const int v_at = kTileBytes + v_row * 256 + (((((lane >> 4) & 1) * 2 + ((l16 & 3) >> 1)) ^ ((v_row & 3) << 2)) * 16) + (l16 & 1) * 8;

  // one step: 32 keys of the tile in buffer `base`; ENDS: only the first `there` exist
  auto step = [&](const char* base, int there, auto ends) __attribute__((always_inline)) {
    // the operands of a product are asked for together and ahead: left to itself the compiler waits for each in turn
    am_bf16x8_t ka[8], va[2][4];
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) ka[ks] = __builtin_bit_cast(am_bf16x8_t, *reinterpret_cast<const uint4*>(base + (k_at ^ (ks * 32))));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const char* at = base + (v_at ^ (c * 64)) + ks * 4096;
        const pf_s16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((pf_lds_s16x4_t*)(at));
        const pf_s16x4_t y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((pf_lds_s16x4_t*)(at + 2048));
        va[ks][c] = __builtin_bit_cast(am_bf16x8_t, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
      }
    pf_f32x16_t s[QG];
#pragma unroll
    for (int g = 0; g < QG; ++g) s[g] = pf_f32x16_t{};
#pragma unroll
    for (int ks = 0; ks < 8; ++ks)
#pragma unroll
      for (int g = 0; g < QG; ++g) s[g] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[ks], q[g][ks], s[g], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
    uint32_t w[QG][8];
#pragma unroll
    for (int g = 0; g < QG; ++g) {
      if constexpr (decltype(ends)::value) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (8 * (i >> 2) + 4 * half + (i & 3) >= there) s[g][i] = kNegBig;
      }
      float sum;
      auto weights = [&]() __attribute__((always_inline)) {
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          w[g][i] = BF16::round2(fast_exp2(fmaf(s[g][2 * i], kSoftmaxScaleLog2, -m[g])), fast_exp2(fmaf(s[g][2 * i + 1], kSoftmaxScaleLog2, -m[g])));
          sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(pf_bf16x2_t, w[g][i]), __builtin_bit_cast(pf_bf16x2_t, 0x3f803f80u), sum, false);
        }
      };
      weights();
      if (__ballot(!(sum <= kPfGrowth)) != 0ull) {
        float top = s[g][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[g][i]);
        top = fmaxf(top, __shfl_xor(top, 32)) * kSoftmaxScaleLog2;
        const float mn = fmaxf(m[g], top), corr = fast_exp2(m[g] - mn);
        m[g] = mn;
        l[g] *= corr;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[g][c][i] *= corr;
        // (the outputs stay in accumulation registers on both ways past here: else all of them are copied in every step)
        if constexpr (QG == 2) {
#pragma unroll
          for (int c = 0; c < 4; ++c) asm volatile("" : "+a"(o[g][c]));
        }
        weights();
      }
      l[g] += sum;
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int g = 0; g < QG; ++g)
          o[g][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              va[ks][c], __builtin_bit_cast(am_bf16x8_t, make_uint4(w[g][4 * ks], w[g][4 * ks + 1], w[g][4 * ks + 2], w[g][4 * ks + 3])), o[g][c], 0, 0, 0);
  };

  load(0);
  store(0);
  __syncthreads();
  for (int t = 0; t < tiles - 1; ++t) {
    load(t + 1);
    const char* base = smem + (t & 1) * 2 * kTileBytes;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) step(base + (s * WK + wk) * 32 * 256, 32, std::false_type{});
    store((t + 1) & 1);
    __syncthreads();
  }
  for (int s = 0; s < kSteps; ++s) {
    const int key = (s * WK + wk) * 32, there = r1 - r0 - (tiles - 1) * KT - key;
    if (there > 0) step(smem + ((tiles - 1) & 1) * 2 * kTileBytes + key * 256, there, std::true_type{});  // (uniform for the wave)
  }
  __syncthreads();

  // both halves of a query's keys; then the waves that had other keys of the same queries
#pragma unroll
  for (int g = 0; g < QG; ++g) l[g] += __shfl_xor(l[g], 32);
  if constexpr (WK > 1) {
    float* ml = reinterpret_cast<float*>(smem);  // [wave][QG][32] (max, sum)
    float4* ob = reinterpret_cast<float4*>(smem + WAVES * QG * 32 * 8);  // [wave of the upper half][QG][4][4][lane]
#pragma unroll
    for (int g = 0; g < QG; ++g)
      if (half == 0) *reinterpret_cast<float2*>(ml + ((wave * QG + g) * 32 + l32) * 2) = make_float2(m[g], l[g]);
    __syncthreads();
#pragma unroll
    for (int g = 0; g < QG; ++g) {
      float mn = kNegBig, ls = 0.f;
#pragma unroll
      for (int w = 0; w < WK; ++w) mn = fmaxf(mn, ml[(((w * WQ + wq) * QG + g) * 32 + l32) * 2]);
#pragma unroll
      for (int w = 0; w < WK; ++w) {
        const float2 x = *reinterpret_cast<const float2*>(ml + (((w * WQ + wq) * QG + g) * 32 + l32) * 2);
        ls = fmaf(x.y, fast_exp2(x.x - mn), ls);
      }
      const float f = fast_exp2(m[g] - mn);
      m[g] = mn;
      l[g] = ls;
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[g][c][i] *= f;
    }
#pragma unroll
    for (int n = WK / 2; n >= 1; n /= 2) {
      if (wk >= n && wk < 2 * n) {
        float4* dst = ob + (size_t)((wk - n) * WQ + wq) * QG * 16 * 64;
#pragma unroll
        for (int g = 0; g < QG; ++g)
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              dst[((g * 4 + c) * 4 + i) * 64 + lane] = make_float4(o[g][c][4 * i], o[g][c][4 * i + 1], o[g][c][4 * i + 2], o[g][c][4 * i + 3]);
      }
      __syncthreads();
      if (wk < n) {
        const float4* src = ob + (size_t)(wk * WQ + wq) * QG * 16 * 64;
#pragma unroll
        for (int g = 0; g < QG; ++g)
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float4 x = src[((g * 4 + c) * 4 + i) * 64 + lane];
              o[g][c][4 * i] += x.x;
              o[g][c][4 * i + 1] += x.y;
              o[g][c][4 * i + 2] += x.z;
              o[g][c][4 * i + 3] += x.w;
            }
      }
      __syncthreads();
    }
    if (wk != 0) return;
  }
  // a lane has four columns of one query at a time: through LDS, so that a store takes four half rows
  char* mine = smem + wave * 8192;  // [32 queries][64 columns], 16-byte chunks exchanged as the keys'
#pragma unroll
  for (int g = 0; g < QG; ++g) {
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const pf_f32x16_t& x = o[g][2 * pass + c];
          *reinterpret_cast<float4*>(mine + l32 * 256 + (((8 * c + 2 * i + half) ^ l16) * 16)) = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
        }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int row = 4 * j + (lane >> 4), r = q0 + 32 * g + row;
        const float4 x = *reinterpret_cast<const float4*>(mine + row * 256 + ((l16 ^ (row & 15)) * 16));
        if (r < M) *reinterpret_cast<float4*>(partial + (prefix_head(r, h, G, Hq) * gridDim.x + split) * kPartStride + 64 * pass + 4 * l16) = x;
      }
      __builtin_amdgcn_wave_barrier();
    }
    const int r = q0 + 32 * g + l32;
    if (half == 0 && r < M)
      *reinterpret_cast<float2*>(partial + (prefix_head(r, h, G, Hq) * gridDim.x + split) * kPartStride + kD) = make_float2(m[g], l[g]);
  }
}

// The block's queries and tiles for M query rows: as few blocks of queries as possible, and waves on different keys where
// they do not fill four waves.
struct PrefixShape {
  int queries, keys, blocks_per_cu;  // of a block; keys: what a run is a multiple of
};
static PrefixShape prefix_shape(const Shape& s) {
  const int M = s.B * s.G;
  if (s.dtype == 0) return M <= 16 ? PrefixShape{16, 64, 3} : M <= 32 ? PrefixShape{32, 64, 2} : PrefixShape{64, 64, 1};
  if (M <= 32) return {32, 128, 1};
  if (M <= 64) return {64, 128, 1};
  if (M <= 128) return {128, 64, 1};
  return {256, 64, 1};
}

static int prefix_run(const Shape& s, int rows) {
  const PrefixShape ps = prefix_shape(s);
  const int tiles = s.Hkv * ((s.B * s.G + ps.queries - 1) / ps.queries);
  int n = ps.blocks_per_cu * device_cus() / tiles;
  if (n < 1) n = 1;
  const int run = (rows + n - 1) / n;
  return (run + ps.keys - 1) / ps.keys * ps.keys;
}

int prefix_splits(const Shape& s, int prefix_rows) {
  if (prefix_rows < 1) return 0;
  const int run = prefix_run(s, prefix_rows);
  return (prefix_rows + run - 1) / run;
}

template <int QG, int WAVES, int WQ>
static hipError_t launch_prefix_mfma(const Shape& s, int splits, const void* q, const void* k, const void* v,
                                     int rows, int cap, float* partial, hipStream_t st) {
  static std::atomic<unsigned long long> raised{0};
  constexpr int bytes = pf_lds_bytes<QG, WAVES, WQ>();
  const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(&prefix_mfma_kernel<QG, WAVES, WQ>), bytes, raised);
  if (e != hipSuccess) return e;
  const int M = s.B * s.G, nq = QG * WQ * 32;
  hipLaunchKernelGGL((prefix_mfma_kernel<QG, WAVES, WQ>), dim3(splits, (M + nq - 1) / nq, s.Hkv), dim3(64 * WAVES), bytes, st,
                     static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v), static_cast<const uint16_t*>(q), partial, M, s.G,
                     s.Hq, rows, cap, prefix_run(s, rows));
  return hipGetLastError();
}

template <int QG>
static hipError_t launch_prefix_f32(const Shape& s, int splits, const void* q, const void* k, const void* v,
                                    int rows, int cap, float* partial, hipStream_t st) {
  const int M = s.B * s.G, nq = QG * 16;
  hipLaunchKernelGGL((prefix_f32_kernel<QG>), dim3(splits, (M + nq - 1) / nq, s.Hkv), dim3(kPfThreads), 0, st,
                     static_cast<const float*>(k), static_cast<const float*>(v), static_cast<const float*>(q), partial, M, s.G, s.Hq,
                     rows, cap, prefix_run(s, rows));
  return hipGetLastError();
}

hipError_t launch_prefix(const Shape& s, int splits, const void* q, const void* k, const void* v, int rows,
                         int cap, float* partial, hipStream_t st) {
  const int nq = prefix_shape(s).queries;
#define LOKI_PREFIX(f) return f(s, splits, q, k, v, rows, cap, partial, st)
  if (s.dtype == 0) {
    if (nq == 16) LOKI_PREFIX(launch_prefix_f32<1>);
    if (nq == 32) LOKI_PREFIX(launch_prefix_f32<2>);
    LOKI_PREFIX(launch_prefix_f32<4>);
  }
  if (nq == 32) LOKI_PREFIX((launch_prefix_mfma<1, 4, 1>));
  if (nq == 64) LOKI_PREFIX((launch_prefix_mfma<1, 8, 2>));
  if (nq == 128) LOKI_PREFIX((launch_prefix_mfma<1, 8, 4>));
  LOKI_PREFIX((launch_prefix_mfma<1, 8, 8>));
#undef LOKI_PREFIX
}

}  // namespace loki
