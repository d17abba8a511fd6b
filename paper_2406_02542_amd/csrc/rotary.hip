// Rotary positions for the queries and keys of new tokens (the step in front of Algorithm 1 lines 2-4 of
// arXiv 2406.02542: q and k are rotated by their positions before they are cached).
//
// The first R columns of a head are R / 2 pairs (a, b); pair i of a token at position t becomes
//   s (a cos - b sin), s (b cos + a sin)   with the angle t f_i (its sign turned for the inverse, which is
// the gradient of the forward rotation too).  Memory bounds it: every element is read and written once, for
// about one multiply-add each.
//
// A block owns up to kRotMaxTokens tokens (or a share of one token's heads when there are few tokens) and works out their
// R / 2 angles once, into LDS, for all heads.  The angle in quarter turns is reduced in 64 bits: 32 would
// leave a position of 100 000 with angles off by 4e-3.  A lane group then takes heads of one token in turn,
// each lane two 16-byte chunks that hold both halves of its pairs, with their angles in registers, six rows in flight.
// 8 x 2048 tokens of 32/8 bf16 heads: 403 MB in 68 us (5.9 TB/s), pairs half a head apart or side by side.  Where half of the columns
// is no whole number of chunks (STYLE 2) a lane's partners lie in other lanes' chunks and are loaded one by one: 136 us with 20 columns,
// 185 with 126; 3 x 1111 tokens of 24/24 fp32 heads 72 us with 20, 47 with 64.
#include "common.h"

namespace loki {

constexpr int kRotThreads = 256;
constexpr int kRotInFlight = 6;
constexpr int kRotMaxTokens = 4;  // of a block: one angle per thread with 64 pairs

// cos and sin of x quarter turns, |x| reduced here; fp32 results.  Taylor polynomials on [-pi/4, pi/4]: the first
// term left out is below 2^-29.
__device__ __forceinline__ float2 cos_sin_quarters(double x) {
  const double k = rint(x);
  const float th = (float)(x - k) * 1.57079632679489662f, t2 = th * th;
  float s = fmaf(t2, 2.7557319224e-6f, -1.9841269841e-4f);
  s = fmaf(s, t2, 8.3333333333e-3f);
  s = fmaf(s, t2, -1.6666666667e-1f);
  s = fmaf(s * t2, th, th);
  float c = fmaf(t2, -2.7557319224e-7f, 2.4801587302e-5f);
  c = fmaf(c, t2, -1.3888888889e-3f);
  c = fmaf(c, t2, 4.1666666667e-2f);
  c = fmaf(c, t2, -0.5f);
  c = fmaf(c, t2, 1.0f);
  const int quarter = (int)((long long)k & 3);
  const float cs = quarter & 1 ? s : c, sn = quarter & 1 ? c : s;
  return make_float2(quarter == 1 || quarter == 2 ? -cs : cs, quarter >= 2 ? -sn : sn);
}

template <typename T>
__device__ __forceinline__ uint4 pack_chunk(const float (&f)[T::EPC]) {
  if constexpr (T::EPC == 8)
    return make_uint4(BF16::round2(f[0], f[1]), BF16::round2(f[2], f[3]), BF16::round2(f[4], f[5]), BF16::round2(f[6], f[7]));
  else
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}

// STYLE: 0 pairs (i, i + R / 2), R / 2 a multiple of a chunk; 1 pairs (2 i, 2 i + 1); 2 as 0, any even R.
// STREAM: rows are loaded and stored past the caches (launch_rotary).
template <typename T, int STYLE, bool STREAM>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotaryArgs a) {
  using ST = typename T::store_t;
  constexpr int EPC = T::EPC;
  constexpr int kLanes = kD / EPC / 2;  // lanes of a row: two chunks each
  constexpr int kGroups = kRotThreads / kLanes;
  constexpr int kAngles = STYLE == 2 ? 1 : EPC;  // of a lane
  __shared__ float2 s_cs[kRotMaxTokens][kD / 2];
  const int tid = threadIdx.x, p = tid % kLanes, gid = tid / kLanes;
  const int pairs = a.R / 2, tok0 = blockIdx.x * a.tokens, ntok = min(a.tokens, a.total - tok0);
  // this lane group's token, and its heads h0 + first, h0 + first + step, ..
  const int mine = gid & (a.tokens - 1), first = gid / a.tokens, step = kGroups / a.tokens;
  const int heads = a.q.heads + a.k.heads + a.v.heads;
  const int h0 = blockIdx.y * a.heads_per_block, h1 = min(h0 + a.heads_per_block, heads);
  const int t = tok0 + min(mine, ntok - 1), b = t / a.n, j = t - b * a.n;
  const int row = a.rows != nullptr ? a.rows[t] : j;

  for (int i = tid; i < ntok * pairs; i += kRotThreads) {
    const int u = i / pairs, f = i - u * pairs;
    const double quarters = (double)a.positions[tok0 + u] * (a.freqs[f] * 0.63661977236758134308);  // 2 / pi
    float2 cs = cos_sin_quarters(quarters);
    cs.x *= a.scale;
    cs.y *= a.inverse ? -a.scale : a.scale;
    s_cs[u][f] = cs;
  }
  __syncthreads();
  if (mine >= ntok) return;

  // the two chunks of this lane: a pair of rotated ones, or two of the columns behind R; and their angles
  int c0 = p, c1 = p + kLanes;
  if (STYLE == 0) {
    const int np = pairs / EPC;
    c0 = p < np ? p : p + np;
    c1 = p < np ? p + np : p + kLanes;
  }
  float2 cs[kAngles];
#pragma unroll
  for (int e = 0; e < kAngles; ++e) {
    if (STYLE == 0) cs[e] = s_cs[mine][min(c0 * EPC + e, pairs - 1)];
    if (STYLE == 1) cs[e] = s_cs[mine][min((e < EPC / 2 ? c0 : c1) * (EPC / 2) + e % (EPC / 2), pairs - 1)];
  }
  const bool in_r = STYLE != 0 || c1 * EPC < a.R;  // (STYLE 0: both chunks or none)
  const bool row_there = a.rows == nullptr || (row >= 0 && row < a.n_rows);

  for (int i0 = h0 + first; i0 < h1; i0 += step * kRotInFlight) {
    uint4 raw[kRotInFlight][2];
    ST* dst[kRotInFlight];
    bool turn[kRotInFlight];
#pragma unroll
    for (int u = 0; u < kRotInFlight; ++u) {
      int h = min(i0 + u * step, h1 - 1);
      const bool is_q = h < a.q.heads;
      if (!is_q) h -= a.q.heads;
      const bool is_k = !is_q && h < a.k.heads;
      if (!is_q && !is_k) h -= a.k.heads;
      const RotaryTensor& x = is_q ? a.q : is_k ? a.k : a.v;
      const ST* src = static_cast<const ST*>(x.in) + (b * x.in_batch + j * x.in_token + h * x.in_head);
      raw[u][0] = load16_hint<STREAM>(src + c0 * EPC);
      raw[u][1] = load16_hint<STREAM>(src + c1 * EPC);
      turn[u] = in_r && (is_q || is_k);
      dst[u] = static_cast<ST*>(x.out) + (b * x.out_batch + (is_q ? j : row) * x.out_token + h * x.out_head);
      if (i0 + u * step >= h1 || !(is_q || row_there)) dst[u] = nullptr;
      if constexpr (STYLE == 2) {
        // partners that no chunk boundary respects, element by element; read before anything of the row is written
        if (turn[u]) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            float x0[EPC];
            T::unpack(raw[u][half], x0);
#pragma unroll
            for (int e = 0; e < EPC; ++e) {
              const int col = (half ? c1 : c0) * EPC + e;
              if (col < a.R) {
                const bool lower = col < pairs;
                const float2 y = s_cs[mine][lower ? col : col - pairs];
                const float other = T::load1(src + (lower ? col + pairs : col - pairs));
                x0[e] = lower ? x0[e] * y.x - other * y.y : x0[e] * y.x + other * y.y;
              }
            }
            raw[u][half] = pack_chunk<T>(x0);
          }
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kRotInFlight; ++u) {
      if constexpr (STYLE == 0) {
        if (turn[u]) {
          float x0[EPC], x1[EPC], y0[EPC], y1[EPC];
          T::unpack(raw[u][0], x0);
          T::unpack(raw[u][1], x1);
#pragma unroll
          for (int e = 0; e < EPC; ++e) {
            y0[e] = x0[e] * cs[e].x - x1[e] * cs[e].y;
            y1[e] = x1[e] * cs[e].x + x0[e] * cs[e].y;
          }
          raw[u][0] = pack_chunk<T>(y0);
          raw[u][1] = pack_chunk<T>(y1);
        }
      } else if constexpr (STYLE == 1) {
        if (turn[u]) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            float x0[EPC];
            T::unpack(raw[u][half], x0);
#pragma unroll
            for (int e = 0; e < EPC; e += 2) {
              if ((half ? c1 : c0) * EPC + e < a.R) {
                const float2 y = cs[(half * EPC + e) / 2];
                const float x = x0[e], z = x0[e + 1];
                x0[e] = x * y.x - z * y.y;
                x0[e + 1] = z * y.x + x * y.y;
              }
            }
            raw[u][half] = pack_chunk<T>(x0);
          }
        }
      }
      if (dst[u] != nullptr) {
        store16_hint<STREAM>(dst[u] + c0 * EPC, raw[u][0]);
        store16_hint<STREAM>(dst[u] + c1 * EPC, raw[u][1]);
      }
    }
  }
}

template <typename T, bool STREAM>
static hipError_t launch_rotary_t(const RotaryArgs& a, dim3 grid, int style, hipStream_t st) {
  const dim3 block(kRotThreads);
  if (style == 0)
    hipLaunchKernelGGL((rotary_kernel<T, 0, STREAM>), grid, block, 0, st, a);
  else if (style == 1)
    hipLaunchKernelGGL((rotary_kernel<T, 1, STREAM>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((rotary_kernel<T, 2, false>), grid, block, 0, st, a);
  return hipGetLastError();
}

hipError_t launch_rotary(const Shape& s, RotaryArgs a, hipStream_t st) {
  const int epc = 16 / s.elem_bytes, heads = a.q.heads + a.k.heads + a.v.heads;
  // few tokens: the heads of a token are spread over blocks until every CU has one or a lane group has one row
  // (us with 4, 2 and 1 tokens a block: 8 x 2048 of 32/8 bf16 heads 69, 78, 115: the angles are worked out by a few lanes; 3 x
  // 1111 of 24/24 fp32 heads 56, 54, 51, 4 x 1024 of 32/8 39, 38, 42: larger blocks leave the last round uneven)
  const int tokens = s.dtype == 0 ? 2 : kRotMaxTokens;
  a.tokens = a.total >= tokens * device_cus() ? tokens : 1;
  a.heads_per_block = heads;
  const int groups = kRotThreads / (kD / epc / 2);
  if (a.tokens == 1) {
    int splits = device_cus() / a.total;
    const int most = (heads + groups - 1) / groups;
    if (splits > most) splits = most;
    if (splits > 1) a.heads_per_block = (heads + splits - 1) / splits;
  }
  const dim3 grid((a.total + a.tokens - 1) / a.tokens, (heads + a.heads_per_block - 1) / a.heads_per_block);
  const int style = a.interleaved ? 1 : (a.R / 2) % epc == 0 ? 0 : 2;
  // From 100 MB read and written on, past the caches.  us through / past: 88 MB 18.5 / 18.8, 101 22.4 / 20.8, 157 34.5 / 30.2,
  // 202 41.9 / 38.0, 246 50.1 / 46.0, 403 77.6 / 72.8.
  const bool past = 2.0 * a.total * heads * kD * s.elem_bytes >= 100e6;
  if (s.dtype == 0)
    return past ? launch_rotary_t<F32, true>(a, grid, style, st) : launch_rotary_t<F32, false>(a, grid, style, st);
  return past ? launch_rotary_t<BF16, true>(a, grid, style, st) : launch_rotary_t<BF16, false>(a, grid, style, st);
}

}  // namespace loki
