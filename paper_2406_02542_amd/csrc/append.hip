// Keys and values of new tokens into a cache held whole, contiguous or on pages, in the storage type or in 4 bits, the keys and the
// queries beside them turned by their positions on the way (in front of Algorithm 1 line 2 of arXiv 2406.02542); and rows of such a
// cache back.
//
// The rotation is that of rotary.hip, and so is the split: a block owns a few tokens (or some heads of one), works their angles
// out once, into LDS, and lane groups take heads of one token in turn.  Memory bounds it.
// In 4 bits the turned row goes through LDS in 32 bits, from the lanes that hold pairs to the lanes that hold words, and is rounded
// once, to its code.  Vector instructions bound that: 79 % of the SIMDs' cycles.
// 8 x up to 2048 tokens of 32/8 bf16 heads (369 MB) 68 us, 5.4 TB/s, 16 x 512 (201 MB) 36 us; 4 x up to 1111 into 4 bits, half of the columns turned 22 us (96 MB);
// one token 4.8 us, a launch.
#include "cache_impl.h"
#include "rotary_impl.h"

namespace loki {

constexpr int kApThreads = 256;
constexpr int kApMaxTokens = 4;  // of a block: one angle per thread with 64 pairs

// Where a token's row goes, from the start of the pool of head 0, and the rows between two heads'; not there: first < 0.
struct RowTarget {
  long long first, between;
};
__device__ __forceinline__ RowTarget row_target(const CacheView& c, int b, int Hkv, int row) {
  if (row < 0 || row >= c.S_cap) return {-1, 0};
  if (c.pg.table == nullptr) return {(long long)b * Hkv * c.S_cap + row, c.S_cap};
  const int page = c.pg.table[(long long)b * c.pg.pages_per_seq + (row >> c.pg.lg_rows)];
  if (page < 0 || page >= c.pg.n_pages) return {-1, 0};
  return {(((long long)page * Hkv) << c.pg.lg_rows) + (row & ((1 << c.pg.lg_rows) - 1)), 1LL << c.pg.lg_rows};
}

// Code of x: the quotient's nearest whole number, the even one half-way.  A product with the rounded reciprocal is off by less than 2^-18 there, and
// what it leaves of x - lowest, which 64 bits hold exactly, says on which side of half a step that was.
__device__ __forceinline__ uint32_t q4_code(float x, float low, float step, float inv) {
  float n = rintf((x - low) * inv);
  const double rest = fma(-(double)n, (double)step, (double)x - (double)low), over = fabs(rest) - 0.5 * (double)step;
  if (over > 0.0 || (over == 0.0 && ((int)n & 1) != 0)) n += copysignf(1.f, (float)rest);
  return step > 0.f ? (uint32_t)fminf(fmaxf(n, 0.f), 15.f) : 0u;
}

// cos and sin of an angle, formed in 64 bits and rounded once: pi / 2 in two terms takes the quarter turns off, Taylor polynomials on
// [-pi / 4, pi / 4], whose first terms left out are below 2^-54.
__device__ __forceinline__ float2 cos_sin_rounded(double x) {
  const double k = rint(x * 0.63661977236758134308), t = fma(-k, 6.123233995736766e-17, fma(-k, 1.5707963267948966, x)), t2 = t * t;
  double s = -1.0 / 1307674368000.0, c = 1.0 / 20922789888000.0;
  s = fma(s, t2, 1.0 / 6227020800.0);
  s = fma(s, t2, -1.0 / 39916800.0);
  s = fma(s, t2, 1.0 / 362880.0);
  s = fma(s, t2, -1.0 / 5040.0);
  s = fma(s, t2, 1.0 / 120.0);
  s = fma(s, t2, -1.0 / 6.0);
  s = fma(s * t2, t, t);
  c = fma(c, t2, -1.0 / 87178291200.0);
  c = fma(c, t2, 1.0 / 479001600.0);
  c = fma(c, t2, -1.0 / 3628800.0);
  c = fma(c, t2, 1.0 / 40320.0);
  c = fma(c, t2, -1.0 / 720.0);
  c = fma(c, t2, 1.0 / 24.0);
  c = fma(c, t2, -0.5);
  c = fma(c, t2, 1.0);
  const int quarter = (int)((long long)k & 3);
  const float cs = (float)(quarter & 1 ? s : c), sn = (float)(quarter & 1 ? c : s);
  return make_float2(quarter == 1 || quarter == 2 ? -cs : cs, quarter >= 2 ? -sn : sn);
}

// a x + b y, each product rounded by itself: what a value becomes, and with it its code, does not turn on which product is fused.
__device__ __forceinline__ float turned(float a, float x, float b, float y) {
#pragma clang fp contract(off)
  return a * x + b * y;
}

// The row in `row` (LDS, 128 floats, complete) as codes and scales, by the LANES lanes of a group; p: the lane's number.
template <int LANES>
__device__ __forceinline__ void store_q4(const float* row, int p, uint32_t* codes, uint32_t* scales) {
  constexpr int W = kQ4Words / LANES;
  float2 x[W][kQ4Groups];
  uint32_t word[W] = {};
#pragma unroll
  for (int w = 0; w < W; ++w)
#pragma unroll
    for (int g = 0; g < kQ4Groups; ++g) x[w][g] = *reinterpret_cast<const float2*>(row + 32 * g + 2 * (W * p + w));
  bool odd = false;  // minima and maxima pass over what is no number
#pragma unroll
  for (int w = 0; w < W; ++w)
#pragma unroll
    for (int g = 0; g < kQ4Groups; ++g) odd |= __builtin_isunordered(x[w][g].x, x[w][g].y);
  const bool any = __ballot(odd) != 0ull;
#pragma unroll
  for (int g = 0; g < kQ4Groups; ++g) {
    float lo = x[0][g].x, hi = lo;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      lo = fminf(lo, fminf(x[w][g].x, x[w][g].y));
      hi = fmaxf(hi, fmaxf(x[w][g].x, x[w][g].y));
    }
    lo = -group_allreduce_max<LANES>(-lo);
    hi = group_allreduce_max<LANES>(hi);
    // (a range past fp16's is clamped to its largest)
    cache_half2_t sc = {(_Float16)fminf((hi - lo) * (1.0f / 15.0f), 65504.f), (_Float16)fminf(fmaxf(lo, -65504.f), 65504.f)};
    if (any) {  // (uniform) a group with such a value stands for no numbers
      bool own = false;
#pragma unroll
      for (int w = 0; w < W; ++w) own |= __builtin_isunordered(x[w][g].x, x[w][g].y);
      const int lane = threadIdx.x & 63;
      if ((__ballot(own) >> (lane & ~(LANES - 1)) & ((1ull << LANES) - 1)) != 0ull) sc = cache_half2_t{(_Float16)__builtin_nanf(""), (_Float16)__builtin_nanf("")};
    }
    const float step = (float)sc.x, low = (float)sc.y, inv = 1.0f / step;
#pragma unroll
    for (int w = 0; w < W; ++w) word[w] |= q4_code(x[w][g].x, low, step, inv) << (4 * g) | q4_code(x[w][g].y, low, step, inv) << (16 + 4 * g);
    if (p == g) scales[g] = __builtin_bit_cast(uint32_t, sc);
  }
#pragma unroll
  for (int w = 0; w < W; ++w) codes[W * p + w] = word[w];
}

// STYLE as rotary_kernel's; LOADS and STORES: past the caches.  Stores past them are of whole lines: where a lane's chunks of a row leave holes, the row
// goes through LDS in front of them; us through the caches / past them with holes / so: 16 x 512 tokens of 32/8 bf16 heads, 96 columns turned 47.3 / 57.9 /
// 36.5, 64 46.6 / 44.4 / 36.3.
template <typename T, int STYLE, bool BITS4, bool LOADS, bool STORES>
__global__ __launch_bounds__(kApThreads) void append_kernel(AppendArgs args) {
  using ST = typename T::store_t;
  constexpr int EPC = T::EPC;
  constexpr int kLanes = kD / EPC / 2;  // lanes of a row: two chunks each
  constexpr int kGroups = kApThreads / kLanes;
  constexpr int kAngles = STYLE == 2 ? 1 : EPC;  // of a lane
  constexpr int U = BITS4 ? 2 : 6;               // rows of a lane group in flight
  const RotaryArgs& a = args.r;
  __shared__ float2 s_cs[kApMaxTokens][kD / 2];
  constexpr bool kLines = STYLE == 0 && STORES;
  __shared__ __align__(16) float s_row[BITS4 ? kGroups : 1][kD + 4];
  __shared__ uint4 s_line[kLines ? kGroups : 1][kD / EPC];
  const int tid = threadIdx.x, p = tid % kLanes, gid = tid / kLanes;
  const int pairs = a.R / 2, tok0 = blockIdx.x * a.tokens, ntok = min(a.tokens, a.total - tok0);
  // this lane group's token, and its heads h0 + first, h0 + first + step, ..
  const int mine = gid & (a.tokens - 1), first = gid / a.tokens, step = kGroups / a.tokens;
  const int Hkv = a.k.heads, heads = a.q.heads + 2 * Hkv;
  const int h0 = blockIdx.y * a.heads_per_block, h1 = min(h0 + a.heads_per_block, heads);
  const int t = tok0 + min(mine, ntok - 1), b = t / a.n, j = t - b * a.n;
  const RowTarget to = row_target(args.cache, b, Hkv, a.rows[t]);

  // the two chunks of this lane: a pair of rotated ones, or two of the columns behind R; and their angles
  int c0 = p, c1 = p + kLanes;
  if (STYLE == 0) {
    const int np = pairs / EPC;
    c0 = p < np ? p : p + np;
    c1 = p < np ? p + np : p + kLanes;
  }
  uint4 raw[U][2];
  const ST* src[U];  // (STYLE 2)
  auto fetch = [&](int i0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      int h = min(i0 + u * step, h1 - 1);
      const bool is_q = h < a.q.heads;
      if (!is_q) h -= a.q.heads;
      const bool is_v = !is_q && h >= Hkv;
      if (is_v) h -= Hkv;
      const RotaryTensor& x = is_q ? a.q : is_v ? a.v : a.k;
      src[u] = static_cast<const ST*>(x.in) + (b * x.in_batch + j * x.in_token + h * x.in_head);
      raw[u][0] = load16_hint<LOADS>(src[u] + c0 * EPC);
      raw[u][1] = load16_hint<LOADS>(src[u] + c1 * EPC);
    }
  };
  fetch(h0 + first);  // (before the angles, which they need not wait for; lane groups without a token take another's)

  for (int i = tid; i < ntok * pairs; i += kApThreads) {
    const int u = i / pairs, f = i - u * pairs;
    float2 cs = cos_sin_rounded((double)a.positions[tok0 + u] * a.freqs[f]);
    cs.x *= a.scale;
    cs.y *= a.inverse ? -a.scale : a.scale;
    s_cs[u][f] = cs;
  }
  __syncthreads();
  if (mine >= ntok) return;

  float2 cs[kAngles];
#pragma unroll
  for (int e = 0; e < kAngles; ++e) {
    if (STYLE == 0) cs[e] = s_cs[mine][max(0, min(c0 * EPC + e, pairs - 1))];
    if (STYLE == 1) cs[e] = s_cs[mine][max(0, min((e < EPC / 2 ? c0 : c1) * (EPC / 2) + e % (EPC / 2), pairs - 1))];
  }
  const bool holes = kLines && a.R > 0 && a.R < kD;  // (uniform)
  const bool in_r = a.R > 0 && (STYLE != 0 || c1 * EPC < a.R);  // (STYLE 0: both chunks or none)

  for (int i0 = h0 + first; i0 < h1; i0 += step * U) {
    ST* dst[U];         // null: not there; in 4 bits of the queries only
    long long at[U];    // in 4 bits, of keys and values: their row, negative: not there
    bool turn[U], is_v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * step;
      int h = min(i, h1 - 1);
      const bool is_q = h < a.q.heads;
      if (!is_q) h -= a.q.heads;
      is_v[u] = !is_q && h >= Hkv;
      if (is_v[u]) h -= Hkv;
      turn[u] = in_r && !is_v[u];
      const bool there = i < h1 && (is_q || to.first >= 0);  // (else padded)
      const long long row = to.first + h * to.between;
      at[u] = there && !is_q ? row : -1;
      dst[u] = is_q ? static_cast<ST*>(a.q.out) + (b * a.q.out_batch + j * a.q.out_token + h * a.q.out_head)
                    : static_cast<ST*>(is_v[u] ? args.cache.v : args.cache.k) + row * kD;
      if (!there || (BITS4 && !is_q)) dst[u] = nullptr;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x0[EPC], x1[EPC], y0[EPC], y1[EPC];
      T::unpack(raw[u][0], x0);
      T::unpack(raw[u][1], x1);
#pragma unroll
      for (int e = 0; e < EPC; ++e) {
        y0[e] = x0[e];
        y1[e] = x1[e];
      }
      if (turn[u]) {
        if constexpr (STYLE == 0) {
#pragma unroll
          for (int e = 0; e < EPC; ++e) {
            y0[e] = turned(x0[e], cs[e].x, x1[e], -cs[e].y);
            y1[e] = turned(x1[e], cs[e].x, x0[e], cs[e].y);
          }
        } else if constexpr (STYLE == 1) {
#pragma unroll
          for (int e = 0; e < EPC; ++e) {
            const float2 z0 = cs[e / 2], z1 = cs[(EPC + e) / 2];
            if (c0 * EPC + e < a.R) y0[e] = turned(x0[e], z0.x, x0[e ^ 1], e % 2 == 0 ? -z0.y : z0.y);
            if (c1 * EPC + e < a.R) y1[e] = turned(x1[e], z1.x, x1[e ^ 1], e % 2 == 0 ? -z1.y : z1.y);
          }
        } else {  // partners that no chunk boundary respects, element by element
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int e = 0; e < EPC; ++e) {
              const int col = (half ? c1 : c0) * EPC + e;
              if (col < a.R) {
                const bool lower = col < pairs;
                const float2 z = s_cs[mine][lower ? col : col - pairs];
                const float other = T::load1(src[u] + (lower ? col + pairs : col - pairs));
                (half ? y1[e] : y0[e]) = turned(half ? x1[e] : x0[e], z.x, other, lower ? -z.y : z.y);
              }
            }
        }
      }
      if (dst[u] != nullptr) {
        uint4 z0 = pack_chunk<T>(y0), z1 = pack_chunk<T>(y1);
        int at0 = c0, at1 = c1;
        if (holes) {
          at0 = p;
          at1 = p + kLanes;
          s_line[gid][c0] = z0;
          s_line[gid][c1] = z1;
          __builtin_amdgcn_wave_barrier();  // (the group's lanes are of one wave, whose LDS operations keep their order)
          z0 = s_line[gid][at0];
          z1 = s_line[gid][at1];
          __builtin_amdgcn_wave_barrier();
        }
        store16_hint<STORES>(dst[u] + at0 * EPC, z0);
        store16_hint<STORES>(dst[u] + at1 * EPC, z1);
      }
      if constexpr (BITS4) {
        if (at[u] >= 0) {  // (the same for the lanes of a group)
          float* mid = s_row[gid];
#pragma unroll
          for (int e = 0; e < EPC; e += 4) {
            *reinterpret_cast<float4*>(mid + c0 * EPC + e) = make_float4(y0[e], y0[e + 1], y0[e + 2], y0[e + 3]);
            *reinterpret_cast<float4*>(mid + c1 * EPC + e) = make_float4(y1[e], y1[e + 1], y1[e + 2], y1[e + 3]);
          }
          __builtin_amdgcn_wave_barrier();
          store_q4<kLanes>(mid, p, static_cast<uint32_t*>(is_v[u] ? args.cache.v : args.cache.k) + at[u] * kQ4Words,
                           static_cast<uint32_t*>(is_v[u] ? args.cache.v_scales : args.cache.k_scales) + at[u] * kQ4Groups);
          __builtin_amdgcn_wave_barrier();
        }
      }
    }
    if (i0 + step * U < h1) fetch(i0 + step * U);
  }
}

template <typename T, bool BITS4, bool LOADS, bool STORES>
static hipError_t launch_append_t(const AppendArgs& a, dim3 grid, int style, hipStream_t st) {
  const dim3 block(kApThreads);
  if (style == 0)
    hipLaunchKernelGGL((append_kernel<T, 0, BITS4, LOADS, STORES>), grid, block, 0, st, a);
  else if (style == 1)
    hipLaunchKernelGGL((append_kernel<T, 1, BITS4, LOADS, STORES>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((append_kernel<T, 2, BITS4, false, STORES>), grid, block, 0, st, a);
  return hipGetLastError();
}

hipError_t launch_append(const Shape& s, AppendArgs args, hipStream_t st) {
  RotaryArgs& a = args.r;
  const int epc = 16 / s.elem_bytes, heads = a.q.heads + 2 * s.Hkv;
  // few tokens: the heads of a token are spread over blocks (as launch_rotary).  In 4 bits, us (loading past the caches) with 4 rows of a lane group in flight and 4 tokens a
  // block, 4 and 2, 2 and 2, 2 and 4, 3 and 1: 4 x 1111 tokens of 32/8 bf16 heads 36.6, 33.7, 33.2, 33.1, 41.6, 2 x 512 15.9, 13.5, 13.4, 15.1, 13.4.
  const bool bits4 = args.cache.k_scales != nullptr;
  const int tokens = s.dtype == 0 || bits4 ? 2 : kApMaxTokens;
  a.tokens = a.total >= tokens * device_cus() ? tokens : 1;
  a.heads_per_block = heads;
  const int groups = kApThreads / (kD / epc / 2);
  if (a.tokens == 1) {
    int splits = device_cus() / a.total;
    const int most = (heads + groups - 1) / groups;
    if (splits > most) splits = most;
    if (splits > 1) a.heads_per_block = (heads + splits - 1) / splits;
  }
  const dim3 grid((a.total + a.tokens - 1) / a.tokens, (heads + a.heads_per_block - 1) / a.heads_per_block);
  const int style = a.interleaved ? 1 : (a.R / 2) % epc == 0 ? 0 : 2;
  // From 100 MB read and written on, rows are stored past the caches (but for codes and scales, which are written piece by piece); from 90 MB of rows on
  // they are loaded past them, but for half lines: us through / past: 4 x 1111 tokens of 32/8 bf16 heads into 4 bits (55 MB) with their rows read
  // back 28.1 / 33.2, 16 x 512 (101 MB) 63.1 / 57.5; into bf16, 8 x 2048 (201 MB) 70.2 / 68.4, 16 x 512 36.1 / 36.6, 96 columns turned 36.5 / 41.6.
  const double bytes = (double)a.total * heads * kD * s.elem_bytes;
  const bool holes = style == 0 && a.R > 0 && a.R < kD, stores = 2.0 * bytes >= 100e6, loads = bytes >= kPastBytes && (bits4 || !holes);
#define LOKI_APPEND(T, BITS4)                                                              \
  return loads    ? launch_append_t<T, BITS4, true, true>(args, grid, style, st)           \
         : stores ? launch_append_t<T, BITS4, false, true>(args, grid, style, st)          \
                  : launch_append_t<T, BITS4, false, false>(args, grid, style, st)
  if (bits4) {
    if (s.dtype == 0) LOKI_APPEND(F32, true);
    LOKI_APPEND(BF16, true);
  }
  if (s.dtype == 0) LOKI_APPEND(F32, false);
  LOKI_APPEND(BF16, false);
#undef LOKI_APPEND
}

// ---- rows of a cache back --------------------------------------------------------------------------------------
// 16 lanes take a row: in 4 bits a word each, so a store instruction takes the pairs of one group of 4 rows; else 16-byte chunks.  Memory bounds it: 4 x up to 1111
// rows of 8 heads out of 4 bits (20 MB) 5.8 us.
template <typename T, bool BITS4>
__global__ __launch_bounds__(256) void read_rows_kernel(CacheView c, const int32_t* __restrict__ rows, int B, int n, int Hkv,
                                                        typename T::store_t* __restrict__ k_out, typename T::store_t* __restrict__ v_out) {
  constexpr int kRows = 16, kChunks = kD / T::EPC;
  const long long at = (long long)blockIdx.x * kRows + (threadIdx.x >> 4), all = (long long)B * n * Hkv;
  const int m = threadIdx.x & 15;
  if (at >= all) return;
  const int j = (int)(at % n), h = (int)(at / n % Hkv), b = (int)(at / n / Hkv);
  const RowTarget from = row_target(c, b, Hkv, rows[(long long)b * n + j]);
  if (from.first < 0) return;
  const long long row = from.first + h * from.between;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    typename T::store_t* dst = (i ? v_out : k_out) + at * kD;
    if (i ? v_out == nullptr : k_out == nullptr) continue;
    if constexpr (BITS4) {
      const uint32_t word = static_cast<const uint32_t*>(i ? c.v : c.k)[row * kQ4Words + m];
      const uint4 sc = load16(static_cast<const uint4*>(i ? c.v_scales : c.k_scales) + row);
      const uint32_t scales[kQ4Groups] = {sc.x, sc.y, sc.z, sc.w};
#pragma unroll
      for (int g = 0; g < kQ4Groups; ++g) {
        const cache_half2_t x = __builtin_bit_cast(cache_half2_t, scales[g]);
        const float lo = fmaf((float)(word >> (4 * g) & 15u), (float)x.x, (float)x.y);
        const float hi = fmaf((float)(word >> (16 + 4 * g) & 15u), (float)x.x, (float)x.y);
        if constexpr (T::EPC == 8)
          *reinterpret_cast<uint32_t*>(dst + 32 * g + 2 * m) = BF16::round2(lo, hi);
        else
          *reinterpret_cast<float2*>(dst + 32 * g + 2 * m) = make_float2(lo, hi);
      }
    } else {
      const uint4* src = reinterpret_cast<const uint4*>(static_cast<const typename T::store_t*>(i ? c.v : c.k) + row * kD);
#pragma unroll
      for (int e = 0; e < kChunks / 16; ++e) reinterpret_cast<uint4*>(dst)[16 * e + m] = src[16 * e + m];
    }
  }
}

hipError_t launch_read_rows(const Shape& s, const CacheView& cache, const int32_t* rows, int n, void* k_out, void* v_out, hipStream_t st) {
  const dim3 grid((unsigned)(((long long)s.B * n * s.Hkv + 15) / 16)), block(256);
  const bool bits4 = cache.k_scales != nullptr;
#define LOKI_READ(T, BITS4)                                                                                              \
  hipLaunchKernelGGL((read_rows_kernel<T, BITS4>), grid, block, 0, st, cache, rows, s.B, n, s.Hkv, static_cast<T::store_t*>(k_out), \
                     static_cast<T::store_t*>(v_out))
  if (s.dtype == 0) {
    if (bits4) LOKI_READ(F32, true);
    else LOKI_READ(F32, false);
  } else {
    if (bits4) LOKI_READ(BF16, true);
    else LOKI_READ(BF16, false);
  }
#undef LOKI_READ
  return hipGetLastError();
}

}  // namespace loki
