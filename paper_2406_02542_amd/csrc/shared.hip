// Attention of a whole batch over the prefix that its sequences share (Section 2, Eq. 1 of arXiv 2406.02542, the
// part of the rows that is the same for all) and over the rows of its own that each sequence has: the prefix's keys and
// values are held once, and the M = B G query rows of a KV head meet each of them in one product.
//
// One launch of two kinds of blocks: a run of the prefix for a tile of query rows (below), and a run of a sequence's own rows
// for its G heads (parts_impl.h).  Each leaves (max, sum, output) per query row, which weigh_merge_kernel joins.  Few
// query rows: memory bounds it (16 sequences of 32/8 heads behind 65536 rows: 268 MB, the call 57 us).  From about 120 on the
// matrix cores do: the prefix is then read once by the chip for 6 M D operations a row.
#include "parts_impl.h"

namespace loki {

constexpr int kPfThreads = 256;
constexpr int kPfWaves = kPfThreads / 64;

struct PrefixArgs {
  const void *k, *v;  // [Hkv, cap, 128]
  float* partial;     // [B Hq, splits] parts
  int M, G, Hq, rows, cap, run, splits, tiles;
};
// Which run of the prefix, which tile of query rows, which KV head a block takes.
struct PrefixAt {
  int split, tile, h;
};

// Row of q (and of the partial results) that query row r of KV head h is: r = b G + g (G is a power of two).
__device__ __forceinline__ size_t prefix_head(int r, int h, int G, int Hq) {
  return (size_t)(r >> (31 - __builtin_clz(G))) * Hq + h * G + (r & (G - 1));
}

// ---- fp32: the loop of parts_impl.h over 16 or 32 query rows of the batch at a time -------------------------------------
template <int QG>
__device__ __forceinline__ void prefix_f32_body(char* smem, const PrefixAt& block, const float* __restrict__ qv, const PrefixArgs& a) {
  const int q0 = block.tile * (QG * 16), r0 = block.split * a.run, r1 = min(a.rows, r0 + a.run);
  attend_f32<QG, kPfWaves, false>(
      *reinterpret_cast<AttendF32Smem<QG, kPfWaves>*>(smem), static_cast<const float*>(a.k) + (size_t)block.h * a.cap * kD,
      static_cast<const float*>(a.v) + (size_t)block.h * a.cap * kD, r0, r1,
      [&](int i) { return qv + prefix_head(min(q0 + i, a.M - 1), block.h, a.G, a.Hq) * kD; },
      [&](int i) { return q0 + i < a.M ? a.partial + (prefix_head(q0 + i, block.h, a.G, a.Hq) * a.splits + block.split) * kPartStride : nullptr; },
      NoLogits{});
}

// ---- bf16: matrix cores on tiles that the block's waves share ------------------------------------------------------
// A wave holds 32 query rows (their columns as operands in 32 registers, and their outputs in 64) and takes steps of 32 keys:
//   S^T[key, query] = K Q^T      v_mfma_f32_32x32x16_bf16, A = 16 bytes of a key row, B = the queries
//   weights                      a lane has 16 of the 32 keys of ONE query, so the sum and the rescaling of its outputs are the
//                                lane's own
//   O^T[column, query] += V^T P^T    B = the weights as they come out of the first product: the order of the keys in a
//                                product is free, so A takes the same one, rows read column-wise by the transposing LDS load
// K and V tiles of KT keys go through LDS once for the block's waves, WQ of which hold different queries and WK = WAVES / WQ
// different keys of the tile; the next tile is loaded into registers while this one is used.  16-byte chunks are stored at
// places exchanged by the row's number, so that neither the key rows (stride 256 bytes) nor the four rows of a transposing
// load meet in a bank (no conflict is counted).  Eight waves of 32 queries keep two on a SIMD, whose products and
// exponentials overlap: four waves of 64 queries, each with the registers of a SIMD to itself, take 130 us where these take 113.
// The weights enter the second product in two bf16 terms, as in the library's other attention over whole caches, and their sum in 32
// bits: 2^-16 of each weight.  One term makes that product half as long, but is off by up to 2^-8 of each weight, which
// outputs whose large rows cancel do not hide: then whole outputs are wrong by their own size (tests/test_gpu_weight_precision.py).
// us in one / two terms, without rows of their own: 4 sequences of 32/8 heads behind 65536 rows 52.3 / 52.9, 16 of them 55.8 / 56.6, 32
// 63.6 / 70.2, 64 of 64/8 behind 4096 29.9 / 33.2, 32768 84.6 / 104.2.
// The reference of the exponentials follows the running maximum only when a step's weights sum up to more than 2^8: the
// outputs are rescaled a few times per run instead of in most steps, weights up to 2^8 lose nothing, and neither the
// maximum nor an exchange between lanes is needed in the other steps.
// Measured: 64 sequences of 64/8 heads behind P rows, 12 us + 2.9 us per 1024 rows (0.74 PFLOP/s of the attention, 1.1 of products
// with the second term; a large product reaches 1.2 on this card): the constant part is a launch, the queries, 528 bytes per query
// row and run written, and their merge.  In one term, of the 46 us of 24576 such rows, the products alone, on operands that do not
// change, took 20, with the LDS reads 38, with the exponentials but no reads 42; halves of the waves a phase apart by barriers,
// one in products while the other is in exponentials, took 48; priorities for one half or for the products changed 1 %.
typedef float pf_f32x16_t __attribute__((ext_vector_type(16)));
typedef short pf_s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) pf_s16x4_t pf_lds_s16x4_t;

template <int WAVES, int WQ>
constexpr int pf_tile_keys() {
  return WAVES / WQ == 4 ? 128 : 64;
}

// LDS: two pairs of tiles; at the end, where waves have other keys of the same queries, what half of them hand over.
template <int WAVES, int WQ>
constexpr int pf_lds_bytes() {
  const int tiles = 4 * pf_tile_keys<WAVES, WQ>() * 256, merge = WQ == WAVES ? 0 : WAVES * 32 * 8 + WAVES / 2 * 64 * 256;
  return tiles > merge ? tiles : merge;
}

template <int WAVES, int WQ>
__device__ __forceinline__ void prefix_mfma_body(char* smem /* [2][K tile, V tile] */, const PrefixAt& block,
                                                 const uint16_t* __restrict__ qv, const PrefixArgs& a) {
  constexpr int kThreads = 64 * WAVES, WK = WAVES / WQ, KT = pf_tile_keys<WAVES, WQ>(), kSteps = KT / (32 * WK), kChunks = KT * 16 / kThreads;
  constexpr int kTileBytes = KT * 256;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, half = lane >> 5, l16 = lane & 15;
  const int wq = wave % WQ, wk = wave / WQ;
  const int h = block.h, q0 = (block.tile * WQ + wq) * 32;
  const int r0 = block.split * a.run, r1 = min(a.rows, r0 + a.run);
  const int tiles = (r1 - r0 + KT - 1) / KT;

  am_bf16x8_t q[8];
  {
    const uint16_t* src = qv + prefix_head(min(q0 + l32, a.M - 1), h, a.G, a.Hq) * kD + 8 * half;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) q[ks] = __builtin_bit_cast(am_bf16x8_t, load16(src + 16 * ks));
  }
  const uint16_t* kh = static_cast<const uint16_t*>(a.k) + (size_t)h * a.cap * kD;
  const uint16_t* vh = static_cast<const uint16_t*>(a.v) + (size_t)h * a.cap * kD;

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

  float m = kNegBig, l = 0.f;
  pf_f32x16_t o[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) o[c] = pf_f32x16_t{};
  const int k_at = l32 * 256 + ((half ^ l16) * 16);
  const int v_row = 4 * half + (l16 >> 2);
  const int v_at = kTileBytes + v_row * 256 + (((((lane >> 4) & 1) * 2 + ((l16 & 3) >> 1)) ^ ((v_row & 3) << 2)) * 16) + (l16 & 1) * 8;

  // one step: 32 keys of the tile in buffer `base`; ENDS: only the first `there` exist
  auto step = [&](const char* base, int there, auto ends) __attribute__((always_inline)) {
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
    pf_f32x16_t s = pf_f32x16_t{};
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[ks], q[ks], s, 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (decltype(ends)::value) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (8 * (i >> 2) + 4 * half + (i & 3) >= there) s[i] = kNegBig;
    }
    float p[16], sum;
    auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] = fast_exp2(fmaf(s[i], kSoftmaxScaleLog2, -m));
      float odd = p[1];
      sum = p[0];
#pragma unroll
      for (int i = 2; i < 16; i += 2) {
        sum += p[i];
        odd += p[i + 1];
      }
      sum += odd;
    };
    weights();
    if (__ballot(!(sum <= kPfGrowth)) != 0ull) {
      float top = s[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
      top = fmaxf(top, __shfl_xor(top, 32)) * kSoftmaxScaleLog2;
      const float mn = fmaxf(m, top), corr = fast_exp2(m - mn);
      m = mn;
      l *= corr;
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[c][i] *= corr;
      weights();
    }
    l += sum;
    uint32_t w[2][8];  // the weights' two terms
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[0][i] = BF16::round2(p[2 * i], p[2 * i + 1]);
      w[1][i] = BF16::round2(p[2 * i] - __uint_as_float(w[0][i] << 16), p[2 * i + 1] - __uint_as_float(w[0][i] & 0xffff0000u));
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int c = 0; c < 4; ++c)
          o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              va[ks][c], __builtin_bit_cast(am_bf16x8_t, make_uint4(w[t][4 * ks], w[t][4 * ks + 1], w[t][4 * ks + 2], w[t][4 * ks + 3])), o[c], 0, 0, 0);
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
  l += __shfl_xor(l, 32);
  if constexpr (WK > 1) {
    float2* ml = reinterpret_cast<float2*>(smem);                       // [wave][32] (max, sum)
    float4* ob = reinterpret_cast<float4*>(smem + WAVES * 32 * 8);      // [wave of the upper half][4][4][lane]
    if (half == 0) ml[wave * 32 + l32] = make_float2(m, l);
    __syncthreads();
    float mn = kNegBig, ls = 0.f;
#pragma unroll
    for (int w = 0; w < WK; ++w) mn = fmaxf(mn, ml[(w * WQ + wq) * 32 + l32].x);
#pragma unroll
    for (int w = 0; w < WK; ++w) {
      const float2 x = ml[(w * WQ + wq) * 32 + l32];
      ls = fmaf(x.y, fast_exp2(x.x - mn), ls);
    }
    const float f = fast_exp2(m - mn);
    m = mn;
    l = ls;
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[c][i] *= f;
#pragma unroll
    for (int n = WK / 2; n >= 1; n /= 2) {
      if (wk >= n && wk < 2 * n) {
        float4* dst = ob + ((wk - n) * WQ + wq) * 16 * 64;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            dst[(c * 4 + i) * 64 + lane] = make_float4(o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]);
      }
      __syncthreads();
      if (wk < n) {
        const float4* src = ob + (wk * WQ + wq) * 16 * 64;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 x = src[(c * 4 + i) * 64 + lane];
            o[c][4 * i] += x.x;
            o[c][4 * i + 1] += x.y;
            o[c][4 * i + 2] += x.z;
            o[c][4 * i + 3] += x.w;
          }
      }
      __syncthreads();
    }
    if (wk != 0) return;
  }
  // a lane has four columns of one query at a time: through LDS, so that a store takes four half rows
  char* mine = smem + wave * 8192;  // [32 queries][64 columns], 16-byte chunks exchanged as the keys'
#pragma unroll
  for (int pass = 0; pass < 2; ++pass) {
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const pf_f32x16_t& x = o[2 * pass + c];
        *reinterpret_cast<float4*>(mine + l32 * 256 + (((8 * c + 2 * i + half) ^ l16) * 16)) = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
      }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int row = 4 * j + (lane >> 4), r = q0 + row;
      const float4 x = *reinterpret_cast<const float4*>(mine + row * 256 + ((l16 ^ (row & 15)) * 16));
      if (r < a.M) *reinterpret_cast<float4*>(a.partial + (prefix_head(r, h, a.G, a.Hq) * a.splits + block.split) * kPartStride + 64 * pass + 4 * l16) = x;
    }
    __builtin_amdgcn_wave_barrier();
  }
  const int r = q0 + l32;
  if (half == 0 && r < a.M)
    *reinterpret_cast<float2*>(a.partial + (prefix_head(r, h, a.G, a.Hq) * a.splits + block.split) * kPartStride + kD) = make_float2(m, l);
}

// ---- the launch -----------------------------------------------------------------------------------------------
// The sequences' own rows: q, their parts and how they are dealt out.
struct OwnArgs {
  const void *k, *v;
  float* partial;
  int B, Hkv, S_cap, S_max, nsplit;
  Ragged rg;
};

// Blocks [0, splits tiles Hkv): the prefix; behind them X = nsplit B blocks for every KV head.  (Neighbours in the grid are
// runs of the prefix, so the tiles of a run, which read the same rows, go to one XCD where the runs are a multiple of 8.)
// KIND: bf16: WQ; fp32: -QG.  (KIND 1: its 128 KB of LDS leave a CU one block of four waves, so each may have all registers of its SIMD.)
template <typename T, int NH, int WAVES, int KIND>
__global__ __launch_bounds__(64 * WAVES, KIND == -1 ? 3 : KIND == 1 ? 1 : 2) void shared_kernel(const void* __restrict__ q, PrefixArgs pa, OwnArgs oa) {
  extern __shared__ __align__(16) char smem[];
  const int prefix_blocks = pa.splits * pa.tiles * oa.Hkv;
  if ((int)blockIdx.x < prefix_blocks) {
    const int id = blockIdx.x, rest = id / pa.splits;
    const PrefixAt block{id - rest * pa.splits, rest % pa.tiles, rest / pa.tiles};
    if constexpr (T::EPC == 8)
      prefix_mfma_body<WAVES, KIND>(smem, block, static_cast<const uint16_t*>(q), pa);
    else
      prefix_f32_body<-KIND>(smem, block, static_cast<const float*>(q), pa);
    return;
  }
  const int X = oa.nsplit * oa.B, id = (int)blockIdx.x - prefix_blocks, x = id / oa.Hkv, h = id - x * oa.Hkv;
  const Dealt d = deal_runs(oa.rg, oa.B, oa.S_max, oa.nsplit);
  const RunAt at = find_run(oa.rg, oa.B, oa.S_max, d.run, x);
  if (at.b >= oa.B) return;  // uniform for the block
  const int form_now = oa.rg.loads.form == kByLengths ? form_of(oa.rg.loads, {d.total, 0.f}) : oa.rg.loads.form;
  auto& s_merge = *reinterpret_cast<PartsSmem<T, NH, WAVES>*>(smem);
  with_form<kPastCaches>(form_now, [&](auto form) __attribute__((always_inline)) {
    parts_body<T, NH, false, decltype(form)::value != kThroughCaches, WAVES>(s_merge, nullptr, at, d.run, h, X, oa.k, oa.v, q, oa.partial,
                                                                             nullptr, 0, oa.Hkv, oa.S_cap);
  });
}

// The block's queries and tiles for M query rows: as few blocks of queries as possible, and waves on different keys where
// they do not fill them.
struct PrefixShape {
  int queries, keys;  // of a block; keys: what a run is a multiple of
};
static PrefixShape prefix_shape(const Shape& s) {
  const int M = s.B * s.G;
  if (s.dtype == 0) return M <= 16 ? PrefixShape{16, 64} : PrefixShape{32, 64};
  if (M <= 32) return {32, 128};
  if (M <= 64) return {64, 128};
  if (M <= 128) return {128, 64};
  return {256, 64};
}

static int prefix_tiles(const Shape& s) {
  const int nq = prefix_shape(s).queries;
  return (s.B * s.G + nq - 1) / nq;
}

// Runs of the prefix at most: a block for every CU, also where more would fit: more runs mean more parts to write and to merge.  us with
// one, two and three or four per CU, fp32: 5 sequences of 16/8 heads behind 5777 rows 16.0, 16.9, 19.0, behind 20000 37.3, 38.3,
// 39.7; 64 of 64/8 behind 6000 124, 150.
static int prefix_most(const Shape& s) {
  const int n = device_cus() / (s.Hkv * prefix_tiles(s));
  return n < 1 ? 1 : n;
}

// Rows of a run at least: 256 from 600 heads of the batch on, whose parts weigh more than their products.  bf16, us with runs as they
// come / of 256 / of 384, behind 1000, 2000 and 4000 rows with a few of their own: 640 heads 14.1 / 15.5 / 17.3, 20.1 / 16.2 / 18.2, 21.2 /
// 17.2 / 18.9; 1024 16.1 / 16.4 / 18.4, 21.6 / 17.5 / 19.4, 22.5 / 18.3 / 20.1; 1536 18.5 / 21.1 / 24.4, 25.6 / 22.2 / 26.0, 25.5 /
// 22.4 / 25.9; 4096 41.9 / 43.2 / 47.3, 44.7 / 45.3 / 48.7, 50.1 / 50.2 / 51.0; 256 heads behind 2048 rows 12.2 / 11.9 / 12.2.
static int prefix_least(const Shape& s) {
  const int least = s.dtype == 0 || s.B * s.Hq < 600 ? 1 : 256, keys = prefix_shape(s).keys;
  return (least + keys - 1) / keys * keys;
}

static int prefix_run(const Shape& s, int rows) {
  const int n = prefix_most(s), least = prefix_least(s), keys = prefix_shape(s).keys;
  int run = (rows + n - 1) / n;
  if (run < least) run = least;
  return (run + keys - 1) / keys * keys;
}

int prefix_splits(const Shape& s, int prefix_rows) {
  if (prefix_rows < 1) return 0;
  const int run = prefix_run(s, prefix_rows);
  return (prefix_rows + run - 1) / run;
}

int prefix_splits_at_most(const Shape& s, int prefix_rows) {
  if (prefix_rows < 1) return 0;
  const int n = prefix_most(s), least = prefix_least(s), whole = (prefix_rows + least - 1) / least;
  return whole < n ? whole : n;
}

// One launch for the prefix and the sequences' own rows while the latter are few: a launch less, but their blocks then have
// the registers and LDS of the prefix's and eight waves fill a CU.  us in one / in two launches: 3 sequences of 32/8 heads behind
// 700 rows with 30 of their own 10.4 / 15.4, 8 behind 2048 with 300 (10 MB) 14.2 / 18.6; 8 of 32/16 heads behind 4096 with 500
// (33 MB) 23.5 / 22.0, 32 of 32/8 with 1500 (197 MB) 44.5 / 41.3, 16 of 32/32 with 2048 (537 MB) 99.6 / 76.6.
constexpr double kOneLaunchBytes = 24e6;
static double own_bytes(const Shape& s, int rows) { return (double)s.B * s.Hkv * rows * (2 * kD * s.elem_bytes); }
static bool in_one_launch(const Shape& s) { return own_bytes(s, s.S) < kOneLaunchBytes; }

// Runs of a sequence's own rows in that one launch: 64 rows for every wave in bf16, 32 in fp32 (with 32 and 64, 8 sequences of 32/8 bf16
// heads with 300 rows behind 2048 14.0 and 11.8 us, 5 of 16/8 fp32 heads with 131 behind 5777 16.1 and 17.1).
static int one_launch_splits(const Shape& s, int own_rows) {
  const int units = s.B * s.Hkv, waves = s.dtype == 0 || prefix_shape(s).queries == 32 ? 4 : 8;
  int n = ((s.dtype == 0 ? 8 : 24 / waves) * device_cus() + units - 1) / units;
  const int rows = (s.dtype == 0 ? 32 : 64) * waves, most = (own_rows + rows - 1) / rows;
  if (n > most) n = most;
  return n < 1 ? 1 : n;
}

int shared_own_splits(const Shape& s) {
  if (s.S < 1) return 0;
  return in_one_launch(s) ? one_launch_splits(s, s.S) : weigh_splits(s);
}

int shared_own_splits_at_most(const Shape& s) {
  if (s.S < 1) return 0;
  if (in_one_launch(s)) return one_launch_splits(s, s.S);
  // the longest rows of one launch, or one more
  const int apart = weigh_splits(s), together = one_launch_splits(s, (int)(kOneLaunchBytes / own_bytes(s, 1)) + 1);
  return apart > together ? apart : together;
}

template <typename T, int NH, int WAVES, int KIND>
static hipError_t launch_shared_k(const Shape& s, const void* q, const PrefixArgs& pa, const OwnArgs& oa, hipStream_t st) {
  static std::atomic<unsigned long long> raised{0};
  int bytes = (int)sizeof(PartsSmem<T, NH, WAVES>);
  if constexpr (T::EPC == 8)
    bytes = max(bytes, pf_lds_bytes<WAVES, KIND>());
  else
    bytes = max(bytes, (int)sizeof(AttendF32Smem<-KIND, kPfWaves>));
  const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(&shared_kernel<T, NH, WAVES, KIND>), bytes, raised);
  if (e != hipSuccess) return e;
  const int blocks = pa.splits * pa.tiles * s.Hkv + oa.nsplit * s.B * s.Hkv;
  if (blocks < 1) return hipSuccess;  // no rows at all
  hipLaunchKernelGGL((shared_kernel<T, NH, WAVES, KIND>), dim3(blocks), dim3(64 * WAVES), bytes, st, q, pa, oa);
  return hipGetLastError();
}

template <int NH>
static hipError_t launch_shared_nh(const Shape& s, const void* q, const PrefixArgs& pa, const OwnArgs& oa, hipStream_t st) {
  const int nq = prefix_shape(s).queries;
  if (s.dtype == 0) {
    if (nq == 16) return launch_shared_k<F32, NH, 4, -1>(s, q, pa, oa, st);
    return launch_shared_k<F32, NH, 4, -2>(s, q, pa, oa, st);
  }
  if (nq == 32) return launch_shared_k<BF16, NH, 4, 1>(s, q, pa, oa, st);
  if (nq == 64) return launch_shared_k<BF16, NH, 8, 2>(s, q, pa, oa, st);
  if (nq == 128) return launch_shared_k<BF16, NH, 8, 4>(s, q, pa, oa, st);
  return launch_shared_k<BF16, NH, 8, 8>(s, q, pa, oa, st);
}

hipError_t launch_shared(const Shape& s, int splits, int nsplit, const void* q, const void* k_prefix, const void* v_prefix, int rows,
                         int cap, const void* k, const void* v, float* prefix, float* partial, hipStream_t st) {
  const PrefixArgs pa{k_prefix, v_prefix, prefix, s.B * s.G, s.G, s.Hq, rows, cap, splits > 0 ? prefix_run(s, rows) : 0, splits, splits > 0 ? prefix_tiles(s) : 0};
  const bool apart = nsplit > 0 && !in_one_launch(s);
  if (apart) {
    const hipError_t e = launch_parts(s, nsplit, q, k, v, partial, nullptr, st);
    if (e != hipSuccess || splits == 0) return e;
  }
  const OwnArgs oa{k, v, partial, s.B, s.Hkv, s.S_cap, s.S, apart ? 0 : nsplit, with_loads(s, kEveryRow)};
  switch (s.G) {
    case 1: return launch_shared_nh<1>(s, q, pa, oa, st);
    case 2: return launch_shared_nh<2>(s, q, pa, oa, st);
    case 4: return launch_shared_nh<4>(s, q, pa, oa, st);
    case 8: return launch_shared_nh<8>(s, q, pa, oa, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace loki
