// Eviction from a cache by accumulated attention weight: of every (sequence, KV head) the first `sinks` rows,
// the newest `recent` ones and between them those with the largest totals go on, `budget` rows in all, in
// their order; equal totals keep the lowest row.
//
// Two launches.  (1) evict_select_kernel, one block per unit: the totals as order-preserving integers in
// registers, the smallest one kept found by three radix passes over LDS histograms, the list written in
// ascending order.  Latency bounds it: a pass is a few barriers.  (2) evict_copy_kernel or evict_compact_kernel: the
// listed rows to their new places, bound by memory; a row is read once and written once.  In place row j comes from
// list[j] >= j: a block owns a slice of the unit's columns, walks the list upwards and writes a run of rows only when
// all of its sources have been read; the sources of later runs lie behind it.
//
// us into another cache / in place, contiguous and paged, bf16: 16 sequences of 8 heads, 16384 rows down to 2048 (280 MB) 62.5 / 79.1, 71.8 /
// 89.4, 2048 down to 1920 (256 MB) 49.6 / 58.2, 57.8 / 72.0; one of 8 heads, 16384 down to 2048 18.0 / 27.1, 20.1 / 38.4, 1024 down to 960 10.0 /
// 11.2, 10.9 / 15.1, 100000 down to 8192 111 / 157, 112 / 208: a unit's selection and, in place, its slices are few blocks there.
#include "common.h"

namespace loki {

constexpr int kEvThreads = 1024;
constexpr int kEvWaves = kEvThreads / 64;
constexpr int kEvBins = 2048;  // 11-bit digits: 32 bits in three passes of 11, 11 and 10

__device__ __forceinline__ int evict_rows(const int32_t* seq_lens, int b, int S_max) {
  return seq_lens == nullptr ? S_max : min(max(seq_lens[b], 0), S_max);
}

// A row as the selection sees it: kForced goes on whatever happens, kNoRow is none (or one whose total does not count).
constexpr uint32_t kNoRow = 0u, kForced = 0xffffffffu;
constexpr uint32_t kZeroTotal = 0x80000000u;  // float_to_key(0)

// What the waves before this one hold, of s_wave[wave].
__device__ __forceinline__ uint32_t before_wave(const uint32_t* s_wave, int wave) {
  const int lane = threadIdx.x & 63;
  const uint32_t x = lane < kEvWaves ? s_wave[lane] : 0u;
  const uint32_t incl = wave_inclusive_scan_u32(x);
  return (uint32_t)(__builtin_amdgcn_readlane((int)incl, wave) - __builtin_amdgcn_readlane((int)x, wave));
}

// NK: keys per lane held in registers (rows up to 1024 NK); 0: read again in every pass.
template <int NK>
__global__ __launch_bounds__(kEvThreads) void evict_select_kernel(EvictArgs a, int32_t* __restrict__ list /* [units, list_pitch] */,
                                                                  int32_t* __restrict__ kept_rows /* [units] */) {
  __shared__ uint32_t s_hist[kEvBins];
  __shared__ uint32_t s_wave[2][kEvWaves];
  __shared__ uint32_t s_pick[3];
  const int unit = blockIdx.x, b = unit / a.Hkv;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int len = evict_rows(a.seq_lens, b, a.S_max), kept = min(len, a.budget);
  int32_t* out = list + (size_t)unit * a.list_pitch;
  if (tid == 0) kept_rows[unit] = kept;
  for (int i = kept + tid; i < a.list_pitch; i += kEvThreads) out[i] = -1;
  if (len <= a.budget) {  // (uniform for the block)
    for (int i = tid; i < len; i += kEvThreads) out[i] = i;
    return;
  }
  const int c0 = a.sinks, c1 = len - a.recent;  // rows whose totals decide: more than are needed, as len > budget
  const uint32_t need = (uint32_t)(a.budget - a.sinks - a.recent);

  // wave w holds rows [w seg, (w + 1) seg), lane by lane in rounds of 64
  const int rounds = (len + kEvThreads - 1) / kEvThreads, first = wave * rounds * 64 + lane;
  const float* w = a.weights + (size_t)unit * a.S_cap;
  // (no branch around the loads: each would be waited for by itself)
  auto load = [&](int i) -> float { return w[min(first + 64 * i, len - 1)]; };
  auto key_of = [&](int i, float x) -> uint32_t {
    const int row = first + 64 * i;
    const uint32_t key = min(max(float_to_key(x), 1u), kForced - 1u);
    return row >= len ? kNoRow : row >= c0 && row < c1 ? key : kForced;
  };
  uint32_t reg[NK > 0 ? NK : 1];
  if constexpr (NK > 0) {
    float x[NK];
#pragma unroll
    for (int i = 0; i < NK; ++i) x[i] = load(i);
#pragma unroll
    for (int i = 0; i < NK; ++i) reg[i] = key_of(i, x[i]);
  }
  auto each = [&](auto f) __attribute__((always_inline)) {  // f(round, key), in ascending order of the wave's rows
    if constexpr (NK > 0) {
#pragma unroll
      for (int i = 0; i < NK; ++i)
        if (i < rounds) f(i, reg[i]);
    } else {
      constexpr int U = 16;
      for (int i0 = 0; i0 < rounds; i0 += U) {
        float x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = load(i0 + u);
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (i0 + u < rounds) f(i0 + u, key_of(i0 + u, x[u]));
      }
    }
  };

  // The need-th largest key, digit by digit.  Rows of total zero, of which a cache can hold many, are counted by
  // ballots, once: as atomics they would queue at one bin.
  uint32_t last = kForced - 1u, equal_kept = 0u;  // kept: keys above `last`, and the first equal_kept of those equal to it
  bool all_equal = true;                          // (which are all of them)
  if (need > 0u) {
    uint32_t prefix = 0u, left = need, zeros = 0u;  // left: how many of the keys that begin with `prefix` are kept
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
      const uint32_t mask = pass == 2 ? 0x3ffu : 0x7ffu;
      s_hist[tid] = 0u;
      s_hist[tid + kEvThreads] = 0u;
      __syncthreads();
      each([&](int, uint32_t key) {
        if (pass == 0) {
          zeros += (uint32_t)__popcll(__ballot(key == kZeroTotal));
          if (key - 1u < kForced - 1u && key != kZeroTotal) atomicAdd(&s_hist[key >> 21], 1u);
        } else if ((key >> (pass == 1 ? 21 : 10)) == prefix && key != kForced && key != kZeroTotal) {
          atomicAdd(&s_hist[(key >> shift) & mask], 1u);
        }
      });
      if (lane == 0 && zeros != 0u && (pass == 0 || (kZeroTotal >> (pass == 1 ? 21 : 10)) == prefix))
        atomicAdd(&s_hist[(kZeroTotal >> shift) & mask], zeros);
      __syncthreads();
      // thread t owns the bins 2047 - 2 t and 2046 - 2 t: the keys of a larger bin come before them
      const int hi = kEvBins - 1 - 2 * tid;
      const uint2 n = *reinterpret_cast<const uint2*>(&s_hist[hi - 1]);  // (x: the lower bin)
      const uint32_t incl = wave_inclusive_scan_u32(n.x + n.y);
      if (lane == 63) s_wave[pass & 1][wave] = incl;
      __syncthreads();
      const uint32_t before = before_wave(s_wave[pass & 1], wave) + incl - (n.x + n.y);
      if (before < left && left <= before + n.x + n.y) {
        const bool upper = left <= before + n.y;
        s_pick[0] = (uint32_t)(upper ? hi : hi - 1);
        s_pick[1] = left - before - (upper ? 0u : n.y);
        s_pick[2] = upper ? n.y : n.x;
      }
      __syncthreads();
      prefix = pass == 0 ? s_pick[0] : pass == 1 ? (prefix << 11) | s_pick[0] : (prefix << 10) | s_pick[0];
      left = s_pick[1];
    }
    last = prefix;
    equal_kept = left;
    all_equal = s_pick[2] == left;
  }

  // (totals that change while they are read again, as those of more rows than registers hold are, cannot leave the list:
  // its places are checked below, and its rows where they are moved)
  // kept rows of every wave's segment, then each wave writes its part of the list; equal keys that do not all stay are
  // counted too
  if (all_equal && need > 0u) --last;  // (a key is at least 1) all of them are above it then
  uint32_t n_sure = 0, n_equal = 0;
  each([&](int, uint32_t key) { n_sure += (uint32_t)__popcll(__ballot(key > last)); });
  if (!all_equal) each([&](int, uint32_t key) { n_equal += (uint32_t)__popcll(__ballot(key == last)); });
  __syncthreads();
  if (lane == 0) {
    s_wave[0][wave] = n_sure;
    s_wave[1][wave] = n_equal;
  }
  __syncthreads();
  uint32_t at = before_wave(s_wave[0], wave);
  if (all_equal) {
    each([&](int i, uint32_t key) {
      const unsigned long long m = __ballot(key > last);
      const uint32_t to = at + __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u));
      if (key > last && to < (uint32_t)kept) out[to] = first + 64 * i;
      at += (uint32_t)__popcll(m);
    });
    return;
  }
  uint32_t eq = before_wave(s_wave[1], wave);  // equal keys before this wave's segment; as many of them stay as there is room for
  at += min(eq, equal_kept);
  const unsigned long long below = (1ull << lane) - 1ull;
  each([&](int i, uint32_t key) {
    const unsigned long long m_equal = __ballot(key == last);
    const bool keep = key > last || (key == last && eq + (uint32_t)__popcll(m_equal & below) < equal_kept);
    const unsigned long long m = __ballot(keep);
    const uint32_t to = at + (uint32_t)__popcll(m & below);
    if (keep && to < (uint32_t)kept) out[to] = first + 64 * i;
    at += (uint32_t)__popcll(m);
    eq += (uint32_t)__popcll(m_equal);
  });
}

// One 16-byte chunk of a row: c < nk: chunk c of the key row (the first nlo in klo, the rest in khi), else of the value row.
struct EvictSide {
  char *klo, *khi, *v;
  int S_cap;
};
__device__ __forceinline__ char* evict_chunk(const EvictSide& x, long long row, int c, int nk, int nlo) {
  if (c >= nk) return x.v + (row * nk + (c - nk)) * 16;
  return c < nlo ? x.klo + (row * nlo + c) * 16 : x.khi + (row * (nk - nlo) + (c - nlo)) * 16;
}

constexpr int kMvThreads = 256;
constexpr int kMvInFlight = 8;
constexpr int kBothPast = 2;  // (kThroughCaches 0, kPastCaches 1: the loads)

// Into another cache: a block takes `rows` list entries of one unit (behind the kept ones the list holds -1).
// FORM: kThroughCaches, loads past the caches, loads and stores past them (launch_evict_move).
template <int CHUNKS, int FORM>  // CHUNKS: of 16 bytes, of a key and a value row together
__global__ __launch_bounds__(kMvThreads) void evict_copy_kernel(EvictArgs a, const int32_t* __restrict__ list,
                                                                const int32_t* __restrict__ kept_rows, int rows) {
  const int unit = blockIdx.y, b = unit / a.Hkv, h = unit - b * a.Hkv, tid = threadIdx.x;
  const int j0 = blockIdx.x * rows, j1 = min(min(a.budget, a.S_max), j0 + rows);
  if (blockIdx.x == 0 && h == 0 && tid == 0 && a.lens_out != nullptr) a.lens_out[b] = kept_rows[unit];
  const int32_t* from = list + (size_t)unit * a.list_pitch;
  if (from[j0] < 0) return;  // uniform for the block
  const EvictSide src{(char*)a.klo, (char*)a.khi, (char*)a.v, a.S_cap};
  const EvictSide dst{(char*)a.klo_out, (char*)a.khi_out, (char*)a.v_out, a.S_cap_out};
  const long long out0 = (long long)unit * a.S_cap_out;
  const int items = (j1 - j0) * CHUNKS;
  for (int i0 = tid; i0 < items; i0 += kMvThreads * kMvInFlight) {
    int at[kMvInFlight];
    uint4 x[kMvInFlight];
#pragma unroll
    for (int u = 0; u < kMvInFlight; ++u) at[u] = from[j0 + min(i0 + u * kMvThreads, items - 1) / CHUNKS];
#pragma unroll
    for (int u = 0; u < kMvInFlight; ++u)
      x[u] = load16_hint<FORM != kThroughCaches>(
          evict_chunk(src, cache_row(a.pg, b, h, a.Hkv, a.S_cap, min(max(at[u], 0), a.S_max - 1)), (i0 + u * kMvThreads) % CHUNKS, CHUNKS / 2, a.nlo));
#pragma unroll
    for (int u = 0; u < kMvInFlight; ++u) {
      const int i = i0 + u * kMvThreads;
      if (i < items && at[u] >= 0) store16_hint<FORM == kBothPast>(evict_chunk(dst, out0 + j0 + i / CHUNKS, i % CHUNKS, CHUNKS / 2, a.nlo), x[u]);
    }
  }
  if (a.weights_out != nullptr)
    for (int j = j0 + tid; j < j1 && from[j] >= 0; j += kMvThreads)
      a.weights_out[out0 + j] = a.weights[(size_t)unit * a.S_cap + min(from[j], a.S_max - 1)];
}

// Every source of a run has been read, by all waves, before one of its rows is overwritten.
__device__ __forceinline__ void evict_all_read() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

constexpr int kIpThreads = 512;
constexpr int kIpSlice = 8;  // chunks of a slice: a 128-byte line
constexpr int kIpRows = kIpThreads / kIpSlice;

// In place: a block takes one slice of the unit's columns; the block behind the last slice moves the totals.
__global__ __launch_bounds__(kIpThreads) void evict_compact_kernel(EvictArgs a, const int32_t* __restrict__ list,
                                                                   const int32_t* __restrict__ kept_rows, int chunks) {
  const int unit = blockIdx.y, b = unit / a.Hkv, h = unit - b * a.Hkv, tid = threadIdx.x;
  const int kept = kept_rows[unit];
  const int slices = chunks / kIpSlice;
  const int32_t* from = list + (size_t)unit * a.list_pitch;
  if ((int)blockIdx.x == slices) {
    if (h == 0 && tid == 0 && a.lens_out != nullptr) a.lens_out[b] = kept;
    float* w = a.weights + (size_t)unit * a.S_cap;
    for (int j0 = 0; j0 < kept; j0 += kIpThreads * 4) {  // (uniform)
      float x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int j = j0 + u * kIpThreads + tid;
        x[u] = w[min(max(from[min(j, kept - 1)], 0), a.S_max - 1)];
      }
      evict_all_read();
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int j = j0 + u * kIpThreads + tid;
        if (j < kept) w[j] = x[u];
      }
    }
    return;
  }
  const EvictSide x{(char*)a.klo, (char*)a.khi, (char*)a.v, a.S_cap};
  const int c = (int)blockIdx.x * kIpSlice + tid % kIpSlice, r = tid / kIpSlice;
  const int nk = chunks / 2;
  constexpr int U = kMvInFlight;
  for (int j0 = 0; j0 < kept; j0 += kIpRows * U) {  // (uniform)
    uint4 y[U];
    int at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u * kIpRows + r;
      at[u] = from[min(j, kept - 1)];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u * kIpRows + r;
      at[u] = j < kept ? min(max(at[u], 0), a.S_max - 1) : j;
      if (at[u] != j) y[u] = load16(evict_chunk(x, cache_row(a.pg, b, h, a.Hkv, a.S_cap, at[u]), c, nk, a.nlo));
    }
    evict_all_read();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u * kIpRows + r;
      if (at[u] != j) *reinterpret_cast<uint4*>(evict_chunk(x, cache_row(a.pg, b, h, a.Hkv, a.S_cap, j), c, nk, a.nlo)) = y[u];
    }
  }
}

hipError_t launch_evict_select(const Shape& s, const EvictArgs& a, int32_t* list, int32_t* kept, hipStream_t st) {
  const dim3 grid(s.B * s.Hkv), block(kEvThreads);
  if (a.S_max <= 4 * kEvThreads)
    hipLaunchKernelGGL((evict_select_kernel<4>), grid, block, 0, st, a, list, kept);
  else if (a.S_max <= 16 * kEvThreads)
    hipLaunchKernelGGL((evict_select_kernel<16>), grid, block, 0, st, a, list, kept);
  else if (a.S_max <= 48 * kEvThreads)
    hipLaunchKernelGGL((evict_select_kernel<48>), grid, block, 0, st, a, list, kept);
  else
    hipLaunchKernelGGL((evict_select_kernel<0>), grid, block, 0, st, a, list, kept);
  return hipGetLastError();
}

hipError_t launch_evict_move(const Shape& s, const EvictArgs& a, const int32_t* list, const int32_t* kept, hipStream_t st) {
  const int units = s.B * s.Hkv, chunks = 2 * kD * s.elem_bytes / 16;
  if (a.klo_out == nullptr) {
    hipLaunchKernelGGL(evict_compact_kernel, dim3(chunks / kIpSlice + 1, units), dim3(kIpThreads), 0, st, a, list, kept, chunks);
    return hipGetLastError();
  }
  const int rows = kMvThreads * kMvInFlight / chunks;
  const int most = a.budget < a.S_max ? a.budget : a.S_max;
  const dim3 grid((most + rows - 1) / rows, units), block(kMvThreads);
  // By the bytes that go on: rows read once, from 48 MB past the caches, from 120 MB written past them too.  us through /
  // loads / both past: 34 MB 21.8 / 23.0 / 22.5, 67 39.4 / 33.5 / 35.2, 92 52.4 / 44.8 / 46.8, 134 72.2 / 68.6 / 64.1.
  const double moved = (double)units * most * 16 * chunks;
  const int form = moved < 48e6 ? kThroughCaches : moved < 120e6 ? kPastCaches : kBothPast;
#define LOKI_EVICT_COPY(C)                                                                                            \
  if (form == kThroughCaches)                                                                                         \
    hipLaunchKernelGGL((evict_copy_kernel<C, kThroughCaches>), grid, block, 0, st, a, list, kept, rows);              \
  else if (form == kPastCaches)                                                                                       \
    hipLaunchKernelGGL((evict_copy_kernel<C, kPastCaches>), grid, block, 0, st, a, list, kept, rows);                 \
  else                                                                                                                \
    hipLaunchKernelGGL((evict_copy_kernel<C, kBothPast>), grid, block, 0, st, a, list, kept, rows)
  if (s.dtype == 0) {
    LOKI_EVICT_COPY(64);
  } else {
    LOKI_EVICT_COPY(32);
  }
#undef LOKI_EVICT_COPY
  return hipGetLastError();
}

}  // namespace loki
