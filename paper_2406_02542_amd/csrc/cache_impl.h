// A cache held whole, contiguous or on pages, in the storage type or in 4 bits: where its rows lie, and the 4-bit form.
//
// 4 bits: a row is four groups of 32 columns.  With lowest = fp16(min) and step = fp16((max - min) * (1 / 15)) of a group, the code of x is
// (x - lowest) / step rounded to nearest (ties to even) within 0 .. 15, 0 where step is 0, and stands for lowest + code * step.  Word m of
// a row's 16 holds columns 2 m and 2 m + 1 of every group, that of group g in bits 4 g .. and 16 + 4 g ..: one shift and one bit
// select turn a word into a register of two matrix-core operands, neighbours of one group, with the same four for all groups.
#pragma once

#include "common.h"

namespace loki {

constexpr int kQ4Words = 16;        // of a row's codes
constexpr int kQ4Groups = 4;        // of a row
constexpr int kQ4RowBytes = 64;     // of codes; and of scales:
constexpr int kQ4ScaleBytes = 16;

typedef _Float16 cache_half2_t __attribute__((ext_vector_type(2)));

// Entries of a page table are read with scalar loads (no launch writes a table that it reads).
typedef const __attribute__((address_space(4))) int32_t cache_const_i32_t;

// Where rows of a unit lie.  entry() asks the page table (a scalar load, whose result is best not touched at once) and place() makes of
// it what is added to the number of a row (uniform for the wave; with pages, of a row of the same page) to get its place from
// the start of the pool.  An entry that names no page is clamped: such rows are never part of a result, but are read.
struct RowPlaces {
  long long first;  // contiguous: row 0 of the unit
  cache_const_i32_t* table;  // (contiguous: the keys, of which one word is read and not used, in place of a branch)
  bool paged;
  int lg, n_pages, Hkv, h;
  __device__ __forceinline__ RowPlaces(const CacheView& c, int b, int h_, int Hkv_)
      : first(((long long)b * Hkv_ + h_) * c.S_cap),
        table((cache_const_i32_t*)(c.pg.table == nullptr ? static_cast<const int32_t*>(c.k) : c.pg.table + (long long)b * c.pg.pages_per_seq)),
        paged(c.pg.table != nullptr), lg(c.pg.lg_rows), n_pages(c.pg.n_pages), Hkv(Hkv_), h(h_) {}
  __device__ __forceinline__ int entry(int row) const { return table[__builtin_amdgcn_readfirstlane(paged ? row >> lg : 0)]; }
  __device__ __forceinline__ long long place(int row, int entry) const {
    const int at = __builtin_amdgcn_readfirstlane(row >> lg);
    const long long in_page = ((long long)min(max(entry, 0), n_pages - 1) * Hkv + h - at) << lg;
    return paged ? in_page : first;
  }
  __device__ __forceinline__ long long operator()(int row) const { return place(row, entry(row)); }
};

}  // namespace loki
