// A paged cache as the kernels see it (spt_cache of spt.h, checked on the host): strides in bytes, the page size as a shift.
#pragma once
#include "common.hpp"

namespace spt {

struct Cache {
  char* K;
  char* V;
  int32_t* table;
  int32_t* len;
  int32_t* refs;
  int64_t layer_bytes, page_bytes, slot_bytes, head_bytes;
  int rows, row_pages, pages, shift;  // page = 1 << shift
  int layers, heads, width_bytes;
  uint32_t page_vecs, slot_vecs;  // page_bytes and slot_bytes in units of 16
};

inline int value_bytes(int dtype) { return dtype == SPT_F32 ? 4 : 2; }

inline Cache cache_view(const spt_cache* c) {
  const int64_t b = value_bytes(c->dtype);
  int shift = 0;
  while ((1 << shift) < c->page) ++shift;
  return {static_cast<char*>(c->K), static_cast<char*>(c->V), c->table, c->len, c->refs, c->layer_stride * b, c->page_stride * b,
          c->slot_stride * b, c->head_stride * b, c->rows, c->row_pages, static_cast<int>(c->pages), shift, c->layers, c->heads,
          static_cast<int>(c->width * b), static_cast<uint32_t>(c->page_stride * b / 16), static_cast<uint32_t>(c->slot_stride * b / 16)};
}

// A CSR pattern: the entries of row r are crd[begin(r) .. end(r)), whatever pos holds.
struct Pattern {
  const int32_t* pos;
  const int32_t* crd;
  int entries;
};

inline Pattern pattern_view(const spt_tensor* t) {
  return t ? Pattern{t->level[1].pos, t->level[1].crd, static_cast<int>(t->nvals)} : Pattern{nullptr, nullptr, 0};
}

// Division of numbers from 0 to 2^31 - 1 by a divisor that the host knows: one multiplication. With 2^shift the next power of two from
// the divisor d on and mul = ceil(2^(31 + shift) / d), mul d exceeds 2^(31 + shift) by less than 2^shift, so x mul / 2^(31 + shift)
// exceeds x / d by less than 1 / d.
struct Divisor {
  uint32_t mul, shift;
};
inline Divisor divisor(uint32_t d) {
  uint32_t shift = 0;
  while ((uint64_t(1) << shift) < d) ++shift;
  return {static_cast<uint32_t>(((uint64_t(1) << (31 + shift)) + d - 1) / d), shift};
}

#if defined(__HIPCC__)

__device__ __forceinline__ int operator/(int x, const Divisor& d) {
  return static_cast<int>(__umulhi(static_cast<uint32_t>(x) << 1, d.mul) >> d.shift);
}

__host__ __device__ __forceinline__ int clamped(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

__device__ __forceinline__ int row_length(const Cache& c, int s) { return clamped(c.len[s], 0, c.row_pages << c.shift); }
// Pages that hold t tokens.
__device__ __forceinline__ int pages_held(const Cache& c, int t) { return (t + (1 << c.shift) - 1) >> c.shift; }
// Page of place j in row s, or -1 if the table names none.
__device__ __forceinline__ int page_at(const Cache& c, int s, int j) {
  const int p = c.table[static_cast<int64_t>(s) * c.row_pages + j];
  return p >= 0 && p < c.pages ? p : -1;
}

// Rows first[s] .. first[s+1] of the call that belong to row s of the cache.
struct Drafted {
  int begin, count;
};
__device__ __forceinline__ Drafted drafted(const int32_t* first, int s, int total) {
  const int a = clamped(first[s], 0, total), b = clamped(first[s + 1], 0, total);
  return {a, b > a ? b - a : 0};
}

__device__ __forceinline__ int pattern_begin(const Pattern& p, int r) { return clamped(p.pos[r], 0, p.entries); }
__device__ __forceinline__ int pattern_end(const Pattern& p, int r) { return clamped(p.pos[r + 1], 0, p.entries); }

// The row s with first[s] <= i < first[s+1], by all lanes of a wave; -1 if there is none.
__device__ __forceinline__ int wave_row_of(const int32_t* first, int rows, int i) {
  const int s = wave_lower_bound(first, rows + 1, i + 1) - 1;
  return s >= 0 && s < rows ? s : -1;
}

#endif

}  // namespace spt
