// Device helpers of the paged cache: whose token a row is, where a slot lies.
#pragma once

#include "hyq_internal.h"

namespace hyq {

// The batch of a step and the pool's geometry, as kernels take them.
struct PagedGeom {
  const int32_t* cu;
  const int32_t* lens;
  const int32_t* table;
  int B, T, max_new, max_len, max_pages;
  int Hq, Hkv, g;
  int page_log2, n_pages;
};

inline PagedGeom paged_geom(const hyq_pcache& c, const hyq_pbatch& b) {
  return PagedGeom{b.cu_new, b.lens, b.table, b.B, b.T, b.max_new, b.max_len, b.max_pages,
                   c.Hq, c.Hkv, c.Hq / c.Hkv, __builtin_ctz((unsigned)c.page), c.n_pages};
}

// One sequence of a step, every count within its bound whatever the device
// arrays say: tokens [t0, t0 + n_new) of the batch, cached slots before them,
// and all its slots (those the table has room for).
struct Seq {
  int t0, n_new, len, n_kv;
};
__device__ __forceinline__ Seq seq_of(const PagedGeom& a, int b) {
  Seq s;
  s.t0 = min(max(a.cu[b], 0), a.T);
  const int end = min(max(a.cu[b + 1], s.t0), a.T);
  s.n_new = min(end - s.t0, a.max_new);
  s.len = min(max(a.lens[b], 0), a.max_len);
  const int64_t cap = (int64_t)a.max_pages << a.page_log2;
  s.n_kv = (int)min((int64_t)s.len + s.n_new, cap);
  return s;
}

// The sequence of token t (the same for every lane of a wave), or -1 if it
// has none: the number of b in [1, B] with cu[b] <= t.
__device__ __forceinline__ int seq_of_token(const PagedGeom& a, int t) {
  const int b = wave_search(a.B, [&](int i) { return a.cu[i + 1] <= t; });
  return b < a.B && a.cu[b] <= t ? b : -1;
}

// Page that holds slot n of sequence b, -1 where the table has none.  No
// branch, so that several lookups are in flight at once.
__device__ __forceinline__ int page_of(const PagedGeom& a, int b, int n) {
  const int i = n >> a.page_log2;
  const int p = a.table[(size_t)b * a.max_pages + min(i, a.max_pages - 1)];
  return i < a.max_pages && (unsigned)p < (unsigned)a.n_pages ? p : -1;
}

// Row of slot n in page p, head j (in rows of the pool).
__device__ __forceinline__ size_t pool_row(const PagedGeom& a, int p, int j, int n) {
  return ((((size_t)p * a.Hkv + j)) << a.page_log2) + (n & ((1 << a.page_log2) - 1));
}

}  // namespace hyq
