// Caches in pages: from a row of a sequence to its place in the pool, and from a row of a ragged
// batch to its sequence.
#pragma once
#include "ck_common.hpp"

namespace ck {

// n / d for 0 <= n < 2^31, d >= 1: the product with a rounded-down reciprocal is the quotient or one less.
struct Divider {
  uint32_t d, magic;
  Divider() : d(1), magic(0xFFFFFFFFu) {}
  explicit Divider(uint32_t d_) : d(d_), magic(d_ > 1 ? (uint32_t)((1ull << 32) / d_) : 0xFFFFFFFFu) {}
  __device__ __forceinline__ int quotient(int n) const {
    const uint32_t q = __umulhi((uint32_t)n, magic);
    return (int)((uint32_t)n - q * d >= d ? q + 1 : q);
  }
};

// 16 bytes that are read or written once: they go past the caches' order of use, and a write does not stay in
// L2 until the end of the launch has it written back.
__device__ __forceinline__ uint4 load_once(const void* p) {
  typedef uint32_t Words __attribute__((ext_vector_type(4)));
  const Words w = __builtin_nontemporal_load(static_cast<const Words*>(p));
  return make_uint4(w.x, w.y, w.z, w.w);
}
__device__ __forceinline__ void store_once(void* p, const uint4& x) {
  typedef uint32_t Words __attribute__((ext_vector_type(4)));
  __builtin_nontemporal_store(Words{x.x, x.y, x.z, x.w}, static_cast<Words*>(p));
}

struct Pages {
  const int32_t* table;
  int n_pages, n_seqs, per_seq, Hkv;
  int rows;                                             // of a sequence: per_seq * page size
  Divider size;
  Pages() = default;
  Pages(const ck_paged_kv& kv, int Hkv_)
      : table(kv.page_table), n_pages(kv.n_pages), n_seqs(kv.n_seqs), per_seq(kv.pages_per_seq), Hkv(Hkv_),
        rows(kv.page_size * kv.pages_per_seq), size((uint32_t)kv.page_size) {}
  __device__ __forceinline__ int clamp_length(int n) const { return n < 0 ? 0 : (n < rows ? n : rows); }
  // Where a row's page number stands (some number that the table has, for a row that it does not have), and
  // from the number the pool row (of d channels) of the row; -1 where there is none.  In two steps and without a
  // branch, so that loads of several rows are under way together.
  struct Entry { int64_t at; int slot; };               // slot < 0: no such row
  __device__ __forceinline__ Entry entry(int s, int r) const {
    const bool is = (uint32_t)r < (uint32_t)rows;
    const int e = size.quotient(is ? r : 0);
    return {(int64_t)s * per_seq + e, is ? r - e * (int)size.d : -1};
  }
  __device__ __forceinline__ int place(int page, int h, int slot) const {
    return slot >= 0 && (uint32_t)page < (uint32_t)n_pages ? (page * Hkv + h) * (int)size.d + slot : -1;
  }
  __device__ __forceinline__ int row(int s, int h, int r) const {
    const Entry e = entry(s, r);
    return place(table[e.at], h, e.slot);
  }
};

// Sequence whose rows [starts[s], starts[s + 1]) hold t, -1 where none does.  By a whole wavefront, 64
// ways a step; t is the same in all lanes.  Whatever starts holds, what is returned satisfies both bounds.
__device__ __forceinline__ int find_sequence(const int32_t* __restrict__ starts, int S, int t) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = S;                                    // the last s of [lo, lo + n) with starts[s] <= t
  while (n > 1) {
    const int step = (n + 63) >> 6, i = lane * step;
    const uint64_t le = __ballot(i < n && starts[lo + (i < n ? i : 0)] <= t);
    const int k = le ? 63 - __builtin_clzll(le) : 0;
    lo += k * step;
    n = n - k * step < step ? n - k * step : step;
  }
  return starts[lo] <= t && t < starts[lo + 1] ? lo : -1;
}

}  // namespace ck
