// Rows of K and V from one cache to another: paged or contiguous, whole or by a list per KV head.
// Bound by memory: every row is read and written once.  A row of 256 (bf16) or 512 (fp32) bytes goes
// through 16 or 32 lanes; a wavefront has several rows of K and of V under way.
// 8 x 4096 listed rows of 8 heads (270 MB) take 53 us, 5.1 TB/s, what a copy reaches: 78 us with loads and stores that stay
// in the caches, the same with 64 rows to a wavefront instead of 16.  One page of each of 24 sequences: 2.8 us in a graph.
#include "paged.hpp"

namespace ck {

namespace {

struct CopyArgs {
  const void *K, *V;
  void *K2, *V2;
  Pages src, dst;
  const int32_t *n_copy, *row_idx, *begin, *src_seq;
  int Hkv, max_rows, idx_stride;
};

constexpr int COPY_ROWS = 64;                           // of a workgroup: 16 of each wavefront

template <int LANES>                                    // of 16 bytes for a row
__global__ __launch_bounds__(256) void k_copy_rows(const CopyArgs a) {
  const int hp = blockIdx.y, s = hp / a.Hkv, h = hp % a.Hkv;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // three loads under way together, then two for every row
  const int n_copy = a.n_copy[s], from_seq = a.src_seq ? a.src_seq[s] : s, begin = a.begin ? a.begin[s] : 0;
  const int n = n_copy < a.max_rows ? n_copy : a.max_rows;
  const int j0 = blockIdx.x * COPY_ROWS + wave * 16;
  // lane x < 16 finds out where row j0 + x comes from and goes to
  const int j = j0 + (lane & 15);
  const int64_t r = (int64_t)begin + j;
  const int rd = j < n && r >= 0 && r < 0x7FFFFFFF ? (int)r : -1;
  const int rs = a.row_idx ? a.row_idx[(int64_t)hp * a.idx_stride + min(j, a.max_rows - 1)] : rd;
  const bool known = (uint32_t)from_seq < (uint32_t)a.src.n_seqs;
  const Pages::Entry es = a.src.entry(known ? from_seq : 0, known ? rs : -1), ed = a.dst.entry(s, rd);
  const int page_s = a.src.table[es.at], page_d = a.dst.table[ed.at];
  int from = a.src.place(page_s, h, es.slot), to = a.dst.place(page_d, h, ed.slot);
  if (to < 0 || from < 0) from = to = -1;
  if (j0 >= n) return;
  constexpr int PER = 64 / LANES;                       // rows a wavefront moves with one instruction
  constexpr int U = 16 / PER;
  const int part = lane % LANES, sub = lane / LANES;
  const uint4 *K = static_cast<const uint4*>(a.K), *V = static_cast<const uint4*>(a.V);
  uint4 *K2 = static_cast<uint4*>(a.K2), *V2 = static_cast<uint4*>(a.V2);
  constexpr int B = U < 4 ? U : 4;
#pragma unroll
  for (int u0 = 0; u0 < U; u0 += B) {
    uint4 k[B], v[B];
    int t[B];
#pragma unroll
    for (int u = 0; u < B; ++u) {
      const int x = (u0 + u) * PER + sub;
      const int f = __shfl(from, x);
      t[u] = __shfl(to, x);
      if (t[u] < 0) continue;
      k[u] = load_once(K + (int64_t)f * LANES + part);
      v[u] = load_once(V + (int64_t)f * LANES + part);
    }
#pragma unroll
    for (int u = 0; u < B; ++u) {
      if (t[u] < 0) continue;
      store_once(K2 + (int64_t)t[u] * LANES + part, k[u]);
      store_once(V2 + (int64_t)t[u] * LANES + part, v[u]);
    }
  }
}

}  // namespace

hipError_t launch_copy_rows(const Dims& dm, const ck_paged_kv& src, const ck_paged_kv& dst, const int32_t* n_copy,
                            int max_rows, const int32_t* row_idx, int idx_stride, const int32_t* begin,
                            const int32_t* src_seq, hipStream_t st) {
  CopyArgs a = {};
  a.K = src.K;
  a.V = src.V;
  a.K2 = dst.K;
  a.V2 = dst.V;
  a.src = Pages(src, dm.Hkv);
  a.dst = Pages(dst, dm.Hkv);
  a.n_copy = n_copy;
  a.row_idx = row_idx;
  a.begin = begin;
  a.src_seq = src_seq;
  a.Hkv = dm.Hkv;
  a.max_rows = max_rows;
  a.idx_stride = idx_stride;
  const dim3 grid((unsigned)((max_rows + COPY_ROWS - 1) / COPY_ROWS), (unsigned)dm.HP);
  if (dm.dtype == CK_BF16)
    hipLaunchKernelGGL(k_copy_rows<16>, grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL(k_copy_rows<32>, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace ck
