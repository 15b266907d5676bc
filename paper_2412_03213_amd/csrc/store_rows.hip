// Rows of keys and values to their slots in a pool of pages, as they are.
// Bound by memory: every row is read and written once.  A token's row of all heads is one run of 16-byte pieces, a
// head's 256 (bf16) or 512 (fp32) bytes of it one run in the pool; each thread has four pieces of K and of V under way.
#include "paged.hpp"

namespace ck {

namespace {

struct StoreArgs {
  const void *k, *v;
  void *K, *V;
  const int32_t* slots;
  int64_t k_stride, v_stride, n_pieces;                 // pieces of 16 bytes: of a token's row, and all of them
  int Hkv, n_slots;
  Divider row, size;                                    // pieces of a token, rows of a page
};

constexpr int ST_PIECES = 4;

template <int LANES>                                    // of 16 bytes for a row of one head
__global__ __launch_bounds__(256) void k_store_rows(const StoreArgs a) {
  const int64_t first = (int64_t)blockIdx.x * (256 * ST_PIECES) + threadIdx.x;
  int64_t from_k[ST_PIECES], from_v[ST_PIECES], to[ST_PIECES];
  int slot[ST_PIECES], piece[ST_PIECES];
#pragma unroll
  for (int u = 0; u < ST_PIECES; ++u) {
    const int64_t e = first + u * 256;
    const int x = (int)(e < a.n_pieces ? e : 0), t = a.row.quotient(x);
    piece[u] = x - t * (int)a.row.d;
    slot[u] = a.slots[t];
    if (e >= a.n_pieces) slot[u] = -1;
    from_k[u] = t * a.k_stride + piece[u];
    from_v[u] = t * a.v_stride + piece[u];
  }
  const uint4 *k = static_cast<const uint4*>(a.k), *v = static_cast<const uint4*>(a.v);
  uint4 *K = static_cast<uint4*>(a.K), *V = static_cast<uint4*>(a.V);
  uint4 kw[ST_PIECES], vw[ST_PIECES];
#pragma unroll
  for (int u = 0; u < ST_PIECES; ++u) {
    kw[u] = load_once(k + from_k[u]);
    vw[u] = load_once(v + from_v[u]);
    const bool is = (uint32_t)slot[u] < (uint32_t)a.n_slots;
    const int h = piece[u] / LANES, page = a.size.quotient(is ? slot[u] : 0);
    to[u] = is ? (int64_t)((page * a.Hkv + h) * (int)a.size.d + (slot[u] - page * (int)a.size.d)) * LANES + piece[u] % LANES : -1;
  }
#pragma unroll
  for (int u = 0; u < ST_PIECES; ++u) {
    if (to[u] < 0) continue;
    store_once(K + to[u], kw[u]);
    store_once(V + to[u], vw[u]);
  }
}

}  // namespace

hipError_t launch_store_rows(const Dims& dm, const void* k, const void* v, int64_t k_stride, int64_t v_stride,
                             int64_t n_rows, const int32_t* slots, const ck_paged_kv& kv, hipStream_t st) {
  const int lanes = dm.dtype == CK_BF16 ? 16 : 32, each = D / lanes;   // elements of a piece
  StoreArgs a = {};
  a.k = k;
  a.v = v;
  a.K = kv.K;
  a.V = kv.V;
  a.slots = slots;
  a.k_stride = k_stride / each;
  a.v_stride = v_stride / each;
  a.n_pieces = n_rows * dm.Hkv * lanes;
  a.Hkv = dm.Hkv;
  a.n_slots = kv.n_pages * kv.page_size;
  a.row = Divider((uint32_t)(dm.Hkv * lanes));
  a.size = Divider((uint32_t)kv.page_size);
  const dim3 grid((unsigned)((a.n_pieces + 256 * ST_PIECES - 1) / (256 * ST_PIECES)));
  if (dm.dtype == CK_BF16)
    hipLaunchKernelGGL(k_store_rows<16>, grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL(k_store_rows<32>, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace ck
