// Page tables, reference counts and slots of new rows from the requests of a batch.
//
// Integers only, and little of them: what counts is the chain of steps that wait for each other.  One workgroup takes
// all of them, so that a step waits for a barrier and not for a launch: pages taken over from parents, pages given back,
// pages given out, slots.  Each step is a list of items (sequence, entry of its table); a prefix sum over the sequences
// numbers them, and a thread finds the sequence of its item by binary search in LDS.  So a sequence with many
// pages and many sequences with one are the same.  Free pages are those that nobody refers to: the counts are read
// once, 16 bytes a lane, and turned to bits in registers; the free page of rank r goes to item r.  Nothing depends
// on the order of atomics.
#include "paged.hpp"

namespace ck {

namespace {

constexpr int PL_THREADS = 1024, PL_WAVES = PL_THREADS / 64;
constexpr int PL_LOADS = 32;                            // of 4 counts a lane, for the pages that are looked at together
// Rows whose slots the planning workgroup writes itself; more are left to a launch of their own.
constexpr int PL_OWN_ROWS = 8192;
constexpr int PL_SLOT_ROWS = 4096;                      // of a workgroup of that launch

struct PlanArgs {
  const int32_t *n_new, *parent, *shared_rows;
  int32_t *lengths, *table, *refs, *q_starts, *slots, *lacking;
  int S, per_seq, n_pages, n_rows;
  Divider size;
  __device__ __forceinline__ int pages_of(int rows) const {
    const int n = size.quotient(rows);
    return n + (rows > n * (int)size.d);
  }
  __device__ __forceinline__ bool is_page(int p) const { return (uint32_t)p < (uint32_t)n_pages; }
};

// Inclusive prefix sums over the workgroup of two numbers a thread, with what earlier chunks left; tmp: LDS.
__device__ __forceinline__ void scan_two(int& x, int& y, int& x_before, int& y_before, int2* tmp) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  x = wave_inclusive_scan(x);
  y = wave_inclusive_scan(y);
  __syncthreads();                                      // tmp may still be in use
  if (lane == WAVE - 1) tmp[wave] = make_int2(x, y);
  __syncthreads();
  int2 mine = make_int2(x_before, y_before), all = mine;
#pragma unroll
  for (int w = 0; w < PL_WAVES; ++w) {
    const int2 t = tmp[w];
    if (w < wave) mine = make_int2(mine.x + t.x, mine.y + t.y);
    all = make_int2(all.x + t.x, all.y + t.y);
  }
  x += mine.x;
  y += mine.y;
  x_before = all.x;
  y_before = all.y;
}

// The first i of [0, n) with upto[i] > x (n - 1 if there is none); upto ascends.
__device__ __forceinline__ int first_beyond(const int* upto, int n, int x) {
  int lo = 0, len = n - 1;                              // in [lo, lo + len]
  while (len > 0) {
    const int half = len >> 1;
    const bool right = upto[lo + half] <= x;
    lo = right ? lo + half + 1 : lo;
    len = right ? len - half - 1 : half;
  }
  return lo;
}

// Slots of rows t, t + step, ..; ends: q_starts[s + 1] of every sequence.
__device__ __forceinline__ void write_slots(const PlanArgs& a, const int* ends, int64_t t, int64_t end, int step) {
  const int total = ends[a.S - 1];
  for (; t < end; t += step) {
    int slot = -1;
    if (t < total) {
      const int s = first_beyond(ends, a.S, (int)t);
      const int64_t r = (int64_t)a.lengths[s] - (ends[s] - (int)t);
      const int e = r >= 0 ? a.size.quotient((int)r) : a.per_seq;
      if (e < a.per_seq) {
        const int page = a.table[(int64_t)s * a.per_seq + e];
        if (a.is_page(page)) slot = page * (int)a.size.d + ((int)r - e * (int)a.size.d);
      }
    }
    a.slots[t] = slot;
  }
}

// What this workgroup wrote to memory before is what its threads read behind it.
__device__ __forceinline__ void memory_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
}

__global__ __launch_bounds__(PL_THREADS) void k_plan_pages(const PlanArgs a) {
  extern __shared__ int lds[];
  int* const rows = lds;                                // [S]: of every sequence, before it gives back or gets tokens
  int* const upto = lds + a.S;                          // [S]: prefix sums
  __shared__ int2 tmp[PL_WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int ps = (int)a.size.d;
  auto after = [&](int s, int n) {                      // rows of a sequence after the call
    const int64_t x = (int64_t)rows[s] + n;
    return (int)(x < 0 ? 0 : (x < 0x7FFFFFFF ? x : 0x7FFFFFFF));
  };
  // items of all sequences, numbered through upto[]: f(sequence, item of it)
  auto for_items = [&](int total, auto f) {
    for (int r = tid; r < total; r += PL_THREADS) {
      const int s = first_beyond(upto, a.S, r);
      f(s, r - (s > 0 ? upto[s - 1] : 0));
    }
  };

  // ---- sequences without rows take over whole pages of a parent, as it stands before the call ----
  int taken = 0, unused = 0, less = 0;
  for (int s0 = 0; s0 < a.S; s0 += PL_THREADS) {
    const int s = s0 + tid;
    int pages = 0, zero = 0;
    if (s < a.S) {
      const int n = a.n_new[s], old = max(a.lengths[s], 0);
      less |= n < 0;
      if (a.parent && old == 0 && n >= 0) {
        const int p = a.parent[s];
        if ((uint32_t)p < (uint32_t)a.S) {
          const int r = max(0, min(a.shared_rows[s], a.lengths[p]));
          pages = min(a.size.quotient(r), a.per_seq);
        }
      }
      rows[s] = old + pages * ps;
    }
    if (a.parent) {
      scan_two(pages, zero, taken, unused, tmp);
      if (s < a.S) upto[s] = pages;
    }
  }
  less = __syncthreads_or(less);
  if (taken > 0) {
    for_items(taken, [&](int s, int e) {
      const int page = a.table[(int64_t)a.parent[s] * a.per_seq + e];
      const bool is = a.is_page(page);
      a.table[(int64_t)s * a.per_seq + e] = is ? page : -1;
      if (is) atomicAdd(a.refs + page, 1);
    });
    memory_barrier();
  }

  // ---- pages that hold no row any more are given back ----
  if (less) {
    int given = 0;
    for (int s0 = 0; s0 < a.S; s0 += PL_THREADS) {
      const int s = s0 + tid;
      int n = 0, zero = 0;
      if (s < a.S && a.n_new[s] < 0)
        n = max(0, min(a.pages_of(rows[s]), a.per_seq) - a.pages_of(after(s, a.n_new[s])));
      scan_two(n, zero, given, unused, tmp);
      if (s < a.S) upto[s] = n;
    }
    __syncthreads();
    for_items(given, [&](int s, int i) {
      int32_t* entry = a.table + (int64_t)s * a.per_seq + a.pages_of(after(s, a.n_new[s])) + i;
      const int page = *entry;
      *entry = -1;
      if (a.is_page(page)) atomicAdd(a.refs + page, -1);
    });
    memory_barrier();
  }

  // ---- pages for new rows ----
  int wanted = 0, tokens = 0, behind = 0;               // behind: pages that the table has no entry for
  for (int s0 = 0; s0 < a.S; s0 += PL_THREADS) {
    const int s = s0 + tid;
    int n = 0, add = 0;
    if (s < a.S) {
      const int m = a.n_new[s], now = after(s, m);
      if (m > 0) {
        const int have = a.pages_of(rows[s]), need = a.pages_of(now);
        n = max(0, min(need, a.per_seq) - have);
        behind += max(0, need - max(have, a.per_seq));
        add = m;
      }
      a.lengths[s] = now;
    }
    scan_two(n, add, wanted, tokens, tmp);
    if (s < a.S) {
      upto[s] = n;
      a.q_starts[s + 1] = add;
    }
  }
  if (tid == 0) a.q_starts[0] = 0;
  __syncthreads();
  auto entry_of = [&](int r) {
    const int s = first_beyond(upto, a.S, r);
    return a.table + (int64_t)s * a.per_seq + a.pages_of(rows[s]) + (r - (s > 0 ? upto[s - 1] : 0));
  };
  int found = 0;                                        // free pages so far
  constexpr int LOAD = WAVE * 4;                        // pages of a wavefront's load
  for (int p0 = 0; p0 < a.n_pages && found < wanted; p0 += PL_WAVES * PL_LOADS * LOAD) {
    const int left = (a.n_pages - p0 + LOAD - 1) / LOAD;
    const int loads = min(PL_LOADS, (left + PL_WAVES - 1) / PL_WAVES);
    const int first = p0 + wave * loads * LOAD + lane * 4;
    uint32_t bits[PL_LOADS / 8];                          // four pages of a load each
    int n = 0, zero = 0;
#pragma unroll
    for (int g = 0; g < PL_LOADS / 8; ++g) {
      bits[g] = 0;
      if (g * 8 >= loads) continue;
      int4 c[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int p = first + (g * 8 + j) * LOAD;
        c[j] = make_int4(1, 1, 1, 1);
        if (g * 8 + j < loads) {
          if (p + 3 < a.n_pages) {
            c[j] = *reinterpret_cast<const int4*>(a.refs + p);
          } else {
            if (p < a.n_pages) c[j].x = a.refs[p];
            if (p + 1 < a.n_pages) c[j].y = a.refs[p + 1];
            if (p + 2 < a.n_pages) c[j].z = a.refs[p + 2];
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j)
        bits[g] |= (uint32_t)((c[j].x == 0) | (c[j].y == 0) << 1 | (c[j].z == 0) << 2 | (c[j].w == 0) << 3) << (4 * j);
      n += __popc(bits[g]);
    }
    int rank = n;
    scan_two(rank, zero, found, unused, tmp);
    rank = __builtin_amdgcn_readfirstlane(rank - n);    // of the wavefront's first free page
#pragma unroll
    for (int g = 0; g < PL_LOADS / 8; ++g) {
#pragma unroll 1
      for (int j = 0; j < 8; ++j) {
        const uint32_t four = (bits[g] >> (4 * j)) & 15u;
        if (__ballot(four != 0) == 0) continue;
        const int c = __popc(four), upto_lane = wave_inclusive_scan(c);
        int r = rank + upto_lane - c;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (!((four >> i) & 1)) continue;
          if (r < wanted) {
            const int p = first + (g * 8 + j) * LOAD + i;
            a.refs[p] = 1;
            *entry_of(r) = p;
          }
          ++r;
        }
        rank += __builtin_amdgcn_readlane(upto_lane, WAVE - 1);
      }
    }
  }
  for (int r = found + tid; r < wanted; r += PL_THREADS) *entry_of(r) = -1;
  int none = 0;
  scan_two(behind, none, unused, none, tmp);
  if (tid == PL_THREADS - 1) *a.lacking = behind + max(0, wanted - found);
  if (!a.slots || a.n_rows > PL_OWN_ROWS) return;

  // ---- slots ----
  memory_barrier();
  for (int s = tid; s < a.S; s += PL_THREADS) upto[s] = a.q_starts[s + 1];
  __syncthreads();
  write_slots(a, upto, tid, a.n_rows, PL_THREADS);
}

__global__ __launch_bounds__(PL_THREADS) void k_plan_slots(const PlanArgs a) {
  extern __shared__ int ends[];
  for (int s = threadIdx.x; s < a.S; s += PL_THREADS) ends[s] = a.q_starts[s + 1];
  __syncthreads();
  const int64_t t0 = (int64_t)blockIdx.x * PL_SLOT_ROWS;
  write_slots(a, ends, t0 + threadIdx.x, min(t0 + PL_SLOT_ROWS, (int64_t)a.n_rows), PL_THREADS);
}

}  // namespace

hipError_t launch_plan_pages(int S, const int32_t* n_new, int32_t* lengths, int32_t* page_table, int pages_per_seq,
                             int32_t* page_refs, int n_pages, int page_size, const int32_t* parent,
                             const int32_t* shared_rows, int32_t* q_starts, int32_t* slots, int64_t n_rows,
                             int32_t* lacking, hipStream_t st) {
  PlanArgs a = {};
  a.n_new = n_new;
  a.parent = parent;
  a.shared_rows = shared_rows;
  a.lengths = lengths;
  a.table = page_table;
  a.refs = page_refs;
  a.q_starts = q_starts;
  a.slots = n_rows > 0 ? slots : nullptr;
  a.lacking = lacking;
  a.S = S;
  a.per_seq = pages_per_seq;
  a.n_pages = n_pages;
  a.n_rows = (int)n_rows;
  a.size = Divider((uint32_t)page_size);
  hipLaunchKernelGGL(k_plan_pages, dim3(1), dim3(PL_THREADS), (size_t)S * 2 * sizeof(int), st, a);
  if (a.slots && n_rows > PL_OWN_ROWS)
    hipLaunchKernelGGL(k_plan_slots, dim3((unsigned)((n_rows + PL_SLOT_ROWS - 1) / PL_SLOT_ROWS)), dim3(PL_THREADS),
                       (size_t)S * sizeof(int), st, a);
  return hipGetLastError();
}

}  // namespace ck
