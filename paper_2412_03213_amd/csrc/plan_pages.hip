// Page tables, reference counts and slots of new rows from the requests of a batch.
//
// Integers only, and few: what counts is the chain of steps that wait for each other.  One workgroup takes
// all of them, so that a step waits for a barrier and not for a launch: pages taken over from parents, pages given back,
// pages given out, slots.  Each step is a list of items (sequence, entry of its table); a prefix sum over the sequences
// numbers them, and a thread finds the sequence of its item by binary search in LDS.  So a sequence with many
// pages and many sequences with one are the same.  Free pages are those that nobody refers to: the counts are read
// once, 16 bytes a lane, and turned to bits in registers; the free page of rank r goes to item r.  Nothing depends
// on the order of atomics.
#include "paged.hpp"

namespace ck {

namespace {

// Threads of the planning workgroup.  Prefix sums are done by every wavefront for itself, over all of them: four are done
// sooner where there are few sequences and few pages to take over or give back, for which the host has the table's size.  Tokens
// given and taken back, two calls in a graph, four / sixteen, us: 64 sequences 11.2 / 13.6, 100 with a table of 502 entries each
// 14.4 / 15.8, 12000 pages taken over and 16500 given back 94 / 71.
constexpr int PL_FEW = 256, PL_MANY = 1024, PL_FEW_ENTRIES = 65536;
constexpr int PL_LOADS = 32;                            // runs of 256 pages that a wavefront looks at together, at most
// ... and the workgroup to begin with, four times as many in each turn.  A token for each of 64 sequences (5 pages of 16384)
// and taken back, two calls in a graph: 11.2 us, 11.8 with 32 runs, 10.9 with 8; 14.0, 14.7 and 16.1 where no page is free.
constexpr int PL_FIRST_RUNS = 16;
constexpr int PL_ITEMS = 4;                             // of a thread at a time
constexpr int PL_LIST = 2048;                           // free pages that are given out together
// Rows whose slots the planning workgroup writes itself; more are left to a launch of their own (two calls, us: 2400 rows
// 13.1 and 13.6, 4000 14.1 and 13.7, 16000 21.6 and 14.8).
constexpr int PL_OWN_ROWS = 3000;
constexpr int PL_SLOT_ROWS = PL_MANY;                   // of a workgroup of that launch

struct PlanArgs {
  const int32_t *n_new, *parent, *shared_rows;
  int32_t *lengths, *table, *refs, *q_starts, *slots, *lacking;
  int S, per_seq, n_pages, n_rows;                      // S * per_seq < 2^31
  Divider size;
  __device__ __forceinline__ int pages_of(int rows) const {
    const int n = size.quotient(rows);
    return n + (rows > n * (int)size.d);
  }
  __device__ __forceinline__ bool is_page(int p) const { return (uint32_t)p < (uint32_t)n_pages; }
};

// Inclusive prefix sums over the workgroup of two numbers a thread, with what earlier chunks left; tmp: LDS.
template <int WAVES>
__device__ __forceinline__ void scan_two(int& x, int& y, int& x_before, int& y_before, int2* tmp) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  x = wave_inclusive_scan(x);
  y = wave_inclusive_scan(y);
  __syncthreads();                                      // tmp may still be in use
  if (lane == WAVE - 1) tmp[wave] = make_int2(x, y);
  __syncthreads();
  int2 mine = make_int2(x_before, y_before), all = mine;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const int2 t = tmp[w];
    if (w < wave) mine = make_int2(mine.x + t.x, mine.y + t.y);
    all = make_int2(all.x + t.x, all.y + t.y);
  }
  x += mine.x;
  y += mine.y;
  x_before = all.x;
  y_before = all.y;
}

// The first i of [0, n) with upto[i] > x (n - 1 if there is none), for several x at a time; upto ascends.
template <int N>
__device__ __forceinline__ void first_beyond(const int* upto, int n, const int (&x)[N], int (&i)[N]) {
#pragma unroll
  for (int u = 0; u < N; ++u) i[u] = 0;
  for (int b = 1 << (31 - __builtin_clz(n)); b; b >>= 1)
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int k = i[u] + b;
      i[u] = upto[min(k, n) - 1] <= x[u] && k < n ? k : i[u];
    }
}
__device__ __forceinline__ int first_beyond(const int* upto, int n, int x) {
  const int one[1] = {x};
  int i[1];
  first_beyond<1>(upto, n, one, i);
  return i[0];
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
        const int page = a.table[(uint32_t)(s * a.per_seq + e)];
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

template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_plan_pages(const PlanArgs a) {
  constexpr int WAVES = THREADS / 64;
  extern __shared__ int lds[];
  int* const rows = lds;                                // [S]: of every sequence, before it gives back or gets tokens
  int* const upto = lds + a.S;                          // [S]: prefix sums
  __shared__ int2 tmp[WAVES];
  __shared__ int behind;                                // pages that the table has no entry for
  __shared__ int list[PL_LIST];                         // free pages
  __shared__ int free_upto[PL_LOADS * WAVES];           // free pages of a run; then before it
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int ps = (int)a.size.d;
  auto after = [&](int s, int n) {                      // rows of a sequence after the call
    const int64_t x = (int64_t)rows[s] + n;
    return (int)(x < 0 ? 0 : (x < 0x7FFFFFFF ? x : 0x7FFFFFFF));
  };
  // Items of all sequences, numbered through upto[]: get(sequence, item of it) asks for what put takes.  Several at a
  // time: an item is a chain of look-ups, one after the other.
  auto for_items = [&](int total, auto get, auto put) {
    for (int r0 = tid; r0 < total; r0 += PL_ITEMS * THREADS) {
      decltype(get(0, 0)) x[PL_ITEMS];
      int r[PL_ITEMS], s[PL_ITEMS];
#pragma unroll
      for (int u = 0; u < PL_ITEMS; ++u) r[u] = min(r0 + u * THREADS, total - 1);   // the last one again behind the end
      first_beyond<PL_ITEMS>(upto, a.S, r, s);
#pragma unroll
      for (int u = 0; u < PL_ITEMS; ++u) x[u] = get(s[u], r[u] - (s[u] > 0 ? upto[s[u] - 1] : 0));
#pragma unroll
      for (int u = 0; u < PL_ITEMS; ++u)
        if (r0 + u * THREADS < total) put(x[u]);
    }
  };
  struct Entry { int32_t* at; int page; };

  // the counts of pages p to p + 3; behind the last there are no free ones
  auto counts_of = [&](int p) {
    int4 c = make_int4(1, 1, 1, 1);
    if (p + 3 < a.n_pages) return *reinterpret_cast<const int4*>(a.refs + p);
    if (p < a.n_pages) c.x = a.refs[p];
    if (p + 1 < a.n_pages) c.y = a.refs[p + 1];
    if (p + 2 < a.n_pages) c.z = a.refs[p + 2];
    return c;
  };
  // Those that are looked at first are asked for before it is known whether pages are wanted.
  constexpr int RUN = WAVE * 4, FIRST = PL_FIRST_RUNS / WAVES;
  int4 counts[FIRST];
#pragma unroll
  for (int k = 0; k < FIRST; ++k) counts[k] = counts_of((k * WAVES + wave) * RUN + lane * 4);
  if (tid == 0) behind = 0;

  // ---- sequences without rows take over whole pages of a parent, as it stands before the call ----
  int taken = 0, unused = 0, less = 0;
  for (int s0 = 0; s0 < a.S; s0 += THREADS) {
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
      scan_two<WAVES>(pages, zero, taken, unused, tmp);
      if (s < a.S) upto[s] = pages;
    }
  }
  less = __syncthreads_or(less);
  if (taken > 0) {
    for_items(taken,
              [&](int s, int e) -> Entry {
                return {a.table + (uint32_t)(s * a.per_seq + e), a.table[(uint32_t)(a.parent[s] * a.per_seq + e)]};
              },
              [&](const Entry& x) {
                const bool is = a.is_page(x.page);
                *x.at = is ? x.page : -1;
                if (is) atomicAdd(a.refs + x.page, 1);
              });
    memory_barrier();
  }

  // ---- pages that hold no row any more are given back ----
  if (less) {
    int given = 0;
    for (int s0 = 0; s0 < a.S; s0 += THREADS) {
      const int s = s0 + tid;
      int n = 0, zero = 0;
      if (s < a.S && a.n_new[s] < 0)
        n = max(0, min(a.pages_of(rows[s]), a.per_seq) - a.pages_of(after(s, a.n_new[s])));
      scan_two<WAVES>(n, zero, given, unused, tmp);
      if (s < a.S) upto[s] = n;
    }
    __syncthreads();
    for_items(given,
              [&](int s, int i) -> Entry {
                int32_t* at = a.table + (uint32_t)(s * a.per_seq + a.pages_of(after(s, a.n_new[s])) + i);
                return {at, *at};
              },
              [&](const Entry& x) {
                *x.at = -1;
                if (a.is_page(x.page)) atomicAdd(a.refs + x.page, -1);
              });
    memory_barrier();
  }

  // ---- pages for new rows ----
  int wanted = 0, tokens = 0;
  for (int s0 = 0; s0 < a.S; s0 += THREADS) {
    const int s = s0 + tid;
    int n = 0, add = 0;
    if (s < a.S) {
      const int m = a.n_new[s], now = after(s, m);
      if (m > 0) {
        const int have = a.pages_of(rows[s]), need = a.pages_of(now);
        n = max(0, min(need, a.per_seq) - have);
        const int none = need - max(have, a.per_seq);
        if (none > 0) atomicAdd(&behind, none);
        add = m;
      }
      a.lengths[s] = now;
    }
    scan_two<WAVES>(n, add, wanted, tokens, tmp);
    if (s < a.S) {
      upto[s] = n;
      a.q_starts[s + 1] = add;
    }
  }
  if (tid == 0) a.q_starts[0] = 0;
  __syncthreads();
  auto entry_of = [&](int r) {
    const int s = first_beyond(upto, a.S, r);
    return a.table + (uint32_t)(s * a.per_seq + a.pages_of(rows[s]) + (r - (s > 0 ? upto[s - 1] : 0)));
  };
  // Free pages, by runs of 256 that go to the wavefronts in turn, so that all of them have some to give out.
  int found = 0;                                        // free pages so far
  const bool unchanged = taken == 0 && !less;           // since the counts were asked for
  for (int p0 = 0, loads = FIRST; p0 < a.n_pages && found < wanted;) {
    const int left = (a.n_pages - p0 + RUN - 1) / RUN - wave;   // runs that are this wavefront's
    const int mine = max(0, min(loads, (left + WAVES - 1) / WAVES));
    auto first_of = [&](int k) { return p0 + (k * WAVES + wave) * RUN; };
    uint32_t bits[PL_LOADS / 8];                          // four pages of a run each
#pragma unroll
    for (int g = 0; g < PL_LOADS / 8; ++g) {
      bits[g] = 0;
      int4 c[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (g * 8 + j >= mine) continue;                // wave-uniform, as below
        if (g * 8 + j < FIRST && p0 == 0 && unchanged)
          c[j] = counts[(g * 8 + j) % FIRST];
        else
          c[j] = counts_of(first_of(g * 8 + j) + lane * 4);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (g * 8 + j >= mine) continue;
        const bool f[4] = {c[j].x == 0, c[j].y == 0, c[j].z == 0, c[j].w == 0};
        int n = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          n += __popcll(__ballot(f[i]));
          bits[g] |= (uint32_t)f[i] << (4 * j + i);
        }
        if (lane == 0) free_upto[(g * 8 + j) * WAVES + wave] = n;
      }
    }
    if (lane == 0)
      for (int k = mine; k < loads; ++k) free_upto[k * WAVES + wave] = 0;
    __syncthreads();
    const bool run = tid < loads * WAVES;
    int n = run ? free_upto[tid] : 0, zero = 0;
    const int n_run = n, found_before = found;
    scan_two<WAVES>(n, zero, found, unused, tmp);
    if (run) free_upto[tid] = n - n_run;                // before the run
    __syncthreads();
    // their numbers in order, so many at a time, then the entries that get them
    const int end = min(found, wanted);
    for (int r0 = found_before; r0 < end; r0 += PL_LIST) {
#pragma unroll
      for (int g = 0; g < PL_LOADS / 8; ++g) {
        if (g * 8 >= mine) continue;
#pragma unroll 1
        for (int j = 0; j < min(8, mine - g * 8); ++j) {
          const int k = g * 8 + j;
          int r = __builtin_amdgcn_readfirstlane(free_upto[k * WAVES + wave]) - r0;
          if (r >= PL_LIST || r + r0 >= end) break;
          const uint32_t four = (bits[g] >> (4 * j)) & 15u;
          const int c = __popc(four);
          r += wave_inclusive_scan(c) - c;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (!((four >> i) & 1)) continue;
            if ((uint32_t)r < (uint32_t)PL_LIST) list[r] = first_of(k) + lane * 4 + i;
            ++r;
          }
        }
      }
      __syncthreads();
      for (int r = r0 + tid; r < min(end, r0 + PL_LIST); r += THREADS) {
        const int p = list[r - r0];
        a.refs[p] = 1;
        *entry_of(r) = p;
      }
      __syncthreads();                                  // list and free_upto are read no more
    }
    p0 += loads * WAVES * RUN;
    loads = min(4 * loads, PL_LOADS);
  }
  for (int r = found + tid; r < wanted; r += THREADS) *entry_of(r) = -1;
  if (tid == 0) *a.lacking = behind + max(0, wanted - found);
  if (!a.slots || a.n_rows > PL_OWN_ROWS) return;

  // ---- slots ----
  memory_barrier();
  for (int s = tid; s < a.S; s += THREADS) upto[s] = a.q_starts[s + 1];
  __syncthreads();
  write_slots(a, upto, tid, a.n_rows, THREADS);
}

__global__ __launch_bounds__(PL_MANY) void k_plan_slots(const PlanArgs a) {
  extern __shared__ int ends[];
  for (int s = threadIdx.x; s < a.S; s += PL_MANY) ends[s] = a.q_starts[s + 1];
  __syncthreads();
  const int64_t t0 = (int64_t)blockIdx.x * PL_SLOT_ROWS;
  write_slots(a, ends, t0 + threadIdx.x, min(t0 + PL_SLOT_ROWS, (int64_t)a.n_rows), PL_MANY);
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
  if (S <= PL_FEW && (int64_t)S * pages_per_seq <= PL_FEW_ENTRIES && n_rows <= 4 * PL_FEW)
    hipLaunchKernelGGL(k_plan_pages<PL_FEW>, dim3(1), dim3(PL_FEW), (size_t)S * 2 * sizeof(int), st, a);
  else
    hipLaunchKernelGGL(k_plan_pages<PL_MANY>, dim3(1), dim3(PL_MANY), (size_t)S * 2 * sizeof(int), st, a);
  if (a.slots && n_rows > PL_OWN_ROWS)
    hipLaunchKernelGGL(k_plan_slots, dim3((unsigned)((n_rows + PL_SLOT_ROWS - 1) / PL_SLOT_ROWS)), dim3(PL_MANY),
                       (size_t)S * sizeof(int), st, a);
  return hipGetLastError();
}

}  // namespace ck
