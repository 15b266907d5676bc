// Page tables, reference counts and slots of new rows from the requests of a batch.
//
// Integers only, and few: what counts is the chain of steps that wait for each other.  One workgroup takes
// all of them, so that a step waits for a barrier and not for a launch: pages taken over from parents, pages given back,
// pages given out, slots.  Each step is a list of entries of tables, single ones or runs of up to 64; a prefix sum over the
// sequences numbers them, and a thread finds the sequence of its entry or run by binary search in LDS.  So a sequence with
// many pages and many sequences with one are the same.  Free pages are those that nobody refers to: the counts are read
// once, 16 bytes a lane, and turned to bits in registers; the free page of rank r goes to item r.  Nothing depends
// on the order of atomics.
#include "paged.hpp"

namespace ck {

namespace {

// Threads of the planning workgroup.  Prefix sums are done by every wavefront for itself, over all of them: four are done
// sooner where there are few sequences and few pages to take over or give back, for which the host has the table's size.  Tokens
// given and taken back, two calls in a graph, four / sixteen, us: 64 sequences 11.0 / 13.8, 100 with a table of 502 entries each
// 13.8 / 16.0, 64 prompts of 1000 tokens 32.5 / 24.2, 12000 pages taken over and 16500 given back 118 / 61.
constexpr int PL_FEW = 256, PL_MANY = 1024, PL_FEW_ENTRIES = 65536;
constexpr int PL_LOADS = 32;                            // runs of 256 pages that a wavefront looks at together, at most
// ... and the workgroup to begin with, four times as many in each turn.  A token for each of 64 sequences (5 pages of 16384)
// and taken back, two calls in a graph: 11.2 us, 11.8 with 32 runs, 10.9 with 8; 14.0, 14.7 and 16.1 where no page is free.
constexpr int PL_FIRST_RUNS = 16;
constexpr int PL_RUNS = 4;                              // of entries that a wavefront takes together (8: as fast)
// Where many counts change, those of the first pages do in LDS, 16 bits each, and then once in memory: a compute unit takes
// 4.5 cycles for an atomic to memory.  Two calls, us, with / without: 4000 entries given back in a pool of 16384 pages 26.0 /
// 27.7; 12000 taken over and 16500 given back in one of 32768 49.5 / 65.7, of 131072 61.2 / 69.3.
constexpr int PL_COUNTED = 65536, PL_COUNTED_MANY = 32768;   // pages; the smaller number where sequences need the room
constexpr int PL_COUNTED_S = 1024;
constexpr int PL_LEAST = 2000, PL_MOST = 32768;         // entries that are taken over, or given back, for that: [least, most)
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

// Up to 64 entries of one sequence: read from, written to, as numbers in the table.
struct Run { int from, to, n; };

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

template <int THREADS, int COUNTED>
__global__ __launch_bounds__(THREADS) void k_plan_pages(const PlanArgs a) {
  constexpr int WAVES = THREADS / 64;
  extern __shared__ int lds[];
  int* const rows = lds;                                // [S]: of every sequence, before it gives back or gets tokens
  int* const upto = lds + a.S;                          // [S]: prefix sums
  __shared__ int2 tmp[WAVES];
  __shared__ int behind;                                // pages that the table has no entry for
  __shared__ int list[PL_LIST];                         // free pages
  __shared__ int free_upto[PL_LOADS * WAVES];           // free pages of a run; then before it
  __shared__ int4 changes[COUNTED / 8];                 // of the counts of the first pages: even ones in the lower half of a word
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int ps = (int)a.size.d;
  auto after = [&](int s, int n) {                      // rows of a sequence after the call
    const int64_t x = (int64_t)rows[s] + n;
    return (int)(x < 0 ? 0 : (x < 0x7FFFFFFF ? x : 0x7FFFFFFF));
  };
  const int counted = min(COUNTED, a.n_pages);
  bool in_lds = false;                                  // changes[] is in use
  auto count_in_lds = [&](int entries) {
    if (in_lds || entries < PL_LEAST) return;
    for (int i = tid; i < (counted + 7) / 8; i += THREADS) changes[i] = make_int4(0, 0, 0, 0);
    in_lds = true;
  };
  auto change = [&](int page, int by, bool here) {
    if (here && page < counted)
      atomicAdd(reinterpret_cast<int*>(changes) + (page >> 1), by * (page & 1 ? 65536 : 1));
    else
      atomicAdd(a.refs + page, by);
  };
  // Entries of all sequences, up to 64 of one of them at a time, numbered through upto[]: a lane finds one such run, of(sequence,
  // number of its run), for its wavefront, which then takes them one after the other, an entry each lane.
  auto for_runs = [&](int total, auto of, auto put) {
    for (int x0 = 0; x0 < total; x0 += THREADS) {
      const int x = min(x0 + lane * WAVES + wave, total - 1);
      const int s = first_beyond(upto, a.S, x);
      const Run mine = of(s, x - (s > 0 ? upto[s - 1] : 0));
      const int runs = min((total - x0 - wave + WAVES - 1) / WAVES, WAVE);   // of this wavefront
      for (int k = 0; k < runs; k += PL_RUNS) {
        int to[PL_RUNS], n[PL_RUNS], page[PL_RUNS];
#pragma unroll
        for (int u = 0; u < PL_RUNS; ++u) {
          const int i = min(k + u, runs - 1);
          const int from = __builtin_amdgcn_readlane(mine.from, i);
          to[u] = __builtin_amdgcn_readlane(mine.to, i);
          n[u] = k + u < runs ? __builtin_amdgcn_readlane(mine.n, i) : 0;
          page[u] = lane < n[u] ? a.table[(uint32_t)(from + lane)] : -1;
        }
#pragma unroll
        for (int u = 0; u < PL_RUNS; ++u)
          if (lane < n[u]) put(a.table + (uint32_t)(to[u] + lane), page[u]);
      }
    }
  };

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
  int taken = 0, taken_entries = 0, less = 0;
  for (int s0 = 0; s0 < a.S; s0 += THREADS) {
    const int s = s0 + tid;
    int pages = 0;
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
      int runs = (pages + WAVE - 1) / WAVE;
      scan_two<WAVES>(runs, pages, taken, taken_entries, tmp);
      if (s < a.S) upto[s] = runs;
    }
  }
  count_in_lds(taken_entries);
  less = __syncthreads_or(less);
  if (taken > 0) {
    const bool here = in_lds && taken_entries < PL_MOST;
    for_runs(taken,
             [&](int s, int k) -> Run {
               const int e = k * WAVE;
               return {a.parent[s] * a.per_seq + e, s * a.per_seq + e, min(a.size.quotient(rows[s]) - e, WAVE)};
             },
             [&](int32_t* at, int page) {
               const bool is = a.is_page(page);
               *at = is ? page : -1;
               if (is) change(page, 1, here);
             });
    memory_barrier();
  }

  // ---- pages that hold no row any more are given back ----
  if (less) {
    int given = 0, given_entries = 0;
    for (int s0 = 0; s0 < a.S; s0 += THREADS) {
      const int s = s0 + tid;
      int pages = 0;
      if (s < a.S && a.n_new[s] < 0)
        pages = max(0, min(a.pages_of(rows[s]), a.per_seq) - a.pages_of(after(s, a.n_new[s])));
      int n = (pages + WAVE - 1) / WAVE;
      scan_two<WAVES>(n, pages, given, given_entries, tmp);
      if (s < a.S) upto[s] = n;
    }
    count_in_lds(given_entries);
    const bool here = in_lds && given_entries < PL_MOST;
    __syncthreads();
    for_runs(given,
             [&](int s, int k) -> Run {
               const int e = a.pages_of(after(s, a.n_new[s])) + k * WAVE, at = s * a.per_seq + e;
               return {at, at, min(min(a.pages_of(rows[s]), a.per_seq) - e, WAVE)};
             },
             [&](int32_t* at, int page) {
               *at = -1;
               if (a.is_page(page)) change(page, -1, here);
             });
    memory_barrier();
  }

  // ---- what was counted in LDS, eight pages a thread; nobody else changes counts now ----
  if (in_lds) {
    constexpr int EACH = 2;
    for (int i0 = tid; i0 * 8 < counted; i0 += EACH * THREADS) {
      int4 d[EACH], c[EACH][2];
      auto whole = [&](int i) { return i * 8 + 7 < counted; };
      auto some = [&](int u) { return (d[u].x | d[u].y | d[u].z | d[u].w) != 0; };
      auto add = [](int4 c, int x, int y) {
        const int x0 = (short)x, y0 = (short)y;
        return make_int4(c.x + x0, c.y + ((x - x0) >> 16), c.z + y0, c.w + ((y - y0) >> 16));
      };
#pragma unroll
      for (int u = 0; u < EACH; ++u) {
        const int i = i0 + u * THREADS;
        d[u] = i * 8 < counted ? changes[i] : make_int4(0, 0, 0, 0);
        if (some(u) && whole(i)) {
          const int4* at = reinterpret_cast<const int4*>(a.refs + 8 * i);
          c[u][0] = at[0];
          c[u][1] = at[1];
        }
      }
#pragma unroll
      for (int u = 0; u < EACH; ++u) {
        const int i = i0 + u * THREADS;
        if (!some(u)) continue;
        if (whole(i)) {
          int4* at = reinterpret_cast<int4*>(a.refs + 8 * i);
          at[0] = add(c[u][0], d[u].x, d[u].y);
          at[1] = add(c[u][1], d[u].z, d[u].w);
        } else {                                        // the last pages
          const int w[4] = {d[u].x, d[u].y, d[u].z, d[u].w};
          for (int k = 0; k < 4; ++k) {
            const int even = (short)w[k], odd = (w[k] - even) >> 16;
            if (even) a.refs[8 * i + 2 * k] += even;    // there are no changes of pages that are not
            if (odd) a.refs[8 * i + 2 * k + 1] += odd;
          }
        }
      }
    }
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
    int n = run ? free_upto[tid] : 0, zero = 0, unused = 0;
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
    hipLaunchKernelGGL((k_plan_pages<PL_FEW, PL_COUNTED>), dim3(1), dim3(PL_FEW), (size_t)S * 2 * sizeof(int), st, a);
  else if (S <= PL_COUNTED_S)
    hipLaunchKernelGGL((k_plan_pages<PL_MANY, PL_COUNTED>), dim3(1), dim3(PL_MANY), (size_t)S * 2 * sizeof(int), st, a);
  else
    hipLaunchKernelGGL((k_plan_pages<PL_MANY, PL_COUNTED_MANY>), dim3(1), dim3(PL_MANY), (size_t)S * 2 * sizeof(int), st, a);
  if (a.slots && n_rows > PL_OWN_ROWS)
    hipLaunchKernelGGL(k_plan_slots, dim3((unsigned)((n_rows + PL_SLOT_ROWS - 1) / PL_SLOT_ROWS)), dim3(PL_MANY),
                       (size_t)S * sizeof(int), st, a);
  return hipGetLastError();
}

}  // namespace ck
