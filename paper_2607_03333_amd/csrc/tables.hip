// gfx950 kernels that keep block tables on the GPU: one step takes every row
// from the tokens it had to the tokens it now has (rollback, fork, append) and
// gives each new token its slot, from lengths that only the device knows.
//
// The rules are the host block manager's (block_manager.h), run over a batch:
// with b(x) = ceil(x / block_size),
//   forks     row s of parent p becomes the first b(len s) entries of row p;
//   releases  in row and table order, the entries of a row behind its first
//             b(len s), and all old entries of a forked row; a block without
//             references goes to the back of the free queue;
//   appends   in row order: a row that appends inside a block which others hold
//             takes a copy target from the queue's front, then every block that
//             it opens takes the next front.
// Done in that order by one thread this is a chain of queue operations; what
// makes it parallel is that only three things depend on the order, and each has
// a closed form: a freed block is put into the queue by the last place that
// releases it, its rank there is a prefix sum; of k rows that append inside a
// block of r references all copy it, except that the last one writes in place
// where k = r; and the fronts that a row takes start at a prefix sum. Counts
// and last places go through atomics whose order does not matter (sums, maxima),
// so the same step gives the same tables every time.
//
// Four launches: count (references and last places), rows (what each row frees and
// takes), release (the sums over the rows and whether the step fits; frees into
// the queue, forked rows, copies), assign (fronts into the tables, slots). The
// references are changed while they are counted, and changed back where the step
// is refused. A workgroup per row, and four entries of its row in flight per
// thread: a fork or the end of a long row is thousands of entries. Up to
// kRowsSummedByAll rows every workgroup of release sums what it needs by itself;
// more are summed once, by a launch between. Few short rows go through the same
// phases in one workgroup and one launch (tables_one), a row to a wave.
#include "device_common.h"
#include "spork.h"
#include "tables_kernels.h"
#include "wave_scan.h"

namespace spork {
namespace {

constexpr int kRowThreads = 256;   // of a row's workgroup
constexpr int kSumThreads = 1024;  // of the one workgroup that sums the rows
constexpr int kAtOnce = 4;         // entries of a row that a thread loads together
// One token for each row, eager and in a graph, summed by all against a launch: 256
// rows 18.7 and 12.8 us against 19.8 and 13.7, 1,024 18.1 and 17.4 against 19.5 and
// 17.8, 2,048 25.3 and 25.4 against 25.1 and 24.9, 4,096 41 against 38.
constexpr int kRowsSummedByAll = 1024;
// Steps of one workgroup: at most so many rows (a wave each), entries of a row,
// and new tokens. Half of the rows forking again, eager and in a graph, one launch
// against four: 1 row 9.0 and 8.4 us against 16.0 and 9.3; 8 rows of 250 tokens 11.5
// and 11.8 against 16.9 and 15.1; 16 rows 12.6 and 12.9 against 17.1 and 14.8; 16 rows
// of 500 blocks 13.2 and 13.5 against 17.1 and 13.4, of 1,000 blocks 19.1 and 19.4
// against 17.1 and 13.5; 4,096 new tokens 10.7 and 10.9 against 17.0 and 13.0. Long
// rows gain where they append one token (4 rows of 2,000 entries 12.4 and 9.4 against
// 21.2 and 12.2, of 8,100 12.2 and 9.4 against 21.1 and 12.3) and lose more where they
// fork (22.6 and 22.8 against 21.7 and 15.3; 69 against 30) or end, each step alone
// (of 500 entries 29 against 27, of 2,000 69 against 34, of 8,100 210 against 72).
// What a step does only the GPU knows, so the limit is on what a row can hold.
constexpr int kOneThreads = 1024;
constexpr int kOneRows = 16, kOneEntries = 512, kOneTokens = 4096;
static_assert(kOneRows * 64 == kOneThreads, "a wave for every row");

struct Row {
  int len, grow, parent, held;
  int keep;        // blocks of the tokens that stay
  int from;        // row that those blocks stand in
  int release_lo;  // first entry of the old row that is released
  int tail;        // block that the row appends into behind tokens that stay, or -1
};

__device__ __forceinline__ int blocks_of(int64_t tokens, int bs) { return static_cast<int>((tokens + bs - 1) / bs); }

__device__ __forceinline__ size_t place(const TablesArgs& a, int s, int col) {
  return static_cast<size_t>(s) * a.max_blocks + col;
}

// Row s as the step asks for it, and the status of that: its fields are used
// only where it is SPORK_OK, and then every index that follows from them is in
// range, entries of the tables apart.
__device__ __forceinline__ int read_row(const TablesArgs& a, int s, Row* r) {
  r->len = a.lens[s];
  r->grow = a.n_new[s];
  r->held = a.held[s];
  r->parent = a.parents != nullptr ? a.parents[s] : -1;
  if (r->len < 0 || r->grow < 0 || r->held < 0 || r->held > a.max_blocks || r->parent >= a.n_seqs) return SPORK_E_INVAL;
  if (r->parent < 0) r->parent = -1;
  int have = r->held;
  if (r->parent >= 0) {
    if (r->parent == s || a.parents[r->parent] >= 0) return SPORK_E_INVAL;
    have = a.held[r->parent];
    if (have < 0 || have > a.max_blocks) return SPORK_E_INVAL;
  }
  const int64_t end = static_cast<int64_t>(r->len) + r->grow;
  if (blocks_of(r->len, a.block_size) > have) return SPORK_E_INVAL;
  if (end > static_cast<int64_t>(a.max_blocks) * a.block_size) return SPORK_E_CAPACITY;
  r->keep = blocks_of(r->len, a.block_size);
  r->from = r->parent >= 0 ? r->parent : s;
  r->release_lo = r->parent >= 0 ? 0 : r->keep;
  r->tail = r->grow == 0 || r->len % a.block_size == 0 ? -1 : a.table[place(a, r->from, r->len / a.block_size)];
  return SPORK_OK;
}

__device__ __forceinline__ bool in_pool(const TablesArgs& a, int block) { return block >= 0 && block < a.num_blocks; }

// What forks and releases change in the columns of table row s from column j0 on,
// kAtOnce of them per thread: the entry that was there and the one that comes.
struct Changes {
  int was[kAtOnce], now[kAtOnce];
  bool loses[kAtOnce], gains[kAtOnce];
};
__device__ __forceinline__ int changes_lo(const Row& r) { return r.release_lo; }
__device__ __forceinline__ int changes_hi(const Row& r) { return r.parent >= 0 ? max(r.held, r.keep) : r.held; }
// kTeam: threads that work on a row, a workgroup or a wave.
template <int kTeam>
__device__ __forceinline__ int column(int j0, int q) {
  return j0 + q * kTeam + static_cast<int>(threadIdx.x % kTeam);
}
template <int kTeam>
__device__ __forceinline__ Changes changes(const TablesArgs& a, int s, const Row& r, int j0) {
  Changes x;
#pragma unroll
  for (int q = 0; q < kAtOnce; ++q) {
    const int j = column<kTeam>(j0, q);
    x.loses[q] = j < r.held;
    x.gains[q] = r.parent >= 0 && j < r.keep;
    x.was[q] = x.loses[q] ? a.table[place(a, s, j)] : -1;
    x.now[q] = x.gains[q] ? a.table[place(a, r.parent, j)] : -1;
  }
  // An entry that a fork gives and takes at once stays as it is: a probe that forks
  // again where it forked before, a few tokens on. (The block keeps this holder, so
  // leaving out one reference more and one less frees nothing and keeps nothing.)
#pragma unroll
  for (int q = 0; q < kAtOnce; ++q)
    if (x.loses[q] && x.gains[q] && x.was[q] == x.now[q] && in_pool(a, x.was[q])) x.loses[q] = x.gains[q] = false;
  return x;
}

// References and last places of a row's changes (`head`: the first of them, of each
// thread kAtOnce); the status of its entries.
template <int kTeam>
__device__ __forceinline__ int count_row(const TablesArgs& a, int s, const Row& r, const Changes& head) {
  int err = SPORK_OK;
  for (int j0 = changes_lo(r); j0 < changes_hi(r); j0 += kAtOnce * kTeam) {
    const Changes x = j0 == changes_lo(r) ? head : changes<kTeam>(a, s, r, j0);
#pragma unroll
    for (int q = 0; q < kAtOnce; ++q) {
      if (x.gains[q]) {
        if (in_pool(a, x.now[q])) atomicAdd(a.refcount + x.now[q], 1);
        else err = SPORK_E_INVAL;
      }
      if (x.loses[q]) {
        if (in_pool(a, x.was[q])) {
          atomicAdd(a.refcount + x.was[q], -1);
          atomicMax(a.last_release + x.was[q], static_cast<int>(place(a, s, column<kTeam>(j0, q))) + 1);
        } else {
          err = SPORK_E_INVAL;
        }
      }
    }
  }
  if (threadIdx.x % kTeam == 0 && r.grow != 0 && r.len % a.block_size != 0) {
    if (in_pool(a, r.tail)) {
      atomicAdd(a.sharers + r.tail, 1);
      atomicMax(a.last_sharer + r.tail, s + 1);
    } else {
      err = SPORK_E_INVAL;
    }
  }
  return err;
}

__global__ void __launch_bounds__(kRowThreads) tables_count(TablesArgs a) {
  const int s = blockIdx.x;
  if (s == 0 && threadIdx.x == 0) a.totals->front = a.queue[0];
  Row r;
  int err = read_row(a, s, &r);
  if (err == SPORK_OK) err = count_row<kRowThreads>(a, s, r, changes<kRowThreads>(a, s, r, changes_lo(r)));
  if (err != SPORK_OK) atomicMin(&a.totals->error, err);
}

// Whether place (s, j) is the one that frees block b.
__device__ __forceinline__ bool frees_block(const TablesArgs& a, int s, int j, int b) {
  return in_pool(a, b) && a.last_release[b] == static_cast<int>(place(a, s, j)) + 1 && a.refcount[b] == 0;
}

// Whether row s, which appends inside a block, copies it.
__device__ __forceinline__ int copies_tail(const TablesArgs& a, int s, const Row& r) {
  if (!in_pool(a, r.tail)) return 0;
  const int refs = a.refcount[r.tail], sharers = a.sharers[r.tail], last = a.last_sharer[r.tail];
  return refs > 1 && !(sharers == refs && last == s + 1);
}

// Blocks that the thread's entries of row s free, summed over its wave.
template <int kTeam>
__device__ __forceinline__ int wave_frees(const TablesArgs& a, int s, const Row& r, const Changes& head) {
  int frees = 0;
  for (int j0 = changes_lo(r); j0 < changes_hi(r); j0 += kAtOnce * kTeam) {
    const Changes x = j0 == changes_lo(r) ? head : changes<kTeam>(a, s, r, j0);
#pragma unroll
    for (int q = 0; q < kAtOnce; ++q) frees += x.loses[q] && frees_block(a, s, column<kTeam>(j0, q), x.was[q]);
  }
#pragma unroll
  for (int o = 32; o >= 1; o /= 2) frees += __shfl_xor(frees, o);
  return frees;
}

__device__ __forceinline__ int row_takes(const TablesArgs& a, const Row& r, int copies) {
  return copies + blocks_of(static_cast<int64_t>(r.len) + r.grow, a.block_size) - r.keep;
}

__global__ void __launch_bounds__(kRowThreads) tables_rows(TablesArgs a) {
  __shared__ int freed[kRowThreads / 64];
  const int s = blockIdx.x, tid = threadIdx.x;
  Row r;
  if (read_row(a, s, &r) != SPORK_OK) {  // the step is refused
    if (tid == 0) a.frees[s] = a.takes[s] = a.copies_of[s] = 0;
    return;
  }
  const int copies = tid == 0 ? copies_tail(a, s, r) : 0;
  int frees = 0;
  if (changes_lo(r) < changes_hi(r)) {
    frees = wave_frees<kRowThreads>(a, s, r, changes<kRowThreads>(a, s, r, changes_lo(r)));
    if ((tid & 63) == 0) freed[tid >> 6] = frees;
    __syncthreads();
    frees = 0;
#pragma unroll
    for (int w = 0; w < kRowThreads / 64; ++w) frees += freed[w];
  }
  if (tid == 0) {
    a.frees[s] = frees;
    a.takes[s] = row_takes(a, r, copies);
    a.copies_of[s] = copies;
  }
}

// What a row adds to the sums.
struct Sums {
  int64_t tokens;
  int frees, takes, copies;
};
__device__ __forceinline__ Sums operator+(const Sums& x, const Sums& y) {
  return {x.tokens + y.tokens, x.frees + y.frees, x.takes + y.takes, x.copies + y.copies};
}
__device__ __forceinline__ Sums row_sums(const TablesArgs& a, int i) {
  return {max(a.n_new[i], 0), a.frees[i], a.takes[i], a.copies_of[i]};
}

// The step's status, from the sums over all rows.
__device__ __forceinline__ int status_of(const TablesArgs& a, const Sums& all, int error, int front, int count) {
  int status = error;
  if (front < 0 || front >= a.num_blocks || count < 0 || count > a.num_blocks - all.frees) status = min(status, SPORK_E_INVAL);
  if (all.tokens > a.max_tokens) status = min(status, SPORK_E_CAPACITY);
  if (status == SPORK_OK && all.takes > count + all.frees) status = SPORK_E_NOBLOCKS;
  return status;
}

__device__ __forceinline__ void write_row_sums(const TablesArgs& a, int i, const Sums& before, const Sums& own) {
  a.take_off[i] = before.takes;
  a.copy_off[i] = own.copies ? before.copies : -1;
  a.row_off[i + 1] = static_cast<int>(min(before.tokens + own.tokens, static_cast<int64_t>(INT_MAX)));
  if (i == 0) a.row_off[0] = 0;
}

__device__ __forceinline__ void write_totals(const TablesArgs& a, const Sums& all, int status) {
  a.totals->status = status;
  a.totals->frees = all.frees;
  a.totals->takes = all.takes;
  *a.status = status;
  *a.n_copies = status == SPORK_OK ? all.copies : 0;
}

__global__ void __launch_bounds__(kSumThreads) tables_sum(TablesArgs a) {
  constexpr int kWaves = kSumThreads / 64;
  __shared__ Sums wave_sums[2][kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int front = a.queue[0], count = a.queue[1], error = a.totals->error;
  Sums done{0, 0, 0, 0};
  for (int s0 = 0, odd = 0; s0 < a.n_seqs; s0 += kSumThreads, odd ^= 1) {
    const int i = s0 + tid;
    Sums x{0, 0, 0, 0};
    if (i < a.n_seqs) x = row_sums(a, i);
    const Sums upto{wave_scan(x.tokens), wave_scan(x.frees), wave_scan(x.takes), wave_scan(x.copies)};
    if (lane == 63) wave_sums[odd][wave] = upto;
    __syncthreads();  // (the other half is free again once everybody is here)
    Sums before = done + Sums{upto.tokens - x.tokens, upto.frees - x.frees, upto.takes - x.takes, upto.copies - x.copies};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const Sums y = wave_sums[odd][w];
      if (w < wave) before = before + y;
      done = done + y;
    }
    if (i < a.n_seqs) {
      a.free_off[i] = before.frees;
      write_row_sums(a, i, before, x);
    }
  }
  if (tid == 0) write_totals(a, done, status_of(a, done, error, front, count));
}

// The same within a workgroup of release: the sums before row s and over all rows.
__device__ __forceinline__ void sum_here(const TablesArgs& a, int s, Sums* before, Sums* all) {
  constexpr int kWaves = kRowThreads / 64;
  __shared__ Sums parts[2][kWaves];
  const int tid = threadIdx.x;
  Sums lo{0, 0, 0, 0}, hi = lo;
  for (int i = tid; i < a.n_seqs; i += kRowThreads) {
    const Sums x = row_sums(a, i);
    if (i < s) lo = lo + x;
    else hi = hi + x;
  }
  lo = {wave_scan(lo.tokens), wave_scan(lo.frees), wave_scan(lo.takes), wave_scan(lo.copies)};
  hi = {wave_scan(hi.tokens), wave_scan(hi.frees), wave_scan(hi.takes), wave_scan(hi.copies)};
  if ((tid & 63) == 63) {
    parts[0][tid >> 6] = lo;
    parts[1][tid >> 6] = hi;
  }
  __syncthreads();
  *before = *all = {0, 0, 0, 0};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    *before = *before + parts[0][w];
    *all = *all + parts[0][w] + parts[1][w];
  }
}

// Place in the ring of the nth entry (at most num_blocks) from the front.
__device__ __forceinline__ int ring(const TablesArgs& a, int front, int nth) {
  const uint32_t at = static_cast<uint32_t>(front) + static_cast<uint32_t>(nth), n = static_cast<uint32_t>(a.num_blocks);
  return static_cast<int>(at >= n ? at - n : at);
}

// Row s of a refused step: its references back, its words clear.
template <int kTeam>
__device__ __forceinline__ void undo_row(const TablesArgs& a, int s, const Row& r) {
  for (int j0 = changes_lo(r); j0 < changes_hi(r); j0 += kAtOnce * kTeam) {
    const Changes x = changes<kTeam>(a, s, r, j0);
#pragma unroll
    for (int q = 0; q < kAtOnce; ++q) {
      if (x.gains[q] && in_pool(a, x.now[q])) atomicAdd(a.refcount + x.now[q], -1);
      if (x.loses[q] && in_pool(a, x.was[q])) {
        atomicAdd(a.refcount + x.was[q], 1);
        a.last_release[x.was[q]] = 0;
      }
    }
  }
  if (threadIdx.x % kTeam == 0) {
    if (in_pool(a, r.tail)) a.sharers[r.tail] = a.last_sharer[r.tail] = 0;
  }
}

// The frees of row s into the queue, behind `at` others, and a forked row's
// entries; its copy's entry (c: index of it, or -1).
template <int kTeam>
__device__ __forceinline__ void release_row(const TablesArgs& a, int s, const Row& r, const Changes& head, int at, int c, int front,
                                            int count) {
  constexpr int kTeamWaves = kTeam / 64;
  __shared__ int freed[kAtOnce][kTeamWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x % kTeam >> 6;
  for (int j0 = changes_lo(r); j0 < changes_hi(r); j0 += kAtOnce * kTeam) {
    const Changes x = j0 == changes_lo(r) ? head : changes<kTeam>(a, s, r, j0);
    bool here[kAtOnce];
#pragma unroll
    for (int q = 0; q < kAtOnce; ++q) here[q] = x.loses[q] && frees_block(a, s, column<kTeam>(j0, q), x.was[q]);
#pragma unroll
    for (int q = 0; q < kAtOnce; ++q) {
      const int place1 = static_cast<int>(place(a, s, column<kTeam>(j0, q))) + 1;
      // The last place alone clears the word: any other compares unequal before and after.
      if (x.loses[q] && a.last_release[x.was[q]] == place1) a.last_release[x.was[q]] = 0;
      if (x.gains[q]) a.table[place1 - 1] = x.now[q];  // (this thread alone reads the column)
      if constexpr (kTeamWaves > 1) {
        const uint64_t bal = __ballot(here[q]);
        if (lane == 0) freed[q][wave] = __popcll(bal);
      }
    }
    if constexpr (kTeamWaves > 1) __syncthreads();
#pragma unroll
    for (int q = 0; q < kAtOnce; ++q) {
      const uint64_t bal = __ballot(here[q]);
      int rank = at + __popcll(bal & ((uint64_t{1} << lane) - 1));
      if constexpr (kTeamWaves > 1) {
#pragma unroll
        for (int w = 0; w < kTeamWaves; ++w) {
          if (w < wave) rank += freed[q][w];
          at += freed[q][w];
        }
      } else {
        at += __popcll(bal);
      }
      if (here[q]) a.free_queue[ring(a, front, count + rank)] = x.was[q];
    }
    if constexpr (kTeamWaves > 1) __syncthreads();  // the counts are read
  }
  if (threadIdx.x % kTeam == 0) {
    if (r.tail >= 0) a.sharers[r.tail] = a.last_sharer[r.tail] = 0;
    if (c >= 0) {
      a.copies[3 * c] = r.tail;
      a.copies[3 * c + 2] = r.len % a.block_size;
    }
  }
}

// kSummed: by tables_sum.
template <bool kSummed>
__global__ void __launch_bounds__(kRowThreads) tables_release(TablesArgs a) {
  const int s = blockIdx.x, tid = threadIdx.x;
  const int front = a.queue[0], count = a.queue[1];
  int at, c, status;  // the row's freed blocks among all, its copy or -1
  if constexpr (kSummed) {
    at = a.free_off[s];
    c = a.copy_off[s];
    status = a.totals->status;
  } else {
    const int error = a.totals->error;
    Sums before, all;
    sum_here(a, s, &before, &all);
    status = status_of(a, all, error, front, count);
    at = before.frees;
    c = a.copies_of[s] ? before.copies : -1;
    if (tid == 0) {
      write_row_sums(a, s, before, row_sums(a, s));
      if (s == 0) write_totals(a, all, status);
    }
  }
  Row r;
  if (read_row(a, s, &r) != SPORK_OK) return;
  if (status != SPORK_OK) undo_row<kRowThreads>(a, s, r);
  else release_row<kRowThreads>(a, s, r, changes<kRowThreads>(a, s, r, changes_lo(r)), at, c, front, count);
}

// The fronts of row s, from the queue's nth on, into its table; its references
// and length (c as above; src: the block that is copied).
template <int kTeam>
__device__ __forceinline__ void assign_row(const TablesArgs& a, int s, int front, int nth, int c, int src) {
  const int tid = threadIdx.x % kTeam, bs = a.block_size;
  const int len = a.lens[s], end = len + a.n_new[s], keep = blocks_of(len, bs), to = blocks_of(end, bs);
  if (c >= 0) {
    if (tid == 0) {
      const int dst = a.free_queue[ring(a, front, nth)];
      atomicAdd(a.refcount + src, -1);
      a.copies[3 * c + 1] = dst;
      if (in_pool(a, dst)) a.refcount[dst] = 1;
      a.table[place(a, s, len / bs)] = dst;
    }
    ++nth;
  }
  for (int j = keep + tid; j < to; j += kTeam) {
    const int b = a.free_queue[ring(a, front, nth + j - keep)];
    a.table[place(a, s, j)] = b;
    if (in_pool(a, b)) a.refcount[b] = 1;  // (the queue's contents are the caller's)
  }
  if (tid == 0) {
    a.held[s] = to;
    a.kv_len[s] = end;
  }
}

// Slot and position of the nth new token of row s: its block from the queue or,
// in front of the row's first new block, from the tail or its copy.
__device__ __forceinline__ int64_t slot_of(const TablesArgs& a, int s, int len, int nth, int front, int take_off, int c,
                                          int* pos) {
  const int bs = a.block_size, keep = blocks_of(len, bs);
  *pos = len + nth;
  const int col = *pos / bs;
  int b;
  if (col >= keep) b = a.free_queue[ring(a, front, take_off + (c >= 0 ? 1 : 0) + col - keep)];
  else if (c >= 0) b = a.free_queue[ring(a, front, take_off)];
  else b = a.table[place(a, s, col)];
  return static_cast<int64_t>(b) * bs + *pos % bs;
}

__global__ void __launch_bounds__(kRowThreads) tables_assign(TablesArgs a) {
  const int tid = threadIdx.x;
  const int status = a.totals->status, front = a.totals->front;
  if (static_cast<int>(blockIdx.x) < a.n_seqs) {  // a row: its table and references
    const int s = blockIdx.x;
    if (s == 0 && tid == 0) {
      if (status == SPORK_OK) {
        const TablesTotals t = *a.totals;
        a.queue[0] = ring(a, front, t.takes);
        a.queue[1] += t.frees - t.takes;
      }
      a.totals->error = 0;
    }
    if (status != SPORK_OK) {
      if (tid == 0) {
        a.row_off[s + 1] = 0;
        a.kv_len[s] = 0;
      }
      return;
    }
    const int c = a.copy_off[s];
    assign_row<kRowThreads>(a, s, front, a.take_off[s], c, c >= 0 ? a.copies[3 * c] : -1);
    return;
  }
  // a token: its row by search in the offsets
  const int i = (static_cast<int>(blockIdx.x) - a.n_seqs) * kRowThreads + tid;
  if (i >= a.max_tokens) return;
  int64_t slot = -1;
  int pos = -1;
  if (status == SPORK_OK && i < a.row_off[a.n_seqs]) {
    int lo = 0, hi = a.n_seqs - 1;  // the last row that starts at or before token i
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.row_off[mid] <= i) lo = mid;
      else hi = mid - 1;
    }
    slot = slot_of(a, lo, a.lens[lo], i - a.row_off[lo], front, a.take_off[lo], a.copy_off[lo], &pos);
  }
  a.slots[i] = slot;
  if (a.positions != nullptr) a.positions[i] = pos;
}

// The whole step in one workgroup: a row to a wave, the sums over the rows in
// every wave's lanes. What the launches above leave each other in the workspace
// is in LDS here; block words, queue and tables go through L2, past which a
// phase's changes are waited for.
__device__ __forceinline__ void settle() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // this wave's stores and atomics have arrived
  __syncthreads();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");  // nothing older is read from the first-level cache
}

__global__ void __launch_bounds__(kOneThreads) tables_one(TablesArgs a) {
  __shared__ int error;
  __shared__ int frees_of[kOneRows], takes_of[kOneRows], copies_of[kOneRows], take_off[kOneRows], copy_off[kOneRows], len_of[kOneRows],
      row_off[kOneRows + 1];
  const int tid = threadIdx.x, lane = tid & 63, n = a.n_seqs;
  const int s = __builtin_amdgcn_readfirstlane(tid >> 6);  // the wave's row
  const int front = a.queue[0], count = a.queue[1];
  if (tid == 0) error = SPORK_OK;
  __syncthreads();
  Row r;
  Changes head;  // (the tables change only behind the last use)
  bool sound = false;
  if (s < n) {
    int err = read_row(a, s, &r);
    sound = err == SPORK_OK;
    if (sound) {
      head = changes<64>(a, s, r, changes_lo(r));
      err = count_row<64>(a, s, r, head);
    }
    if (err != SPORK_OK) atomicMin(&error, err);
  }
  settle();
  if (s < n) {
    int copies = 0, frees = 0, takes = 0;
    if (sound) {  // (else the step is refused)
      copies = copies_tail(a, s, r);
      frees = wave_frees<64>(a, s, r, head);
      takes = row_takes(a, r, copies);
    }
    if (lane == 0) {
      frees_of[s] = frees;
      takes_of[s] = takes;
      copies_of[s] = copies;
    }
  }
  __syncthreads();
  Sums x{0, 0, 0, 0};
  if (lane < n) x = {max(a.n_new[lane], 0), frees_of[lane], takes_of[lane], copies_of[lane]};
  const Sums upto{wave_scan(x.tokens), wave_scan(x.frees), wave_scan(x.takes), wave_scan(x.copies)};
  const Sums all{static_cast<int64_t>(__shfl(static_cast<long long>(upto.tokens), 63)), __shfl(upto.frees, 63),
                 __shfl(upto.takes, 63), __shfl(upto.copies, 63)};
  const int status = status_of(a, all, error, front, count);
  const bool fits = status == SPORK_OK;
  const int copy = x.copies ? upto.copies - x.copies : -1;
  if (s == 0) {
    if (lane < n) {
      take_off[lane] = upto.takes - x.takes;
      copy_off[lane] = copy;
      len_of[lane] = a.lens[lane];
      row_off[lane + 1] = a.row_off[lane + 1] = fits ? static_cast<int>(upto.tokens) : 0;
      if (!fits) a.kv_len[lane] = 0;
    }
    if (lane == 0) {
      row_off[0] = a.row_off[0] = 0;
      *a.status = status;
      *a.n_copies = fits ? all.copies : 0;
    }
  }
  if (sound) {
    const int at = __shfl(upto.frees - x.frees, s), c = __shfl(copy, s);
    if (fits) release_row<64>(a, s, r, head, at, c, front, count);
    else undo_row<64>(a, s, r);
  }
  settle();
  if (fits) {
    if (tid == 0) {
      a.queue[0] = ring(a, front, all.takes);
      a.queue[1] = count + all.frees - all.takes;
    }
    if (s < n) assign_row<64>(a, s, front, take_off[s], copy_off[s], r.tail);
  }
  for (int i = tid; i < a.max_tokens; i += kOneThreads) {
    int64_t slot = -1;
    int pos = -1;
    if (i < row_off[n]) {  // (0 where the step is refused)
      int lo = 0, hi = n - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (row_off[mid] <= i) lo = mid;
        else hi = mid - 1;
      }
      slot = slot_of(a, lo, len_of[lo], i - row_off[lo], front, take_off[lo], copy_off[lo], &pos);
    }
    a.slots[i] = slot;
    if (a.positions != nullptr) a.positions[i] = pos;
  }
}

__global__ void __launch_bounds__(256) tables_init_kernel(TablesArgs a, const int32_t* free_order) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < a.num_blocks) {
    a.free_queue[i] = free_order != nullptr ? free_order[i] : i;
    a.refcount[i] = 0;
  }
  if (i < a.n_seqs) a.held[i] = 0;
  if (i == 0) {
    a.queue[0] = 0;
    a.queue[1] = a.num_blocks;
  }
}

__global__ void __launch_bounds__(256) words_clear_kernel(int32_t* words, int64_t n) {
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * 256)
    words[i] = 0;
}

// The copies of copy-on-write, from the list that a step wrote: a workgroup per
// (copy, KV head). K: the first n_valid tokens are one run of bytes. V: of each
// channel's run of block_size elements the first n_valid, 16 bytes at a time but
// for the last ones.
template <typename T>
__global__ void __launch_bounds__(256) kv_copy_batch_kernel(int hkv, int D, int BS, int num_blocks, T* kc, T* vc,
                                                            const int32_t* copies, const int32_t* n_copies, int max_copies) {
  constexpr int VEC = 16 / sizeof(T);
  const int c = blockIdx.x / hkv, h = blockIdx.x % hkv;
  if (c >= min(*n_copies, max_copies)) return;
  const int src = copies[3 * c], dst = copies[3 * c + 1], nv = copies[3 * c + 2];
  if (src < 0 || src >= num_blocks || dst < 0 || dst >= num_blocks || src == dst || nv <= 0 || nv > BS) return;
  const size_t size = static_cast<size_t>(D) * BS;
  const size_t from = (static_cast<size_t>(src) * hkv + h) * size, to = (static_cast<size_t>(dst) * hkv + h) * size;
  const uint4* ks = reinterpret_cast<const uint4*>(kc + from);
  uint4* kd = reinterpret_cast<uint4*>(kc + to);
  for (int i = threadIdx.x; i < nv * (D / VEC); i += 256) kd[i] = ks[i];
  const T* vs = vc + from;
  T* vd = vc + to;
  if (BS % VEC == 0) {
    const int pieces = BS / VEC;  // of a channel
    for (int i = threadIdx.x; i < D * pieces; i += 256) {
      const int n = nv - i % pieces * VEC;
      if (n >= VEC) {
        reinterpret_cast<uint4*>(vd)[i] = reinterpret_cast<const uint4*>(vs)[i];
      } else {
        for (int e = 0; e < n; ++e) vd[i * VEC + e] = vs[i * VEC + e];
      }
    }
  } else {
    for (int i = threadIdx.x; i < D * BS; i += 256)
      if (i % BS < nv) vd[i] = vs[i];
  }
}

}  // namespace

size_t tables_control_bytes(int32_t num_blocks) {
  return sizeof(TablesTotals) + (3 * sizeof(int32_t) * static_cast<size_t>(num_blocks) + 255) / 256 * 256;
}

size_t tables_workspace_bytes(int32_t num_blocks, int32_t n_seqs) {
  return tables_control_bytes(num_blocks) + 6 * sizeof(int32_t) * static_cast<size_t>(n_seqs);
}

void tables_workspace(TablesArgs* a, void* workspace) {
  a->totals = static_cast<TablesTotals*>(workspace);
  a->last_release = reinterpret_cast<int32_t*>(a->totals + 1);
  a->sharers = a->last_release + a->num_blocks;
  a->last_sharer = a->sharers + a->num_blocks;
  a->frees = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + tables_control_bytes(a->num_blocks));
  a->takes = a->frees + a->n_seqs;
  a->copies_of = a->takes + a->n_seqs;
  a->free_off = a->copies_of + a->n_seqs;
  a->take_off = a->free_off + a->n_seqs;
  a->copy_off = a->take_off + a->n_seqs;
}

hipError_t launch_tables_init(const TablesArgs& a, const int32_t* free_order, hipStream_t stream) {
  const int n = a.num_blocks > a.n_seqs ? a.num_blocks : a.n_seqs;
  hipLaunchKernelGGL(tables_init_kernel, dim3((static_cast<unsigned>(n) + 255) / 256), dim3(256), 0, stream, a, free_order);
  return hipGetLastError();
}

hipError_t launch_words_clear(int32_t* words, int64_t n, hipStream_t stream) {
  if (n <= 0) return hipSuccess;
  const int64_t blocks = (n + 255) / 256;
  hipLaunchKernelGGL(words_clear_kernel, dim3(static_cast<unsigned>(blocks < 1024 ? blocks : 1024)), dim3(256), 0, stream, words,
                     n);
  return hipGetLastError();
}

hipError_t launch_tables_step(const TablesArgs& a, hipStream_t stream) {
  const unsigned rows = static_cast<unsigned>(a.n_seqs);
  if (a.n_seqs <= kOneRows && a.max_blocks <= kOneEntries && a.max_tokens <= kOneTokens) {
    hipLaunchKernelGGL(tables_one, dim3(1), dim3(kOneThreads), 0, stream, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(tables_count, dim3(rows), dim3(kRowThreads), 0, stream, a);
  hipLaunchKernelGGL(tables_rows, dim3(rows), dim3(kRowThreads), 0, stream, a);
  if (a.n_seqs > kRowsSummedByAll) {
    hipLaunchKernelGGL(tables_sum, dim3(1), dim3(kSumThreads), 0, stream, a);
    hipLaunchKernelGGL(tables_release<true>, dim3(rows), dim3(kRowThreads), 0, stream, a);
  } else {
    hipLaunchKernelGGL(tables_release<false>, dim3(rows), dim3(kRowThreads), 0, stream, a);
  }
  const unsigned tokens = (static_cast<unsigned>(a.max_tokens) + kRowThreads - 1) / kRowThreads;
  hipLaunchKernelGGL(tables_assign, dim3(rows + tokens), dim3(kRowThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_kv_copy_batch(int32_t elem_bytes, int32_t hkv, int32_t head_dim, int32_t block_size, int32_t num_blocks,
                                void* k_cache, void* v_cache, const int32_t* copies, const int32_t* n_copies,
                                int32_t max_copies, hipStream_t stream) {
  if (max_copies <= 0) return hipSuccess;
  const dim3 grid(static_cast<unsigned>(max_copies) * static_cast<unsigned>(hkv));
  if (elem_bytes == 2)
    hipLaunchKernelGGL(kv_copy_batch_kernel<uint16_t>, grid, dim3(256), 0, stream, hkv, head_dim, block_size, num_blocks,
                       static_cast<uint16_t*>(k_cache), static_cast<uint16_t*>(v_cache), copies, n_copies, max_copies);
  else
    hipLaunchKernelGGL(kv_copy_batch_kernel<float>, grid, dim3(256), 0, stream, hkv, head_dim, block_size, num_blocks,
                       static_cast<float*>(k_cache), static_cast<float*>(v_cache), copies, n_copies, max_copies);
  return hipGetLastError();
}

}  // namespace spork
