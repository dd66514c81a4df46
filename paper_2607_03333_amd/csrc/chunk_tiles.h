// What the attentions of a ragged batch's new tokens over a paged cache share
// (chunk.hip, chunk_kvq.hip): the line of tiles and its cut into slices, loads and
// waits of stages, and a workgroup's way through its slice. The stage engines, one
// for each type of queries and cache, are the including files'.
//
//   o_r = sum_{t <= p_r} softmax_t(scale q_r.k_t) v_t,  p_r = kv_len - rows + r
//
// Tiles. The query rows of a sequence times the G query heads of a KV head are
// its packed rows; a tile is up to 256 of them (whole query rows), in row tiles
// of 32, against the positions up to its last row's. A sequence of up to 256
// packed rows is one tile per KV head: then there are row tiles for only some of
// the workgroup's 8 waves, and the others take other tokens of the tile (8, 4 or
// 2 ways), joined through LDS at its end, or other KV heads where the batch has
// tiles enough for every compute unit (chunk_tile_heads).
//
// Slices. All tiles in a row, each as long as it costs (a start-up plus its
// tokens), make a line that is cut into equal slices, one per compute unit. A
// slice computes its place by itself, from a sum over the sequences' lengths, so
// the split costs no launch and no atomics, and the same lengths are always cut
// alike. A tile that a cut goes through has pieces in several slices; every
// slice writes at most two pieces (its first tile's and its last's), so the
// workspace does not grow with the batch. The merge launch joins them by
// log-sum-exp. Neighbouring slices (the row tiles of one sequence and KV head,
// which read the same keys and values) go to one die, whose L2 they share.
#pragma once
#include "chunk_kernels.h"
#include "device_common.h"
#include "wave_scan.h"

namespace spork {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) void* lds_ptr;

constexpr int kWaves = kChunkWaves;
constexpr int kDies = 8;
// Cache policy of keys and values: non-temporal where one wave reads them, kept
// where several row tiles do (24 prompts of up to 777 tokens with 16 heads of 64
// channels, 78 us with non-temporal loads throughout, 69 without).
constexpr int kStream = 2, kKeep = 0;
constexpr float kSlack = 8.0f;       // base-2 headroom before the reference moves: of a score (fp32),
constexpr float kSlackSum = 256.0f;  // of the sum of a lane's probabilities of a stage (bf16)

// The line's unit is half the time that a token of 128 bf16 channels takes where
// HBM bounds it, about 9 ns on one compute unit.
// A tile's start-up and end: 24 prompts of up to 777 tokens with 16 heads of 64
// took 54.5 us at 640, 52.7 at 1,000, 53.1 at 1,400 (three long chunks beside 29
// single tokens 157, 156, 160).
constexpr int kTileCost = 1000;
// Least length of a slice: three fp32 prompts took 47.4 us at 2,048, 33.2 at 1,024,
// 31.3 at 512, 27.8 at 320; one token over 1,000 positions 25.5, 17.8, 16.9, 16.5.
constexpr int kMinSlice = 320;
constexpr int kShortSlice = 256;  // with kShifts
static_assert(kChunkSlices == 256, "slices of a long line by shifts");
// Least cost of a piece: a cut closer to a tile's end moves to it. At 64, 256, 512 and
// 1,024: eight fp32 tokens over up to 1,500 positions 16.9, 18.2, 19.1, 26.5 us, one
// bf16 token over 1,000 17.0, 16.6, 17.5, 20.4; pieces of many rows, which cost more
// to write and join, 24 prompts of up to 777 tokens 54.9, 53.7, 53.8, 51.9, four
// chunks beside 60 tokens, 64 heads, 193, 193, 192, 188; the other batches the same.
constexpr int kMinPiece = 256;
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return (static_cast<int64_t>(uniform(static_cast<int>(x >> 32))) << 32) |
         static_cast<uint32_t>(uniform(static_cast<int>(x)));
}

// A sequence's tiles and their cost on the line. On the line a sequence's tiles
// of a KV head go first, last, second, last but one, ...: the later a tile, the
// more it sees, and so every two neighbours cost the same and slices end where
// tiles do (in the order of the tiles a 4,096-token prompt's first slices held
// eleven start-ups each).
template <int TILE>
struct SeqOf {
  int row0, rows, kv;
  int per;    // query rows of a tile
  int tiles;  // per group of KV heads
  int heads, groups;  // KV heads of a tile, and how many such groups there are
  int cost;   // of a token
  int64_t group_cost;
  // positions that tile j sees
  __device__ __forceinline__ int end(int j) const { return max(0, kv - rows + min(rows, (j + 1) * per)); }
  __device__ __forceinline__ int64_t tile_cost(int j) const { return TILE + static_cast<int64_t>(end(j)) * cost; }
  // cost of the tiles 0 .. j - 1
  __device__ __forceinline__ int64_t first(int j) const {
    const int64_t base = kv - rows;
    const int whole = min(j, tiles - 1);  // tiles that end at a multiple of `per`
    const int blind = base >= 0 ? 0 : static_cast<int>(-base / per);  // of these, that see nothing
    int64_t tokens = 0;
    if (whole > blind)
      tokens = (whole - blind) * base +
               per * (static_cast<int64_t>(whole) * (whole + 1) / 2 - static_cast<int64_t>(blind) * (blind + 1) / 2);
    if (j == tiles) tokens += max(0, kv);
    return static_cast<int64_t>(j) * TILE + tokens * cost;
  }
  // the k-th tile on the line, and the cost of those before it
  __device__ __forceinline__ int at(int k) const { return k & 1 ? tiles - 1 - (k >> 1) : k >> 1; }
  __device__ __forceinline__ int64_t before(int k) const {
    return first((k + 1) >> 1) + group_cost - first(tiles - (k >> 1));
  }
};

// Offsets and lengths are clamped to what the buffers hold.
template <typename E>
__device__ __forceinline__ SeqOf<E::kTile> seq_of(const ChunkArgs& a, int off, int next_off, int kv) {
  SeqOf<E::kTile> s;
  s.row0 = min(max(off, 0), a.n_rows);
  s.rows = max(0, min(max(next_off, 0), a.n_rows) - s.row0);
  s.kv = min(max(kv, 0), a.max_blocks * a.block_size);
  s.per = a.tile_rows;
  s.tiles = s.rows <= s.per ? s.rows > 0 : (s.rows + s.per - 1) / s.per;
  const int row_tiles = (min(s.rows, s.per) * a.group + 31) / 32;
  s.heads = s.tiles == 1 ? chunk_heads<E::kNarrowTiles>(a.most_heads, row_tiles) : 1;
  s.groups = (a.hkv + s.heads - 1) / s.heads;
  s.cost = E::token_cost(a, row_tiles, s.heads);
  s.group_cost = s.tiles <= 1 ? s.tiles * s.tile_cost(0) : s.first(s.tiles);
  return s;
}
template <typename E>
__device__ __forceinline__ SeqOf<E::kTile> seq_of(const ChunkArgs& a, int i) {
  return seq_of<E>(a, a.row_off[i], a.row_off[i + 1], a.kv_len[i]);
}
// The same for an i that all lanes share, in scalar registers.
template <typename E>
__device__ __forceinline__ SeqOf<E::kTile> seq_uniform(const ChunkArgs& a, int i) {
  return seq_of<E>(a, uniform(a.row_off[i]), uniform(a.row_off[i + 1]), uniform(a.kv_len[i]));
}

// Where the line of length `total` is cut in front of slice i of n. (Fewer slices
// than workgroups: the line is short.)
// Engines with kShifts have costs that are powers of two and short lines in slices
// of kShortSlice: no division of 64 bits is left on the way to a tile, which took 1.6
// us from the slice's place to the tile's queries.
template <typename E>
__device__ __forceinline__ int64_t line_cut(int64_t total, int i, int n) {
  if constexpr (E::kShifts)
    return n == kChunkSlices ? (total >> 8) * i + ((total & 255) * i >> 8) : min(total, static_cast<int64_t>(i) * kShortSlice);
  return n == kChunkSlices ? total / kChunkSlices * i + total % kChunkSlices * i / kChunkSlices
                           : static_cast<int64_t>(static_cast<uint64_t>(total) * i / n);
}

// Token at which a cut at `y` of a tile's cost goes through its `end` tokens.
template <typename E>
__device__ __forceinline__ int cut(int64_t y, int64_t tile_cost, int cost, int end) {
  if (y <= 0) return 0;
  if (y >= tile_cost) return end;
  if constexpr (E::kShifts) {
    const int by = 31 - __builtin_clz(cost);
    const int t = static_cast<int>(max(static_cast<int64_t>(0), y - E::kTile) >> by) & ~31;
    const int least = max(32, kMinPiece >> by & ~31);
    return t < least ? 0 : t > end - least ? end : t;
  }
  const int t = static_cast<int>(max(static_cast<int64_t>(0), y - E::kTile) / cost) & ~31;
  const int least = max(32, kMinPiece / cost & ~31);
  return t < least ? 0 : t > end - least ? end : t;
}

// --------------------------------------------------------------------------
// The stage engines: a wave's loads, products and softmax.
// --------------------------------------------------------------------------
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  return __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(a), static_cast<__bf16>(b)});
}

// Where a stage's blocks lie: the table row, and the entries that exist.
struct Pages {
  const int32_t* table;
  int last, num_blocks;
  __device__ __forceinline__ int entry(int i) const { return table[min(i, last)]; }
  // an entry as a block of the pools
  __device__ __forceinline__ int block(int entry) const {
    return static_cast<int>(min(static_cast<uint32_t>(entry), static_cast<uint32_t>(num_blocks - 1)));
  }
};

// Byte off + more (a constant) of a block, 16 bytes per lane, to `dst` (+ 16
// bytes per lane). POLICY: see kStream.
template <int POLICY>
__device__ __forceinline__ void load_lds(const char* block, uint32_t bytes, uint32_t off, int more, void* dst) {
  const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(block), 0, bytes, 0x00027000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_ptr)(dst), 16, off, more, 0, POLICY);
}

// A value that the compiler takes for new: what is computed from it inside a
// loop stays there instead of in a register for each stage's every address.
__device__ __forceinline__ uint32_t anew(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Until at most N of this wave's vector loads and stores are in flight.
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}

// LDS reads outside the compiler's view, which would wait for the direct loads in
// flight before each. A read's register counts as written only behind an
// lds_wait that names it (and waits for all reads but the `keep` issued last:
// they complete in order).
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_ptr)(const_cast<void*>(p))));
}
__device__ __forceinline__ u32x4 lds_read_b128(uint32_t addr, int off) {
  u32x4 r;
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(r) : "v"(addr), "i"(off) : "memory");
  return r;
}
__device__ __forceinline__ void lds_wait(u32x4& r, int keep) {
  asm volatile("s_waitcnt lgkmcnt(%1)" : "+v"(r) : "i"(keep) : "memory");
}
template <int N>
__device__ __forceinline__ void lds_wait(u32x4 (&r)[N]) {
  lds_wait(r[0], 0);
#pragma unroll
  for (int i = 1; i < N; ++i) asm volatile("" : "+v"(r[i]) : : "memory");
}

// Whether the lane or the other one of its row (32 lanes on) is among `past`: the
// row's reference then moves to its largest score, however little that lies above
// it. (Scores 4 to 8 above the reference would take every stage back here: 2,048
// rows behind 30,000 positions, each 6 above its first stage, 2.24 ms against 1.60.)
__device__ __forceinline__ bool row_past(uint64_t past, int lane) {
  return ((past | past >> 32 | past << 32) >> lane & 1) != 0;
}

// A lane's share of the addresses of a stage: of its loads inside a block and of
// its operand reads inside a slot.
struct Bases {
  uint32_t kload, vload, kread, vread;
};

__device__ __forceinline__ void barrier_lds() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ void barrier_only() { asm volatile("s_barrier" ::: "memory"); }

// A tile, or the piece of it that a slice works on.
struct Tile {
  int n_packed, head;
  int tok_lo, tok_hi;
};

// A row's factor and log-sum-exp from its reference (base 2) and sum: zero and -inf
// where it attends to nothing, which is where the sum is zero. (One that is no
// number goes on into both.)
__device__ __forceinline__ float reciprocal_sum(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }
__device__ __forceinline__ float log_sum(float m, float l) {
  return l == 0.0f ? kNegInf : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Eight channels of a row, in the output type.
__device__ __forceinline__ void store_out(float* p, f32x4 x, f32x4 y) {
  reinterpret_cast<f32x4*>(p)[0] = x;
  reinterpret_cast<f32x4*>(p)[1] = y;
}
__device__ __forceinline__ void store_out(__bf16* p, f32x4 x, f32x4 y) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(y[0], y[1]), pack2(y[2], y[3]));
}

// Index of a slice's piece: 0 of a tile that began before it, 1 of one that goes on behind it.
__device__ __forceinline__ size_t piece_row(int slice, int which) {
  return (static_cast<size_t>(slice) * 2 + which) * kChunkTileRows;
}

// Where a slice begins.
struct Start {
  int seq, row0, rows, kv, group, nth;
  int64_t y0;
};

// The line's length and this slice's part of it, in [pos, stop); false: none.
template <typename E>
__device__ __forceinline__ bool find_slice(const ChunkArgs& a, int slice, int tid, int64_t* wave_sum, Start* start, int* n_slices,
                                           int64_t* total_out, int64_t* pos_out, int64_t* stop_out) {
  const int lane = tid & 63, wave = tid >> 6;
  // Up to 64 sequences: every wave finds the place by itself, without a barrier.
  const bool few = E::kShifts && a.n_seqs <= 64;
  const int per_thread = few ? 1 : (a.n_seqs + 64 * kWaves - 1) / (64 * kWaves), me = few ? lane : tid;
  const int i0 = min(me * per_thread, a.n_seqs), i1 = min(i0 + per_thread, a.n_seqs);
  int64_t sum = 0;
  SeqOf<E::kTile> s;
  for (int i = i0; i < i1; ++i) {
    s = seq_of<E>(a, i);
    sum += s.group_cost * s.groups;
  }
  int64_t upto = wave_scan(sum);
  int64_t total = 0;
  if (few) {
    total = __shfl(upto, 63);
  } else {
    if (lane == 63) wave_sum[wave] = upto;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) upto += wave_sum[w];
      total += wave_sum[w];
    }
  }
  total = uniform(total);
  const int64_t wanted = E::kShifts ? (total + kShortSlice - 1) / kShortSlice : max(total / kMinSlice, static_cast<int64_t>(1));
  const int n = static_cast<int>(min(wanted, static_cast<int64_t>(kChunkSlices)));
  *n_slices = n;
  *total_out = total;
  if (slice >= n || total == 0) return false;
  const int64_t pos = line_cut<E>(total, slice, n);
  *pos_out = pos;
  *stop_out = line_cut<E>(total, slice + 1, n);
  int64_t at = upto - sum;
  if (pos >= at && pos < upto) {
    int i = i0;
    for (; i1 - i0 > 1; ++i) {
      s = seq_of<E>(a, i);
      if (pos < at + s.group_cost * s.groups) break;
      at += s.group_cost * s.groups;
    }
    int64_t y0 = pos - at;
    int group = 0;
    if (y0 >= s.group_cost) {
      group = static_cast<int>(static_cast<double>(y0) / static_cast<double>(s.group_cost));
      if (group * s.group_cost > y0) --group;
      else if ((group + 1) * s.group_cost <= y0) ++group;
      y0 -= group * s.group_cost;
    }
    // The last tile that begins at or before y0: neighbours cost the same, so a
    // division finds it, but where the last tile is part of one or tiles are blind.
    int nth = 0;
    if (s.tiles > 1) {
      const double pair = static_cast<double>(s.tile_cost(0) + s.tile_cost(s.tiles - 1));
      nth = min(2 * static_cast<int>(static_cast<double>(y0) / pair), s.tiles - 1);
      while (s.before(nth) > y0) --nth;
      while (nth + 1 < s.tiles && s.before(nth + 1) <= y0) ++nth;
    }
    if (nth > 0) y0 -= s.before(nth);
    *start = Start{i, s.row0, s.rows, s.kv, group, nth, y0};
  }
  if (few) {  // (every wave has written the same)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  } else {
    __syncthreads();
  }
  return true;
}

// A workgroup's slice, with the stage engine E: types and sizes (Elem, kD, kBlock,
// kTokens, kUnits, kSlot), prices (token_cost, kShifts), a wave's own stages (kDepth 1:
// the loop below; more: Stages) and, with kWide, tiles of more than kNarrowTiles row
// tiles whose stages the waves share (wide_tile). The kernel itself, and no function
// that kernels call: with one, the bf16 engine took one token 0.3 us more.
template <typename E>
__global__ void __launch_bounds__(64 * kWaves, 1) chunk_attn_kernel(ChunkArgs a) {
  using T = typename E::Elem;
  constexpr int D = E::kD, BS = E::kBlock;
  constexpr int kFloat4s = D / 8;  // of a lane's accumulator
  constexpr bool kWide = E::kWide;
  __shared__ __align__(256) uint4 smem[kWaves][E::kSlot];  // a slot for each wave; wide: the ring
  __shared__ float2 ml[kWaves][32];
  __shared__ int64_t wave_sum[kWaves];
  __shared__ Start start;
  static_assert(E::kSlot >= kFloat4s * 64, "a wave's slot holds its accumulator");
  static_assert(!kWide || chunk_heads<E::kNarrowTiles>(kWaves, E::kNarrowTiles + 1) == 1, "waves that share stages are of one KV head");
  const int tid = threadIdx.x, wave = uniform(tid >> 6);
  const int group = a.group;  // query heads of a KV head
  const int per_die = kChunkSlices / kDies;
  const int slice = static_cast<int>(blockIdx.x) % kDies * per_die + static_cast<int>(blockIdx.x) / kDies;
  if (tid == 0) {
    a.splits[slice].n_rows = 0;
    a.continues[slice] = 0;
  }
  int n_slices;
  int64_t total, pos, stop;
  if (!find_slice<E>(a, slice, tid, wave_sum, &start, &n_slices, &total, &pos, &stop)) return;
  int seq = start.seq, head_group = start.group, nth = start.nth;
  int64_t y0 = start.y0;
  SeqOf<E::kTile> sq;
  sq.row0 = start.row0;
  sq.rows = start.rows;
  sq.kv = start.kv;

  for (;;) {
    // ---- one tile, or the slice's piece of it ----
    // All of this is the same in every lane; said to the compiler, it stays in
    // scalar registers (64-bit comparisons would move it to vector ones, and a
    // load from a block there takes a loop over the lanes' addresses). A lane's
    // addresses are computed anew for each tile: kept over tiles, those of both
    // paths would fill the registers and spill.
    const int lane = static_cast<int>(anew(tid & 63));
    seq = uniform(seq);
    head_group = uniform(head_group);
    nth = uniform(nth);
    y0 = uniform(y0);
    pos = uniform(pos);
    stop = uniform(stop);
    sq = seq_of<E>(a, uniform(sq.row0), uniform(sq.row0 + sq.rows), uniform(sq.kv));
    const int tile = sq.at(nth), end = uniform(sq.end(tile));
    const int64_t tile_cost = uniform(sq.tile_cost(tile));
    const int64_t y1 = uniform(min(tile_cost, y0 + stop - pos));
    const int tok_lo = uniform(cut<E>(y0, tile_cost, sq.cost, end)), tok_hi = uniform(cut<E>(y1, tile_cost, sq.cost, end));
    if (tok_hi > tok_lo || (end == 0 && y0 == 0)) {
      const int r0 = tile * sq.per;  // first query row of the tile, in the sequence
      const int n_packed = min(sq.per, sq.rows - r0) * group;
      const int row_tiles = (n_packed + 31) / 32;
      const int head0 = head_group * sq.heads, heads = min(sq.heads, a.hkv - head0);
      // a wave's unit (KV head and row tile), and its share of the tokens
      static_assert(kWaves == 8, "ways of 8 waves");
      const int units = row_tiles * heads, ways = units == 1 ? 8 : units == 2 ? 4 : units <= 4 ? 2 : 1;
      const int unit = wave % units, way = wave / units;
      const int head = head0 + unit / row_tiles, rt = unit % row_tiles;
      const bool works = way < ways;  // wide: every wave loads, those with a row tile compute
      // The tokens of the piece that the wave's row tile sees end here. (Three fp32
      // prompts of up to 200 rows, 2 KV heads of 64: 35 us where every wave went on to the
      // piece's end, 31 so. A wide tile's waves stay together: it brought them nothing.)
      const int seen = works ? min(tok_hi, sq.kv - sq.rows + r0 + (min(32 * rt + 32, n_packed) - 1) / group + 1) : 0;
      E e;
      e.clear();
      const Pages pg{a.table + static_cast<size_t>(seq) * a.max_blocks, max(0, (sq.kv + BS - 1) / BS - 1), a.num_blocks};
      const int first = tok_lo + way * E::kTokens, stride = ways * E::kTokens;
      const bool wide = kWide && row_tiles > E::kNarrowTiles && tok_hi > tok_lo;  // rows with nothing to see: no stages
      const Bases at = E::bases(lane);
      // (kDepth > 1: the wave's stages of its own are the engine's)
      [[maybe_unused]] typename E::Stages stages;
      int ent[E::kBlocks], ahead[E::kBlocks];  // blocks of the stage that is loaded next, and of the one behind it
      auto look_up = [&](int (&to)[E::kBlocks], int tb) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < E::kBlocks; ++b) to[b] = pg.entry(tb / BS + b);
      };
      const bool alone = row_tiles == 1;
      auto issue_k = [&](int off) __attribute__((always_inline)) {
        if constexpr (E::kDepth == 1) {
          if (alone) E::template issue_k<kStream>(a, pg, at, ent, head, off, smem[wave]);
          else E::template issue_k<kKeep>(a, pg, at, ent, head, off, smem[wave]);
        }
      };
      auto issue_v = [&](int off) __attribute__((always_inline)) {
        if constexpr (E::kDepth == 1) {
          if (alone) E::template issue_v<kStream>(a, pg, at, ent, head, off, smem[wave]);
          else E::template issue_v<kKeep>(a, pg, at, ent, head, off, smem[wave]);
        }
      };
      if (!wide && first < seen) {
        if constexpr (E::kDepth == 1) {
          look_up(ent, first);
          look_up(ahead, first + stride);
          issue_k(first % BS);
          issue_v(first % BS);
        } else {
          stages.look_up(a, pg, head, first, stride, seen, lane);
        }
      }
      int least = INT_MAX;
      const bool second = E::kUnits == 1 || n_packed - 32 * rt > 16;
#pragma unroll
      for (int u = 0; u < E::kUnits; ++u) {
        const int p = 32 * rt + E::row(lane, u), pp = p < n_packed ? p : 0;
        const int row = r0 + pp / group;
        // rows that are none see everything: they never hold up a stage
        e.hz[u] = p < n_packed ? sq.kv - sq.rows + row : INT_MAX;
        least = min(least, e.hz[u]);
        e.load_q(static_cast<const T*>(a.q) + static_cast<int64_t>(sq.row0 + row) * a.q_stride +
                     (head * group + pp % group) * D, lane, u);
      }
      if constexpr (E::kDepth > 1) {  // behind the queries: a wait for these is none for the stages
        if (!wide && first < seen) {
          if (alone) stages.template begin<kStream>(pg, at, smem[wave]);
          else stages.template begin<kKeep>(pg, at, smem[wave]);
        }
      }
      least = uniform(wave_min_int(least));
      const float c = a.scale_log2;
      if (wide) {
        if constexpr (kWide)
          E::wide_tile(a, Tile{n_packed, head, tok_lo, tok_hi}, pg, smem, lane, wave, e);
        barrier_lds();  // the ring is read: a wave may load its slot for the next tile
      } else if (works) {
        // K and V of a stage are loaded as soon as the slot's halves have been read:
        // at every wait the loads behind the awaited half are the other half's, kLoads
        // of them. (Lookups are issued in front of the loads of a half: they can only
        // make a wait longer.)
        const uint32_t slot = lds_addr(smem[wave]);
        e.settle_q();
        if constexpr (E::kDepth == 1) {
          for (int tb = first; tb < seen; tb += stride) {
            const bool more = tb + stride < seen;
            wait_vmcnt<E::kLoads>();
            e.read_k(slot, at);  // (waited for: the half may be written again)
#pragma unroll
            for (int b = 0; b < E::kBlocks; ++b) ent[b] = ahead[b];
            look_up(ahead, tb + 2 * stride);
            asm volatile("" ::: "memory");
            if (more) issue_k((tb + stride) % BS);
            e.softmax(tb, tok_hi, tb + E::kTokens > tok_hi || tb + E::kTokens - 1 > least, c, lane, second);
            if (more) wait_vmcnt<E::kLoads>();
            else wait_vmcnt<0>();
            e.read_v(slot, at);
            if (more) issue_v((tb + stride) % BS);
            e.values(tb, tok_hi, lane, second);
          }
        } else {
          if (first < seen) {
            if (alone) stages.template run<kStream>(e, a, pg, at, tok_hi, least, c, lane, second, smem[wave]);
            else stages.template run<kKeep>(e, a, pg, at, tok_hi, least, c, lane, second, smem[wave]);
          }
        }
      }
      // ---- join the ways, and write the outputs or the piece for the merge ----
      // Every wave puts its sums into LDS by rows, then takes rows of the tile:
      // kRows at a time, eight channels a lane, so that stores fill lines.
      constexpr int kLanesPerRow = D / 8, kRows = 64 / kLanesPerRow, kPasses = 32 / kRows;
      auto chunk_at = [&](int w, int r, int c) __attribute__((always_inline)) {
        return reinterpret_cast<f32x4*>(smem[w]) + r * (D / 4) + (c ^ (r & (D / 4 - 1)));
      };
      if (works) {
#pragma unroll
        for (int u = 0; u < E::kUnits; ++u) {
          const float sum = e.row_sum(u);
          if (lane < 32 / E::kUnits) ml[wave][E::row(lane, u)] = make_float2(e.m[u], sum);
        }
#pragma unroll
        for (int i = 0; i < kFloat4s; ++i) {
          if (!E::kShifts || 32 * rt + E::out_row(lane, i) < n_packed)  // (rows that are none have no place to go)
            *chunk_at(wave, E::out_row(lane, i), E::out_channel(lane, i) / 4) = e.get(i);
        }
      }
      if (ways > 1) __syncthreads();
      const bool whole = tok_lo == 0 && tok_hi == end;
      // Rows id * kRows .. of the units, of the sums of the waves that had them.
      // (kWays is a constant, so that its reads are in flight together: 96 tokens over up
      // to 8,190 positions 281 us with a loop over the ways, 276 so; two over 131,000 93.8
      // and 91.5.)
      auto finish = [&](int id, auto ways_c) __attribute__((always_inline)) {
        constexpr int kWays = decltype(ways_c)::value;
        const int tr = id / kPasses, r = id % kPasses * kRows + lane / kLanesPerRow;
        const int p = tr % row_tiles * 32 + r, c = 2 * (lane % kLanesPerRow);
        if (tr >= units || p >= n_packed) return;
        const float2 s = ml[tr][r];
        float m = s.x, l = s.y;
        f32x4 x = *chunk_at(tr, r, c), y = *chunk_at(tr, r, c + 1);
        if constexpr (kWays > 1) {
          float2 others[kWays];
#pragma unroll
          for (int v = 1; v < kWays; ++v) others[v] = ml[v * units + tr][r];
#pragma unroll
          for (int v = 1; v < kWays; ++v) m = fmaxf(m, others[v].x);
          const float ref = m == kNegInf ? 0.0f : m, f = exp2_fast(s.x - ref);
          l *= f;
          x *= f;
          y *= f;
#pragma unroll
          for (int v = 1; v < kWays; ++v) {
            const int w = v * units + tr;
            const float g = exp2_fast(others[v].x - ref);
            l += others[v].y * g;
            x += *chunk_at(w, r, c) * g;
            y += *chunk_at(w, r, c + 1) * g;
          }
        }
        if (whole) {
          const int row = p / group;
          const size_t at_row =
              static_cast<size_t>(sq.row0 + r0 + row) * a.hq + (head0 + tr / row_tiles) * group + (p - row * group);
          const float inv = reciprocal_sum(l);
          store_out(static_cast<T*>(a.out) + at_row * D + 4 * c, x * inv, y * inv);
          if (a.lse != nullptr && c == 0) a.lse[at_row] = log_sum(m, l);
        } else {
          const size_t at_row = piece_row(slice, tok_lo == 0 ? 1 : 0) + 32 * tr + r;
          store_out(a.part_o + at_row * D + 4 * c, x, y);
          if (c == 0) reinterpret_cast<float2*>(a.part_ml)[at_row] = make_float2(m, l);
        }
      };
      if (ways > 1) {
        for (int id = wave; id < units * kPasses; id += kWaves) {
          if (ways == 8) finish(id, std::integral_constant<int, 8>{});
          else if (ways == 4) finish(id, std::integral_constant<int, 4>{});
          else finish(id, std::integral_constant<int, 2>{});
        }
      } else if (works) {
#pragma unroll 4
        for (int k = 0; k < kPasses; ++k) finish(unit * kPasses + k, std::integral_constant<int, 1>{});
      }
      if (ways > 1) __syncthreads();  // the slots are read
      if (!whole && tid == 0) {
        if (tok_lo > 0) {
          a.continues[slice] = 1;
        } else {
          // the last slice that begins inside the tile
          const int64_t tile_end = pos - y0 + tile_cost;
          int last = min(static_cast<int>(static_cast<double>(tile_end) / static_cast<double>(total) * n_slices), n_slices - 1);
          while (line_cut<E>(total, last, n_slices) >= tile_end) --last;
          while (last + 1 < n_slices && line_cut<E>(total, last + 1, n_slices) < tile_end) ++last;
          a.splits[slice] = ChunkSplit{sq.row0 + r0, head0, n_packed, row_tiles, heads, last};
        }
      }
    }
    // ---- the next tile of the line ----
    pos = uniform(pos + y1 - y0);
    y0 = 0;
    if (pos >= stop) break;
    if (++nth == sq.tiles) {
      nth = 0;
      if (++head_group == sq.groups) {
        head_group = 0;
        // the next sequence with rows, 64 at a time
        int found = -1;
        for (int i = seq + 1; found < 0 && i < a.n_seqs; i += 64) {
          const bool has = i + lane < a.n_seqs && seq_of<E>(a, i + lane).tiles > 0;
          const uint64_t bal = __ballot(has);
          if (bal != 0) found = i + __builtin_ctzll(bal);
        }
        if (found < 0) break;  // not reached: the line ends with the last tile
        seq = uniform(found);
        sq = seq_uniform<E>(a, seq);
      }
    }
  }
}

}  // namespace
}  // namespace spork
