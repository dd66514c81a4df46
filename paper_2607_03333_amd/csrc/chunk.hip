// gfx950 attention of the new tokens of a ragged batch, prompt chunks and single
// tokens alike, over the paged cache. Lengths, offsets and block tables are read
// on the device; nothing of the work split comes from the host.
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
//
// In tiles of up to four row tiles, and all of fp32's, each wave streams its
// 32-token stages (fp32: 16) of K and V into a slot of its own in LDS by direct
// loads (lane i of an instruction lands at its base + 16 i) and reads them from
// there as operands; the loads of the next stage are in flight while it computes,
// and no wave waits for another inside a tile. In bf16 tiles of more row tiles the
// waves share their stages (wide_tile).
//   bf16  S^T = K Q^T and O^T += V^T P^T in 32x32x16 products. A-row r of the
//         scores is token 16*(r/16) + 8*(r/4%2) + 4*(r/8%2) + r%4, so that a lane
//         receives its query row's scores of tokens 16h + 8g + j (element 8h + j,
//         g = lane / 32), which are its operand of the second product.
//   fp32  16x16x4 products, two row tiles of 16 per wave; tokens 4g + i
//         (g = lane / 16) likewise.
// Softmax in base 2 with a lazily moved reference: it moves to the row's largest
// score, and the accumulator is rescaled, only where a lane's probabilities of a
// stage sum past 2^8 (fp32: where a score lies more than 8 above it).
// Probabilities enter the second product in the input type (bf16: rounded to
// nearest, at most 2^-8 of each; the row sum is of the unrounded ones); sums, reference
// and accumulators are fp32.
#include "chunk_kernels.h"
#include "device_common.h"
#include "wave_scan.h"

namespace spork {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) void* lds_ptr;

constexpr int kWaves = 8;
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
// Least cost of a piece: a cut closer to a tile's end moves to it. At 64, 256, 512 and
// 1,024: eight fp32 tokens over up to 1,500 positions 16.9, 18.2, 19.1, 26.5 us, one
// bf16 token over 1,000 17.0, 16.6, 17.5, 20.4; pieces of many rows, which cost more
// to write and join, 24 prompts of up to 777 tokens 54.9, 53.7, 53.8, 51.9, four
// chunks beside 60 tokens, 64 heads, 193, 193, 192, 188; the other batches the same.
constexpr int kMinPiece = 256;
// A token of a tile of `heads` KV heads with so many row tiles each: bf16 by
// bytes until the products weigh more; fp32 products (64 flop per cycle and SIMD)
// weigh more from the first row tile. Three bf16 chunks beside 29 tokens 157 us, with
// one price for all tiles 185, with twice as much from five row tiles on 197; four
// chunks beside 60 tokens 193, 215, 237. Three fp32 prompts 28 us, at half the price
// 30, at twice 27.5, at one price for any number of row tiles 57; two fp32 chunks
// behind 1,500 to 2,000 positions 38.8, 38.9, 42.6, 59.
__device__ __forceinline__ int token_cost(const ChunkArgs& a, int row_tiles, int heads) {
  const int wide = a.head_dim == 128 ? 2 : 1;
  if (a.dtype == 0) return 2 * wide * row_tiles * heads;
  return wide * max(heads, row_tiles <= 2 ? 1 : 2);
}

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
struct Seq {
  int row0, rows, kv;
  int per;    // query rows of a tile
  int tiles;  // per group of KV heads
  int heads, groups;  // KV heads of a tile, and how many such groups there are
  int cost;   // of a token
  int64_t group_cost;
  // positions that tile j sees
  __device__ __forceinline__ int end(int j) const { return max(0, kv - rows + min(rows, (j + 1) * per)); }
  __device__ __forceinline__ int64_t tile_cost(int j) const { return kTileCost + static_cast<int64_t>(end(j)) * cost; }
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
    return static_cast<int64_t>(j) * kTileCost + tokens * cost;
  }
  // the k-th tile on the line, and the cost of those before it
  __device__ __forceinline__ int at(int k) const { return k & 1 ? tiles - 1 - (k >> 1) : k >> 1; }
  __device__ __forceinline__ int64_t before(int k) const {
    return first((k + 1) >> 1) + group_cost - first(tiles - (k >> 1));
  }
};

// Offsets and lengths are clamped to what the buffers hold.
__device__ __forceinline__ Seq seq_of(const ChunkArgs& a, int off, int next_off, int kv) {
  Seq s;
  s.row0 = min(max(off, 0), a.n_rows);
  s.rows = max(0, min(max(next_off, 0), a.n_rows) - s.row0);
  s.kv = min(max(kv, 0), a.max_blocks * a.block_size);
  s.per = a.tile_rows;
  s.tiles = s.rows <= s.per ? s.rows > 0 : (s.rows + s.per - 1) / s.per;
  const int row_tiles = (min(s.rows, s.per) * a.group + 31) / 32;
  s.heads = s.tiles == 1 ? min(a.most_heads, kWaves / row_tiles) : 1;
  s.groups = (a.hkv + s.heads - 1) / s.heads;
  s.cost = token_cost(a, row_tiles, s.heads);
  s.group_cost = s.tiles <= 1 ? s.tiles * s.tile_cost(0) : s.first(s.tiles);
  return s;
}
__device__ __forceinline__ Seq seq_of(const ChunkArgs& a, int i) {
  return seq_of(a, a.row_off[i], a.row_off[i + 1], a.kv_len[i]);
}
// The same for an i that all lanes share, in scalar registers.
__device__ __forceinline__ Seq seq_uniform(const ChunkArgs& a, int i) {
  return seq_of(a, uniform(a.row_off[i]), uniform(a.row_off[i + 1]), uniform(a.kv_len[i]));
}

// Where the line of length `total` is cut in front of slice i of n. (Fewer slices
// than workgroups: the line is short.)
__device__ __forceinline__ int64_t line_cut(int64_t total, int i, int n) {
  return n == kChunkSlices ? total / kChunkSlices * i + total % kChunkSlices * i / kChunkSlices
                           : static_cast<int64_t>(static_cast<uint64_t>(total) * i / n);
}

// Token at which a cut at `y` of a tile's cost goes through its `end` tokens.
__device__ __forceinline__ int cut(int64_t y, int64_t tile_cost, int cost, int end) {
  if (y <= 0) return 0;
  if (y >= tile_cost) return end;
  const int t = static_cast<int>(max(static_cast<int64_t>(0), y - kTileCost) / cost) & ~31;
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

template <typename T, int D, int BS>
struct Engine;

template <int D, int BS>
struct Engine<__bf16, D, BS> {
  static constexpr int kTokens = 32;                // of a stage
  static constexpr int kUnits = 1;                  // rows of a lane
  static constexpr int kChunksPerToken = D / 8;     // 16-byte chunks
  static constexpr int kHalf = kTokens * D / 8;     // chunks of K, and of V
  static constexpr int kLoads = kHalf / 64;         // instructions of K, and of V
  static constexpr int kSteps = D / 16, kCt = D / 32;
  bf16x8 q[kSteps];
  f32x16 o[kCt];
  float m[1], l[1];
  int hz[1];  // last visible position of the lane's row

  static __device__ __forceinline__ int row(int lane, int) { return lane & 31; }
  static __device__ __forceinline__ int out_row(int lane, int) { return lane & 31; }
  static __device__ __forceinline__ int out_channel(int lane, int i) { return 32 * (i / 4) + 8 * (i % 4) + 4 * (lane >> 5); }
  __device__ __forceinline__ f32x4 get(int i) const {
    const f32x16& v = o[i / 4];
    const int e = 4 * (i % 4);
    return f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]};
  }
  __device__ __forceinline__ float row_sum(int) const { return l[0] + __shfl_xor(l[0], 32); }

  // K: chunk t * kChunksPerToken + (c ^ swizzle(t)) holds channels 8c .. 8c + 7 of
  // token t. V: chunk 2d + q of half h (16-token blocks) or 4d + (q ^ swizzle(d)),
  // tokens 8q .. of channel d. The swizzles spread the lanes of an operand read
  // over the banks.
  static __device__ __forceinline__ int kswz(int t) {
    return ((t & 7) | ((t >> 1) & 8)) & (kChunksPerToken - 1);
  }
  static __device__ __forceinline__ int vswz(int d) { return BS == 16 ? (d >> 3) & 1 : (d >> 3) & 3; }

  __device__ __forceinline__ void load_q(const __bf16* p, int lane, int) {
    const int g = lane >> 5;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) q[s] = as_bf16x8(*reinterpret_cast<const uint4*>(p + 16 * s + 8 * g));
  }
  // The queries have arrived: no wait for them is left for the loops.
  __device__ __forceinline__ void settle_q() {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) asm volatile("" : "+v"(q[s]));
  }
  __device__ __forceinline__ void clear() {
    m[0] = kNegInf;
    l[0] = 0.0f;
#pragma unroll
    for (int i = 0; i < kCt; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[i][e] = 0.0f;
  }

  static __device__ __forceinline__ Bases bases(int lane) {
    const int tl = lane / kChunksPerToken, c = lane % kChunksPerToken, r = lane & 31, g = lane >> 5;
    const int t = 16 * (r >> 4) + 8 * ((r >> 2) & 1) + 4 * ((r >> 3) & 1) + (r & 3);
    Bases x;
    x.kload = 2 * tl * D + 16 * (c ^ kswz(tl));
    x.vload = BS == 16 ? 32 * (lane >> 1) + 16 * ((lane & 1) ^ vswz(lane >> 1)) : 64 * (lane >> 2) + 16 * ((lane & 3) ^ vswz(lane >> 2));
    x.kread = 2 * t * D + 16 * (g ^ kswz(t));
    x.vread = 16 * kHalf + (BS == 16 ? 32 : 64) * r + 16 * (g ^ vswz(r));
    return x;
  }
  static constexpr int kBlocks = kTokens / BS;  // of a stage: 2 or 1

  // K, or V, of the stage of the blocks `ent` (from their token `first`) into the
  // wave's slot.
  template <int POLICY>
  static __device__ __forceinline__ void issue_k(const ChunkArgs& a, const Pages& pg, const Bases& x, const int (&ent)[kBlocks], int head, int,
                                                 uint4* slot) {
    constexpr uint32_t kBytes = BS * D * 2;
    const char* from[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
      from[b] = static_cast<const char*>(a.k_cache) + (static_cast<size_t>(pg.block(uniform(ent[b]))) * a.hkv + head) * kBytes;
    const uint32_t kl = anew(x.kload);
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {  // tokens tk .. of the stage
      const int tk = 64 * k / kChunksPerToken;
      load_lds<POLICY>(from[tk / BS], kBytes, kl ^ (16u * kswz(tk)), 2 * (tk % BS) * D, slot + 64 * k);
    }
  }
  template <int POLICY>
  static __device__ __forceinline__ void issue_v(const ChunkArgs& a, const Pages& pg, const Bases& x, const int (&ent)[kBlocks], int head, int,
                                                 uint4* slot) {
    constexpr uint32_t kBytes = BS * D * 2;
    const char* from[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
      from[b] = static_cast<const char*>(a.v_cache) + (static_cast<size_t>(pg.block(uniform(ent[b]))) * a.hkv + head) * kBytes;
    const uint32_t vl = anew(x.vload);
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {  // channels dk .. of a half, or of all 32 tokens
      const int dk = BS == 16 ? 64 * k % (kHalf / 2) / 2 : 16 * k;
      load_lds<POLICY>(from[BS == 16 ? 64 * k / (kHalf / 2) : 0], kBytes, vl ^ (16u * vswz(dk)), 2 * dk * BS,
                        slot + kHalf + 64 * k);
    }
  }

  u32x4 kop[kSteps], vop[2 * kCt];
  // The slot's halves into registers: issued, and waited for by lds_wait.
  __device__ __forceinline__ void read_k(uint32_t slot, const Bases& b) {
    const uint32_t kr = anew(b.kread);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) kop[s] = lds_read_b128(slot + (kr ^ (32u * s)), 0);
    lds_wait(kop);
  }
  __device__ __forceinline__ void read_v(uint32_t slot, const Bases& b) {
    const uint32_t vr = anew(b.vread);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int ct = 0; ct < kCt; ++ct)
        vop[h * kCt + ct] = BS == 16 ? lds_read_b128(slot + vr, 8 * kHalf * h + 1024 * ct) : lds_read_b128(slot + (vr ^ (32u * h)), 2048 * ct);
    lds_wait(vop);
  }

  // Zero the elements of an 8-token chunk from position `first` on that lie at or
  // past `end`.
  static __device__ __forceinline__ u32x4 zero_past(u32x4 w, int first, int end) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] &= (first + 2 * i < end ? 0x0000FFFFu : 0u) | (first + 2 * i + 1 < end ? 0xFFFF0000u : 0u);
    return w;
  }

  uint32_t pw[8];  // the stage's probabilities, as bf16 pairs

  // Scores and softmax of the stage at tb; positions from `end` on are not there,
  // `masked`: a row of the wave doesn't see all of the stage.
  __device__ __forceinline__ void softmax(int tb, int end, bool masked, float c, int lane, bool) {
    const int g = lane >> 5;
    f32x16 sc;
#pragma unroll
    for (int e = 0; e < 16; ++e) sc[e] = 0.0f;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kop[s]), q[s], sc, 0, 0, 0);
    float sv[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) sv[e] = sc[e];
    if (masked) {
      const int hi = min(end - 1, hz[0]) - tb - 8 * g;  // the last visible one, from the lane's first
      const float none = c < 0.0f ? -kNegInf : kNegInf;
#pragma unroll
      for (int e = 0; e < 16; ++e) sv[e] = 16 * (e >> 3) + (e & 7) > hi ? none : sv[e];
    }
    float ps = 0.0f;
    auto probs = [&](float ref) __attribute__((always_inline)) {
      ps = 0.0f;
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const float p0 = exp2_fast(__builtin_fmaf(sv[e], c, -ref)), p1 = exp2_fast(__builtin_fmaf(sv[e + 1], c, -ref));
        ps += p0 + p1;
        pw[e / 2] = pack2(p0, p1);
      }
    };
    probs(m[0]);
    const uint64_t past = __ballot(!(ps <= kSlackSum));
    if (__builtin_expect(past != 0, 0)) {
      float mx = sv[0] * c;
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, sv[e] * c);
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      if (row_past(past, lane) && mx > m[0]) {
        const float alpha = exp2_fast(m[0] - mx);
        l[0] *= alpha;
#pragma unroll
        for (int i = 0; i < kCt; ++i) o[i] *= alpha;
        m[0] = mx;
      }
      probs(m[0] == kNegInf ? 0.0f : m[0]);
    }
    l[0] += ps;
  }

  // P.V of the stage.
  __device__ __forceinline__ void values(int tb, int end, int lane, bool) {
    if (tb + kTokens > end) {  // what lies behind the end may be anything: 0 * NaN
#pragma unroll
      for (int i = 0; i < 2 * kCt; ++i) vop[i] = zero_past(vop[i], tb + 16 * (i / kCt) + 8 * (lane >> 5), end);
    }
#pragma unroll
    for (int i = 0; i < 2 * kCt; ++i) {
      const int h = 4 * (i / kCt), ct = i % kCt;
      o[ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          __builtin_bit_cast(bf16x8, vop[i]), __builtin_bit_cast(bf16x8, u32x4{pw[h], pw[h + 1], pw[h + 2], pw[h + 3]}), o[ct], 0, 0, 0);
    }
  }
};

template <int D, int BS>
struct Engine<float, D, BS> {
  static constexpr int kTokens = 16;
  static constexpr int kUnits = 2;
  static constexpr int kChunksPerToken = D / 4;
  static constexpr int kHalf = kTokens * D / 4;
  static constexpr int kLoads = kHalf / 64;
  static constexpr int kDt = D / 16;
  f32x4 q[2][kDt];  // channels 16j + 4g + i
  f32x4 o[2][kDt];
  float m[2], l[2];
  int hz[2];

  static __device__ __forceinline__ int row(int lane, int u) { return 16 * u + (lane & 15); }
  static __device__ __forceinline__ int out_row(int lane, int i) { return 16 * (i / kDt) + (lane & 15); }
  static __device__ __forceinline__ int out_channel(int lane, int i) { return 16 * (i % kDt) + 4 * (lane >> 4); }
  __device__ __forceinline__ f32x4 get(int i) const { return o[i / kDt][i % kDt]; }
  __device__ __forceinline__ float row_sum(int u) const {
    const float x = l[u] + __shfl_xor(l[u], 16);
    return x + __shfl_xor(x, 32);
  }
  static __device__ __forceinline__ int kswz(int t) { return t & (kChunksPerToken - 1) & 15; }
  static __device__ __forceinline__ int vswz(int d) { return (d >> 2) & 3; }

  __device__ __forceinline__ void load_q(const float* p, int lane, int u) {
    const int g = lane >> 4;
#pragma unroll
    for (int j = 0; j < kDt; ++j) q[u][j] = *reinterpret_cast<const f32x4*>(p + 16 * j + 4 * g);
  }
  __device__ __forceinline__ void settle_q() {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int j = 0; j < kDt; ++j) asm volatile("" : "+v"(q[u][j]));
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      m[u] = kNegInf;
      l[u] = 0.0f;
#pragma unroll
      for (int j = 0; j < kDt; ++j) o[u][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }

  static __device__ __forceinline__ Bases bases(int lane) {
    const int tl = lane / kChunksPerToken, c = lane % kChunksPerToken, r = lane & 15, g = lane >> 4;
    Bases x;
    x.kload = 4 * tl * D + 16 * (c ^ kswz(tl));
    x.vload = 4 * (lane >> 2) * BS + 16 * ((lane & 3) ^ vswz(lane >> 2));
    x.kread = 4 * r * D + 16 * (g ^ kswz(r));
    x.vread = 16 * kHalf + 64 * r + 16 * (g ^ vswz(r));
    return x;
  }
  static constexpr int kBlocks = 1;

  static __device__ __forceinline__ const char* block(const ChunkArgs& a, const Pages& pg, const void* pool, int ent, int head) {
    return static_cast<const char*>(pool) + (static_cast<size_t>(pg.block(uniform(ent))) * a.hkv + head) * (BS * D * 4);
  }
  template <int POLICY>
  static __device__ __forceinline__ void issue_k(const ChunkArgs& a, const Pages& pg, const Bases& x, const int (&ent)[1], int head, int first,
                                                 uint4* slot) {
    const char* from = block(a, pg, a.k_cache, ent[0], head);
    const uint32_t kl = anew(x.kload);
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      const int tk = 64 * k / kChunksPerToken;
      load_lds<POLICY>(from, BS * D * 4, kl ^ (16u * kswz(tk)), 4 * (first + tk) * D, slot + 64 * k);
    }
  }
  template <int POLICY>
  static __device__ __forceinline__ void issue_v(const ChunkArgs& a, const Pages& pg, const Bases& x, const int (&ent)[1], int head, int first,
                                                 uint4* slot) {
    const char* from = block(a, pg, a.v_cache, ent[0], head);
    const uint32_t vl = anew(x.vload);
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
      load_lds<POLICY>(from, BS * D * 4, vl, 4 * (16 * k * BS + first), slot + kHalf + 64 * k);
  }

  u32x4 kop[kDt], vop[kDt];
  float p[2][4];  // the stage's probabilities
  __device__ __forceinline__ void read_k(uint32_t slot, const Bases& b) {
    const uint32_t kr = anew(b.kread);
#pragma unroll
    for (int j = 0; j < kDt; ++j) kop[j] = lds_read_b128(slot + (kr ^ (64u * j)), 0);
    lds_wait(kop);
  }
  __device__ __forceinline__ void read_v(uint32_t slot, const Bases& b) {
    const uint32_t vr = anew(b.vread);
#pragma unroll
    for (int j = 0; j < kDt; ++j) vop[j] = lds_read_b128(slot + vr, 1024 * j);
    lds_wait(vop);
  }

  // second: the wave's rows 16 .. 31 are there.
  __device__ __forceinline__ void softmax(int tb, int end, bool masked, float c, int lane, bool second) {
    const int g = lane >> 4;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (u == 1 && !second) break;
      f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < kDt; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kop[j][i]), q[u][j][i], sc, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[u][i] = sc[i] * c;
        if (masked && tb + 4 * g + i > min(end - 1, hz[u])) p[u][i] = kNegInf;
      }
      float mx = fmaxf(fmaxf(p[u][0], p[u][1]), fmaxf(p[u][2], p[u][3]));
      if (__ballot(mx > m[u] + kSlack) != 0) {
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        if (mx > m[u] + kSlack) {  // a row's own: its bits do not depend on its neighbours
          const float alpha = exp2_fast(m[u] - mx);
          l[u] *= alpha;
#pragma unroll
          for (int j = 0; j < kDt; ++j) o[u][j] *= alpha;
          m[u] = mx;
        }
      }
      const float ref = m[u] == kNegInf ? 0.0f : m[u];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[u][i] = exp2_fast(p[u][i] - ref);
        l[u] += p[u][i];
      }
    }
  }

  __device__ __forceinline__ void values(int tb, int end, int lane, bool second) {
    if (tb + kTokens > end) {
#pragma unroll
      for (int j = 0; j < kDt; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (tb + 4 * (lane >> 4) + i >= end) vop[j][i] = 0;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (u == 1 && !second) break;
#pragma unroll
      for (int j = 0; j < kDt; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[u][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vop[j][i]), p[u][i], o[u][j], 0, 0, 0);
    }
  }
};

// --------------------------------------------------------------------------
// The wide path: bf16 tiles of more than 128 packed rows. Each wave owns one row
// tile of 32 and all of them share every 32-token stage (16 KB for 128 channels),
// which goes through a ring of eight in LDS; a barrier publishes two stages at a
// time and frees the two that were read. The matrix cores bound a stage (D / 8
// 32x32x16 products per wave, 32 cycles each, two waves to a SIMD), so beside the
// softmax of stage s run the P.V products of stage s - 1 and the scores of stage
// s + 1, one product and a few vector instructions at a time; operand reads are
// spread over the slots likewise. The reads and barriers are outside the
// compiler's view (it would wait for the loads of later stages at every read),
// with waits that name the registers; no read is in flight where a loop goes
// round. 2,048 rows behind 30,000 positions, 64 heads in groups of 8: 1.72 to 1.84 ms,
// 1.13 to 1.21 PFLOP/s, at the 1.65 to 1.75 GHz that power leaves. (With stages of each
// wave's own, a prompt of 4,096 tokens took 202 us against 134, three long chunks
// beside 29 tokens 222 against 154, 24 prompts with heads of 64 channels 69 against 52.)
// --------------------------------------------------------------------------
constexpr int kRing = 8, kPer = 2;   // stages; stages that a barrier publishes
constexpr int kAhead = kRing - kPer;

__device__ __forceinline__ void barrier_lds() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ void barrier_only() { asm volatile("s_barrier" ::: "memory"); }
// A tile, or the piece of it that a slice works on.
struct Tile {
  int n_packed, head;
  int tok_lo, tok_hi;
};

// A wave's loads of the shared stages: instruction k of wave w fills chunks
// (kStageLoads * w + k) * 64 + lane of a stage (the lower four waves K, the upper
// four V), from one block, at a scalar base plus the lane's fixed offset. The
// table goes through registers: lane i holds entry i of the window of 64 that the
// loads are in, and of the next one.
template <int D, int BS>
struct RingLoader {
  using E = Engine<__bf16, D, BS>;
  static constexpr int kStageLoads = D / 64;
  static constexpr int kPerStage = 32 / BS;  // entries of a stage
  static constexpr int kWindow = 64 / kPerStage;  // stages of a window
  const char* pool;
  Pages pages;
  int first;  // the tile's first entry
  int64_t head, hkv;
  uint32_t off[kStageLoads];
  int wave, lane, half;
  int now, next;
  __device__ __forceinline__ void init(const ChunkArgs& a, const Pages& pg, int kv_head, int tb0, int wave_, int lane_) {
    wave = wave_;
    lane = lane_;
    pages = pg;
    first = tb0 / BS;
    head = kv_head;
    hkv = a.hkv;
    pool = static_cast<const char*>(wave < 4 ? a.k_cache : a.v_cache);
    half = BS == 16 ? (wave >> 1) & 1 : 0;  // which block of a stage the wave loads
    now = pages.entry(first + lane);
    next = pages.entry(first + 64 + lane);
#pragma unroll
    for (int k = 0; k < kStageLoads; ++k) {
      const int chunk = (kStageLoads * wave + k) * 64 + lane;
      if (wave < 4) {
        const int t = chunk / E::kChunksPerToken;
        off[k] = 2u * ((t % BS) * D + 8 * ((chunk % E::kChunksPerToken) ^ E::kswz(t)));
      } else if (BS == 16) {
        const int d = (chunk % (E::kHalf / 2)) >> 1;
        off[k] = 2u * (d * BS + 8 * ((chunk & 1) ^ E::vswz(d)));
      } else {
        const int d = (chunk - E::kHalf) >> 2;
        off[k] = 2u * (d * BS + 8 * ((chunk & 3) ^ E::vswz(d)));
      }
    }
  }
  // The window of stage st, which begins with it; windows are entered in order.
  __device__ __forceinline__ void enter(int st) {
    now = next;
    next = pages.entry(first + (st + kWindow) * kPerStage + lane);
  }
  __device__ __forceinline__ const char* block(int st) const {
    const int64_t e = pages.block(__builtin_amdgcn_readlane(now, st % kWindow * kPerStage + half));
    return pool + (e * hkv + head) * (BS * D * 2);
  }
  __device__ __forceinline__ void load(const char* src, uint4* slot, int k) const {
    load_lds<kKeep>(src, BS * D * 2, off[k], 0, slot + (kStageLoads * wave + k) * 64);
  }
};

// Every wave of the workgroup runs this for the same tile; on return e holds the
// wave's row tile (nothing where wave * 32 >= n_packed), and its rows' loads are
// done.
template <int D, int BS>
__device__ __forceinline__ void wide_tile(const ChunkArgs& a, const Tile& w, const Pages& pg, uint4 (*smem)[D * 8], int lane,
                                          int wave, Engine<__bf16, D, BS>& e) {
  using E = Engine<__bf16, D, BS>;
  using Loader = RingLoader<D, BS>;
  constexpr int kStageLoads = Loader::kStageLoads;
  constexpr int NP = D / 16;     // products of the scores, and of P.V: a slot each
  constexpr int NCt = D / 32;
  static_assert(2 * E::kHalf == D * 8, "a ring slot is a stage");
  const int r32 = lane & 31, g = lane >> 5;
  const bool owns = wave * 32 < w.n_packed;
  const int hmin = uniform(wave_min_int(e.hz[0]));
  const float c = a.scale_log2, masked = c < 0.0f ? -kNegInf : kNegInf;
  float& m = e.m[0];
  float& l = e.l[0];
  auto& o = e.o;
  // Per-lane LDS addresses of the operands in ring slot 0 (see Engine).
  const uint32_t smem_base = lds_addr(&smem[0][0]);
  uint32_t kaddr[4], vaddr[2];
  {
    const int t = 16 * (r32 >> 4) + 8 * ((r32 >> 2) & 1) + 4 * ((r32 >> 3) & 1) + (r32 & 3);
#pragma unroll
    for (int s = 0; s < 4; ++s) kaddr[s] = smem_base + 16u * (t * E::kChunksPerToken + ((2 * s + g) ^ E::kswz(t)));
#pragma unroll
    for (int h = 0; h < 2; ++h)
      vaddr[h] = smem_base + 16u * (E::kHalf + (BS == 16 ? E::kHalf / 2 * h + 2 * r32 + (g ^ E::vswz(r32))
                                                         : 4 * r32 + ((2 * h + g) ^ E::vswz(r32))));
  }
  auto slot_off = [&](int st) __attribute__((always_inline)) { return static_cast<uint32_t>(st % kRing) * (E::kHalf * 32); };
  auto read_k = [&](u32x4 (&kr)[NP], int s, uint32_t soff) __attribute__((always_inline)) {
    kr[s] = lds_read_b128(s < 4 ? kaddr[s] + soff : (kaddr[s - 4] + soff) ^ 128u, 0);
  };
  auto read_v = [&](u32x4 (&vr)[NP], int i, uint32_t soff) __attribute__((always_inline)) {  // vr[NCt * h + ct]
    const int h = i / NCt, ct = i % NCt;
    vr[i] = BS == 16 ? lds_read_b128(vaddr[0] + soff, E::kHalf * 8 * h + 1024 * ct) : lds_read_b128(vaddr[h] + soff, 2048 * ct);
  };

  {
    const int tb0 = w.tok_lo, tok_hi = w.tok_hi;
    const int nstage = (tok_hi - tb0 + 31) / 32;
    Loader ld;
    ld.init(a, pg, w.head, tb0, wave, lane);
    barrier_lds();  // the last tile's reads of the ring are done
    // Stages from here on hold positions outside the range or past a row's last.
    const int inner = max(0, (min(tok_hi, hmin < INT_MAX ? hmin + 1 : INT_MAX) - tb0) / 32);

    struct State {
      f32x16 sc;       // scores of the stage
      uint32_t pw[8];  // probabilities of the stage before, as bf16 pairs
      u32x4 vr[NP];    // V of the stage before
    };
    auto score_product = [&](f32x16& sc, int s, const u32x4 (&kr)[NP]) __attribute__((always_inline)) {
      f32x16 acc;
      if (s == 0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] = 0.0f;
      } else {
        acc = sc;
      }
      sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kr[s]), e.q[s], acc, 0, 0, 0);
    };
    auto pv_product = [&](int i, const State& x) __attribute__((always_inline)) {
      const int h = 4 * (i / NCt), ct = i % NCt;
      o[ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          __builtin_bit_cast(bf16x8, x.vr[i]),
          __builtin_bit_cast(bf16x8, u32x4{x.pw[h], x.pw[h + 1], x.pw[h + 2], x.pw[h + 3]}), o[ct], 0, 0, 0);
    };
    // The pair of stages a publish makes room for, loaded until the next one.
    // Behind the last stage these are loads of blocks that nothing reads: so the
    // number of loads in flight is always the same (but for those of the table,
    // which can only make a wait longer), and the loop needs no variant for its
    // end.
    const char* src[kPer] = {nullptr, nullptr};
    int st_load = 0;
    auto load = [&](int i) __attribute__((always_inline)) {
      ld.load(src[i / kStageLoads], smem[(st_load + i / kStageLoads) % kRing], i % kStageLoads);
    };
    // One stage. FIRST: no stage before it; LAST: none after it; PUBLISH: stages
    // st + 1 and st + 2 become readable (this wave's loads of them have landed,
    // and the barrier says so of every wave's), stages up to st - 1 are no longer
    // read. LOAD: first of the two loads issued here.
    auto stage = [&](auto owns_c, auto first_c, auto last_c, auto publish_c, auto load_c, int st, State& x,
                     u32x4 (&kr)[NP]) __attribute__((always_inline)) {
      constexpr bool OWNS = decltype(owns_c)::value, FIRST = decltype(first_c)::value;
      constexpr bool LAST = decltype(last_c)::value, PUBLISH = decltype(publish_c)::value;
      constexpr int LOAD = decltype(load_c)::value;
      if constexpr (PUBLISH) {
        wait_vmcnt<3 * kStageLoads>();
        barrier_only();
        st_load = st + kAhead;
        if (st_load % Loader::kWindow == 0) ld.enter(st_load);
#pragma unroll
        for (int i = 0; i < kPer; ++i) src[i] = ld.block(st_load + i);
      }
      if constexpr (!OWNS) {
        if constexpr (LOAD >= 0) {
#pragma unroll
          for (int i = 0; i < kStageLoads; ++i) load(LOAD + i);
        }
      } else {
        // 2 NP slots of one product each: the first half the P.V of the stage before,
        // the second the scores of the stage after. The steps of an element (scale,
        // exponential, sum, conversion) lie one or more slots apart so that none waits.
        float sv[16], ex[16], pv[16], ps = 0.0f;
        uint32_t pw[8];
#pragma unroll
        for (int i = 0; i < 16; ++i) sv[i] = x.sc[i];
        if (__builtin_expect(st >= inner, 0)) {
          const int hi = min(tok_hi - 1, e.hz[0]) - (tb0 + st * 32 + 8 * g);
#pragma unroll
          for (int i = 0; i < 16; ++i) sv[i] = 16 * (i >> 3) + (i & 7) > hi ? masked : sv[i];
        }
        const float nm = -m;
        const uint32_t k_off = slot_off(st + 1), v_off = slot_off(st);
        // The slot that scales element i; its sum and conversion follow kLag later.
        constexpr int kLag = NP == 8 ? 3 : 2;
        auto slot_of = [](int i) { return 3 * i * NP / 32; };
        // Slots between the read of a K operand and its product, and the LDS reads
        // issued since at the wait for it. (Read as late as this, the operands of K
        // and V fit the registers together.)
        constexpr int kLate = NP == 8 ? 3 : 2, kFirstV = NP == 8 ? 6 : 3;
        constexpr int kSince[8] = {NP == 8 ? 4 : 2, NP == 8 ? 5 : 3, NP == 8 ? 5 : 3, NP == 8 ? 5 : 2, 5, 5, 4, 2};
#pragma unroll
        for (int t = 0; t < 2 * NP; ++t) {
          if (!FIRST && t < NP) pv_product(t, x);
          if (!LAST && t >= NP) {
            lds_wait(kr[t - NP], kSince[t - NP]);
            score_product(x.sc, t - NP, kr);
          }
          if (!LAST && t >= NP - kLate && t < 2 * NP - kLate) read_k(kr, t - (NP - kLate), k_off);
          if (t >= kFirstV && t < NP + kFirstV) read_v(x.vr, t - kFirstV, v_off);
          if (LOAD >= 0 && t % 8 == 4) load(LOAD + t / 8);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            if (t == slot_of(i)) ex[i] = __builtin_fmaf(sv[i], c, nm);
            if (t == slot_of(i) + 1) pv[i] = exp2_fast(ex[i]);
            if (t == slot_of(i) + kLag) ps += pv[i];
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (t == slot_of(2 * i + 1) + kLag) {
              pw[i] = pack2(pv[2 * i], pv[2 * i + 1]);
              asm volatile("" : "+v"(pw[i]));  // here, not behind the branch below
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        const uint64_t past = __ballot(!(ps <= kSlackSum));
        if (__builtin_expect(past != 0, 0)) {
          float mx = sv[0] * c;
#pragma unroll
          for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sv[i] * c);
          mx = fmaxf(mx, __shfl_xor(mx, 32));
          if (row_past(past, lane) && mx > m) {  // both lanes of the row agree
            const float alpha = exp2_fast(m - mx);
            l *= alpha;
#pragma unroll
            for (int i = 0; i < NCt; ++i) o[i] *= alpha;
            m = mx;
          }
          const float ref = m == kNegInf ? 0.0f : m;
          ps = 0.0f;
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            const float p0 = exp2_fast(__builtin_fmaf(sv[i], c, -ref)), p1 = exp2_fast(__builtin_fmaf(sv[i + 1], c, -ref));
            ps += p0;  // in the order above: rows that stay keep their bits
            ps += p1;
            pw[i / 2] = pack2(p0, p1);
          }
        }
        l += ps;
#pragma unroll
        for (int i = 0; i < 8; ++i) x.pw[i] = pw[i];
        lds_wait(x.vr);
        if constexpr (LAST) {
          const int tb = tb0 + st * 32;
          if (tb + 32 > tok_hi) {  // what lies behind the end may be anything: 0 * NaN
#pragma unroll
            for (int i = 0; i < NP; ++i) x.vr[i] = E::zero_past(x.vr[i], tb + 16 * (i / NCt) + 8 * g, tok_hi);
          }
#pragma unroll
          for (int i = 0; i < NP; ++i) pv_product(i, x);
        }
      }
    };

    // The ring's first stages in flight. (The compiler waits for every load in
    // flight where the queries are first used: four stages are issued before that
    // point and two behind it.)
    auto prologue = [&](auto lo_c, auto hi_c) __attribute__((always_inline)) {
      constexpr int LO = decltype(lo_c)::value, N = decltype(hi_c)::value - LO;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const char* from = ld.block(LO + i);
#pragma unroll
        for (int k = 0; k < kStageLoads; ++k) ld.load(from, smem[LO + i], k);
      }
    };
    prologue(std::integral_constant<int, 0>{}, std::integral_constant<int, 4>{});
    e.settle_q();
    prologue(std::integral_constant<int, 4>{}, std::integral_constant<int, kAhead>{});

    // Every wave runs the same barriers, whether it owns a row tile or not.
    auto run = [&](auto owns_c) __attribute__((always_inline)) {
      constexpr bool OWNS = decltype(owns_c)::value;
      constexpr std::true_type yes{};
      constexpr std::false_type no{};
      constexpr std::integral_constant<int, -1> none{};
      constexpr std::integral_constant<int, 0> load0{};
      constexpr std::integral_constant<int, kStageLoads> load1{};  // the second stage's
      State x;
      u32x4 kr[NP];
      wait_vmcnt<(kAhead - 1) * kStageLoads>();
      barrier_only();  // stage 0 is readable
      if constexpr (OWNS) {
#pragma unroll
        for (int s = 0; s < NP; ++s) read_k(kr, s, 0);
        lds_wait(kr);
#pragma unroll
        for (int s = 0; s < NP; ++s) score_product(x.sc, s, kr);
      }
      if (nstage == 1) {
        stage(owns_c, yes, yes, no, none, 0, x, kr);
      } else {
        stage(owns_c, yes, no, yes, load0, 0, x, kr);
        int st = 0;  // the last stage done
        while (st + 3 < nstage) {
          stage(owns_c, no, no, no, load1, st + 1, x, kr);
          stage(owns_c, no, no, yes, load0, st + 2, x, kr);
          st += 2;
        }
        // One or two stages are left, all loaded.
        if (st + 2 < nstage) {
          stage(owns_c, no, no, no, none, st + 1, x, kr);
          ++st;
        }
        stage(owns_c, no, yes, no, none, st + 1, x, kr);
      }
      wait_vmcnt<0>();
    };
    if (owns) run(std::true_type{});
    else run(std::false_type{});
  }
}

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
__device__ __forceinline__ bool find_slice(const ChunkArgs& a, int slice, int tid, int64_t* wave_sum, Start* start, int* n_slices,
                                           int64_t* total_out, int64_t* pos_out, int64_t* stop_out) {
  const int lane = tid & 63, wave = tid >> 6;
  const int per_thread = (a.n_seqs + 64 * kWaves - 1) / (64 * kWaves);
  const int i0 = min(tid * per_thread, a.n_seqs), i1 = min(i0 + per_thread, a.n_seqs);
  int64_t sum = 0;
  Seq s;
  for (int i = i0; i < i1; ++i) {
    s = seq_of(a, i);
    sum += s.group_cost * s.groups;
  }
  int64_t upto = wave_scan(sum);
  if (lane == 63) wave_sum[wave] = upto;
  __syncthreads();
  int64_t total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) upto += wave_sum[w];
    total += wave_sum[w];
  }
  total = uniform(total);
  const int n = static_cast<int>(min(max(total / kMinSlice, static_cast<int64_t>(1)), static_cast<int64_t>(kChunkSlices)));
  *n_slices = n;
  *total_out = total;
  if (slice >= n || total == 0) return false;
  const int64_t pos = line_cut(total, slice, n);
  *pos_out = pos;
  *stop_out = line_cut(total, slice + 1, n);
  int64_t at = upto - sum;
  if (pos >= at && pos < upto) {
    int i = i0;
    for (; i1 - i0 > 1; ++i) {
      s = seq_of(a, i);
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
  __syncthreads();
  return true;
}

template <typename T, int D, int BS>
__global__ void __launch_bounds__(64 * kWaves, 1) chunk_attn_kernel(ChunkArgs a) {
  using E = Engine<T, D, BS>;
  constexpr int kFloat4s = D / 8;  // of a lane's accumulator
  constexpr bool kWide = std::is_same_v<T, __bf16>;
  __shared__ __align__(256) uint4 smem[kWaves][2 * E::kHalf];  // a slot for each wave; wide: the ring
  __shared__ float2 ml[kWaves][32];
  __shared__ int64_t wave_sum[kWaves];
  __shared__ Start start;
  static_assert(2 * E::kHalf >= kFloat4s * 64, "a wave's slot holds its accumulator");
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
  if (!find_slice(a, slice, tid, wave_sum, &start, &n_slices, &total, &pos, &stop)) return;
  int seq = start.seq, head_group = start.group, nth = start.nth;
  int64_t y0 = start.y0;
  Seq sq;
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
    sq = seq_of(a, uniform(sq.row0), uniform(sq.row0 + sq.rows), uniform(sq.kv));
    const int tile = sq.at(nth), end = uniform(sq.end(tile));
    const int64_t tile_cost = uniform(sq.tile_cost(tile));
    const int64_t y1 = uniform(min(tile_cost, y0 + stop - pos));
    const int tok_lo = uniform(cut(y0, tile_cost, sq.cost, end)), tok_hi = uniform(cut(y1, tile_cost, sq.cost, end));
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
      const bool wide = kWide && row_tiles > kWaves / 2 && tok_hi > tok_lo;  // rows with nothing to see: no stages
      const Bases at = E::bases(lane);
      int ent[E::kBlocks], ahead[E::kBlocks];  // blocks of the stage that is loaded next, and of the one behind it
      auto look_up = [&](int (&to)[E::kBlocks], int tb) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < E::kBlocks; ++b) to[b] = pg.entry(tb / BS + b);
      };
      const bool alone = row_tiles == 1;
      auto issue_k = [&](int off) __attribute__((always_inline)) {
        if (alone) E::template issue_k<kStream>(a, pg, at, ent, head, off, smem[wave]);
        else E::template issue_k<kKeep>(a, pg, at, ent, head, off, smem[wave]);
      };
      auto issue_v = [&](int off) __attribute__((always_inline)) {
        if (alone) E::template issue_v<kStream>(a, pg, at, ent, head, off, smem[wave]);
        else E::template issue_v<kKeep>(a, pg, at, ent, head, off, smem[wave]);
      };
      if (!wide && first < seen) {
        look_up(ent, first);
        look_up(ahead, first + stride);
        issue_k(first % BS);
        issue_v(first % BS);
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
      least = uniform(wave_min_int(least));
      const float c = a.scale_log2;
      if (wide) {
        if constexpr (kWide)
          wide_tile<D, BS>(a, Tile{n_packed, head, tok_lo, tok_hi}, pg, smem, lane, wave, e);
        barrier_lds();  // the ring is read: a wave may load its slot for the next tile
      } else if (works) {
        // K and V of a stage are loaded as soon as the slot's halves have been read:
        // at every wait the loads behind the awaited half are the other half's, kLoads
        // of them. (Lookups are issued in front of the loads of a half: they can only
        // make a wait longer.)
        const uint32_t slot = lds_addr(smem[wave]);
        e.settle_q();
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
        for (int i = 0; i < kFloat4s; ++i) *chunk_at(wave, E::out_row(lane, i), E::out_channel(lane, i) / 4) = e.get(i);
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
          while (line_cut(total, last, n_slices) >= tile_end) --last;
          while (last + 1 < n_slices && line_cut(total, last + 1, n_slices) < tile_end) ++last;
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
          const bool has = i + lane < a.n_seqs && seq_of(a, i + lane).tiles > 0;
          const uint64_t bal = __ballot(has);
          if (bal != 0) found = i + __builtin_ctzll(bal);
        }
        if (found < 0) break;  // not reached: the line ends with the last tile
        seq = uniform(found);
        sq = seq_uniform(a, seq);
      }
    }
  }
}

// Log-sum-exp merge of a split tile: D / 4 lanes per packed row, four channels a
// lane. What bounds it is the way of a load, so many are in flight: with up to
// four pieces (most tiles that a cut goes through have two) a wave takes its next
// rows together, their weights beside their outputs; with more, lane i of a row
// takes the maximum and sum of pieces i, i + D / 4, ..., and the pieces' rows come
// in eight or sixteen at a time, the first of them beside the weights. (Three long
// chunks beside 29 tokens, nearly every tile in two pieces: 19 us when a wave took
// its rows one after the other, 12 so; one token over 1,000 positions in 8 pieces:
// 16.5 us of both launches when the rows came behind the weights, 15.6 so.)
constexpr int kMergeWaves = 4, kMergeGroups = 16;  // of a workgroup; workgroups of a slice

// A packed row of a split tile, as the merge reads and writes it.
struct MergeRow {
  int in_tile;  // of a piece's rows
  size_t out;   // row of out and lse
  __device__ __forceinline__ MergeRow(const ChunkArgs& a, const ChunkSplit& s, int at) {
    const int head = at / s.n_rows, p = at - head * s.n_rows, row = p / a.group;
    in_tile = head * s.row_tiles * 32 + p;
    out = static_cast<size_t>(s.row0 + row) * a.hq + (s.head + head) * a.group + (p - row * a.group);
  }
};

template <typename T, int D>
__device__ __forceinline__ void merge_out(const ChunkArgs& a, const MergeRow& r, int sub, f32x4 o, float m, float l) {
  o *= reciprocal_sum(l);
  if constexpr (sizeof(T) == 4)
    *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + r.out * D + 4 * sub) = o;
  else
    *reinterpret_cast<uint2*>(static_cast<__bf16*>(a.out) + r.out * D + 4 * sub) = make_uint2(pack2(o[0], o[1]), pack2(o[2], o[3]));
  if (a.lse != nullptr && sub == 0) a.lse[r.out] = log_sum(m, l);
}

// Up to kPieces pieces, kTogether steps of rows at a time.
template <typename T, int D, int kPieces, int kTogether>
__device__ __forceinline__ void merge_few(const ChunkArgs& a, const ChunkSplit& s, int slice, int pieces, int lane, int first, int step) {
  constexpr int LPR = D / 4, kRows = 64 / LPR;
  const int rows = s.n_rows * s.heads, sub = lane % LPR;
  bool there[kPieces];
#pragma unroll
  for (int q = 0; q < kPieces; ++q) there[q] = q == 0 || (q < pieces && a.continues[slice + min(q, pieces - 1)] != 0);
  // (the lanes of a wave stay together: rows past the last are computed again)
  for (int i0 = first * kRows * kTogether; i0 < rows; i0 += step * kRows * kTogether) {
    float2 x[kTogether][kPieces];
    f32x4 v[kTogether][kPieces];
#pragma unroll
    for (int k = 0; k < kTogether; ++k) {
      const MergeRow r(a, s, min(i0 + k * kRows + lane / LPR, rows - 1));
#pragma unroll
      for (int q = 0; q < kPieces; ++q) {
        const int i = min(q, pieces - 1);
        const size_t at = piece_row(slice + i, i == 0) + r.in_tile;
        x[k][q] = reinterpret_cast<const float2*>(a.part_ml)[at];
        v[k][q] = *reinterpret_cast<const f32x4*>(a.part_o + at * D + 4 * sub);
      }
    }
#pragma unroll
    for (int k = 0; k < kTogether; ++k) {
      float m = x[k][0].x;
#pragma unroll
      for (int q = 1; q < kPieces; ++q) m = there[q] ? fmaxf(m, x[k][q].x) : m;
      const float ref = m == kNegInf ? 0.0f : m;
      float l = 0.0f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int q = 0; q < kPieces; ++q) {  // (what is no piece's may hold anything)
        const float w = there[q] ? exp2_fast(x[k][q].x - ref) : 0.0f;
        if (there[q]) l += x[k][q].y * w;
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] += there[q] ? v[k][q][c] * w : 0.0f;
      }
      merge_out<T, D>(a, MergeRow(a, s, min(i0 + k * kRows + lane / LPR, rows - 1)), sub, o, m, l);
    }
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(64 * kMergeWaves) chunk_merge_kernel(ChunkArgs a) {
  constexpr int LPR = D / 4, kRows = 64 / LPR;
  const int slice = blockIdx.x, lane = threadIdx.x & 63, sub = lane % LPR;
  const ChunkSplit s = a.splits[slice];
  if (s.n_rows == 0) return;
  const int pieces = s.last - slice + 1, rows = s.n_rows * s.heads;
  const int first = blockIdx.y * kMergeWaves + static_cast<int>(threadIdx.x >> 6), step = kMergeGroups * kMergeWaves;
  if (pieces <= 2) {
    merge_few<T, D, 2, 4>(a, s, slice, pieces, lane, first, step);
    return;
  }
  if (pieces <= 4) {
    merge_few<T, D, 4, 2>(a, s, slice, pieces, lane, first, step);
    return;
  }
  for (int i0 = first * kRows; i0 < rows; i0 += step * kRows) {
    const MergeRow r(a, s, min(i0 + lane / LPR, rows - 1));
    float m = kNegInf, l = 0.0f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int base = 0; base < pieces; base += LPR) {
      const int n = min(LPR, pieces - base), i = base + min(sub, n - 1);
      float2 x = reinterpret_cast<const float2*>(a.part_ml)[piece_row(slice + i, i == 0) + r.in_tile];
      const bool there = sub < n && (i == 0 || a.continues[slice + i] != 0);
      // (what is no piece's may hold anything; a weight of zero leaves it out)
      auto rows_of = [&](auto batch_c) __attribute__((always_inline)) {
        constexpr int kBatch = decltype(batch_c)::value;
        f32x4 v[kBatch];
        auto load = [&](int from) __attribute__((always_inline)) {
#pragma unroll
          for (int q = 0; q < kBatch; ++q) {
            const int k = base + min(from + q, n - 1);
            v[q] = *reinterpret_cast<const f32x4*>(a.part_o + (piece_row(slice + k, k == 0) + r.in_tile) * D + 4 * sub);
          }
        };
        load(0);  // beside the weights
        if (!there) x = make_float2(kNegInf, 0.0f);
        float top = x.x;
#pragma unroll
        for (int by = LPR / 2; by >= 1; by /= 2) top = fmaxf(top, __shfl_xor(top, by));
        top = fmaxf(top, m);
        const float ref = top == kNegInf ? 0.0f : top, mine = exp2_fast(m - ref), f = exp2_fast(x.x - ref);
        float sum = x.y * f;
#pragma unroll
        for (int by = LPR / 2; by >= 1; by /= 2) sum += __shfl_xor(sum, by);
        l = l * mine + sum;
        m = top;
        o *= mine;
        for (int from = 0; from < n; from += kBatch) {
          if (from > 0) load(from);
#pragma unroll
          for (int q = 0; q < kBatch; ++q) {
            const float w = from + q < n ? __shfl(f, lane - sub + min(from + q, n - 1)) : 0.0f;
#pragma unroll
            for (int c = 0; c < 4; ++c) o[c] += w != 0.0f ? v[q][c] * w : 0.0f;
          }
        }
      };
      if (n <= 8) rows_of(std::integral_constant<int, 8>{});
      else rows_of(std::integral_constant<int, 16>{});
    }
    merge_out<T, D>(a, r, sub, o, m, l);
  }
}

using ChunkKernel = void (*)(ChunkArgs);

template <typename T>
ChunkKernel pick_attn(int d, int bs) {
  if (bs != 16 && bs != 32) return nullptr;
  if (d == 64) return bs == 16 ? chunk_attn_kernel<T, 64, 16> : chunk_attn_kernel<T, 64, 32>;
  if (d == 128) return bs == 16 ? chunk_attn_kernel<T, 128, 16> : chunk_attn_kernel<T, 128, 32>;
  return nullptr;
}

template <typename T>
ChunkKernel pick_merge(int d) {
  return d == 64 ? chunk_merge_kernel<T, 64> : d == 128 ? chunk_merge_kernel<T, 128> : nullptr;
}

}  // namespace

// By the sequences that there may be: how many have rows only the GPU knows.
// (Single tokens, 32 query and 8 KV heads of 128, a tile per KV head against this
// rule: 128 sequences of up to 400 positions 51.1 and 38.3 us, 1,024 of up to 64
// 209 and 66, of up to 400 309 and 234, of up to 2,000 994 and 1,002, 256 of up to
// 2,000 254 and 264; 16 heads of 64, 256 of up to 400 127 and 61, 1,024 of up to 2,000
// 1,037 and 955.)
int32_t chunk_tile_heads(int32_t n_seqs, int32_t hkv) {
  int32_t n = 1;
  while (2 * n <= hkv && 2 * n <= kWaves && static_cast<int64_t>(n_seqs) * hkv >= 2ll * n * kChunkSlices) n *= 2;
  return n;
}

bool chunk_supported(int32_t dtype, int32_t head_dim, int32_t block_size) {
  return (dtype == 0 || dtype == 1) && (head_dim == 64 || head_dim == 128) && (block_size == 16 || block_size == 32);
}

static constexpr size_t kNotes = kChunkSlices * (sizeof(ChunkSplit) + sizeof(int32_t));
static constexpr size_t kPieceRows = static_cast<size_t>(kChunkSlices) * 2 * kChunkTileRows;

size_t chunk_workspace_bytes(int32_t head_dim) {
  return kNotes + kPieceRows * (2 + static_cast<size_t>(head_dim)) * sizeof(float);
}

void chunk_workspace(ChunkArgs* a, void* workspace) {
  a->splits = static_cast<ChunkSplit*>(workspace);
  a->continues = reinterpret_cast<int32_t*>(a->splits + kChunkSlices);
  a->part_ml = reinterpret_cast<float*>(static_cast<char*>(workspace) + kNotes);
  a->part_o = a->part_ml + 2 * kPieceRows;
}

hipError_t launch_chunk_attn(const ChunkArgs& a, hipStream_t stream) {
  const ChunkKernel k = a.dtype == 1 ? pick_attn<__bf16>(a.head_dim, a.block_size) : pick_attn<float>(a.head_dim, a.block_size);
  if (k == nullptr) return hipErrorInvalidValue;
  hipLaunchKernelGGL(k, dim3(kChunkSlices), dim3(64 * kWaves), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_chunk_merge(const ChunkArgs& a, hipStream_t stream) {
  const ChunkKernel k = a.dtype == 1 ? pick_merge<__bf16>(a.head_dim) : pick_merge<float>(a.head_dim);
  if (k == nullptr) return hipErrorInvalidValue;
  hipLaunchKernelGGL(k, dim3(kChunkSlices, kMergeGroups), dim3(64 * kMergeWaves), 0, stream, a);
  return hipGetLastError();
}

}  // namespace spork
