// gfx950 attention of a ragged batch's new tokens over the paged cache of 8-bit
// codes (chunk_tiles.h has the split of the work, kvq.hip the cache).
//
// Codes become bf16 (bf16 queries) or fp32 on their way from LDS into the matrix
// instructions, by the conversion that takes the block's power of two along: that
// is exact, so products, softmax and sums are those of a cache of these values,
// at half the bytes. HBM bounds tiles of few rows as it does in bf16; in tiles of
// many the products do, at bf16's rate.
//
// A 16-byte piece of a pool is 16 values, twice what a product takes from a lane:
// it feeds two products. So the products' channels, and tokens, go in another
// order than memory's, the same one for both operands:
//   bf16  stages of 32 tokens. Scores: product 2s + i takes channels 32s + 16g + 8i
//         .. + 7 of a lane (g = lane / 32). A-row r is token 16 (r/4 % 2) + 4 (r/8) +
//         r%4, so that a lane receives its query row's scores of tokens 16g + e
//         (element e): 16 tokens of one block. Values: product i takes tokens 16g +
//         8i .. + 7, so one piece of a channel is both products' operand.
//   fp32  stages of 16 tokens, two row tiles of 16. Scores: product 16s + i takes
//         channels 64s + 16g + i (g = lane / 16); values: product i takes tokens
//         4g + i.
// Each wave keeps kDepth stages in flight (chunk_tiles.h's engines: one behind the
// one it computes), as many bytes as they have. The blocks' entries and scales come 64 at a
// time, a window ahead, into registers: loads beside the stages' would be counted
// with them at every wait.
//
// Probabilities enter the second product in the queries' type (bf16: rounded to
// nearest, at most 2^-8 of each, for the matrix instructions' rate; the row sum is of the
// unrounded ones): outputs of bf16 queries are 0.0020 to 0.0023 (root mean square, of the
// outputs') from those of 64 bits, where their own rounding makes 0.0017. Sums, reference
// and accumulators are fp32.
#include "chunk_wide.h"

namespace spork {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));

// A value in scalar registers of its own: kept in those of the kernel's arguments it
// would be stored and fetched with all sixteen of them. (A pointer is generic then:
// only for those of direct loads, which take it as an integer.)
template <typename T>
__device__ __forceinline__ T alone_in_scalars(T x) {
  asm volatile("" : "+s"(x));
  return x;
}

// The scale of a byte: its power of two.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight codes (two dwords) as bf16 times the scale.
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi, float scale) {
  const u32x4 w = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true))};
  return __builtin_bit_cast(bf16x8, w);
}

__device__ __forceinline__ uint32_t lds_read_b32(uint32_t addr, int off) {
  uint32_t r;
  asm volatile("ds_read_b32 %0, %1 offset:%2" : "=v"(r) : "v"(addr), "i"(off) : "memory");
  return r;
}
template <int N>
__device__ __forceinline__ void lds_wait(uint32_t (&r)[N]) {
  asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(r[0]) : : "memory");
#pragma unroll
  for (int i = 1; i < N; ++i) asm volatile("" : "+v"(r[i]) : : "memory");
}

// Zero the bytes of a dword of 4 tokens from position `first` on that lie at or past `end`.
__device__ __forceinline__ uint32_t zero_past4(uint32_t w, int first, int end) {
  const int n = min(max(end - first, 0), 4);
  return n == 4 ? w : w & ((1u << (8 * n)) - 1u);
}

// A wave's stages of its own: kDepth in flight. Stage k (the wave's k-th) is loaded
// into place k % kDepth of the wave's slot; K and V of stage k + kDepth as soon as
// those of stage k have been read.
template <typename E>
struct DeepStages {
  static constexpr int kB = E::kBlocks;       // entries of a stage
  static constexpr int kWindow = 64 / kB;     // stages of a window
  static constexpr int L = E::kLoads, N = E::kDepth;
  static_assert(N >= 2 && N < kWindow && (2 * N - 1) * L < 64, "waits and windows");
  int first, stride, count;
  const char *k_head, *v_head;  // the head's part of block 0
  uint32_t block_bytes;         // of all heads
  const uint8_t *k_scales, *v_scales;
  int hkv;
  int now, next;  // lane i: block of entry i of the window that is loaded; entry i of the next one, as it is loaded
  // lane i: K and V scale of entry i of the window that is computed (as one: V 16 bits
  // up), and of the next one, as they are loaded: combined there, they would be waited for
  uint32_t scales;
  uint8_t k_first, v_first, k_next, v_next;

  __device__ __forceinline__ int entries(const Pages& pg, int window, int lane) const {
    const int k = min(window * kWindow + lane / kB, count - 1);
    return pg.entry((first + k * stride) / E::kBlock + lane % kB);
  }
  __device__ __forceinline__ void load_scales(uint8_t& k, uint8_t& v) const {
    const size_t at = static_cast<size_t>(now) * hkv;
    k = k_scales[at];
    v = v_scales[at];
  }
  static __device__ __forceinline__ uint32_t both(uint8_t k, uint8_t v) {
    uint32_t x = k | static_cast<uint32_t>(v) << 16;
    asm volatile("" : "+v"(x));  // here: no wait for it is left for the loop
    return x;
  }
  template <int POLICY, bool kValues>
  __device__ __forceinline__ void issue(const Bases& at, int k, uint4* slot) const {
    const char* from[kB];
#pragma unroll
    for (int b = 0; b < kB; ++b) {
      const int block = __builtin_amdgcn_readlane(now, k % kWindow * kB + b);
      from[b] = (kValues ? v_head : k_head) + static_cast<uint64_t>(static_cast<uint32_t>(block)) * block_bytes;
    }
    uint4* to = slot + k % N * E::kStage;
    const int off = (first + k * stride) % E::kBlock;  // (bf16: 0)
    E::template load<POLICY, kValues>(from, at, off, to);
  }
  // Entries of the first windows are asked for, in front of all else of the tile.
  __device__ __forceinline__ void look_up(const ChunkArgs& a, const Pages& pg, int head, int first_, int stride_, int seen, int lane) {
    constexpr int kBytes = E::kBlock * E::kD;
    hkv = a.hkv;
    block_bytes = alone_in_scalars(static_cast<uint32_t>(hkv) * kBytes);
    k_head = alone_in_scalars(static_cast<const char*>(a.k_cache) + static_cast<size_t>(head) * kBytes);
    v_head = alone_in_scalars(static_cast<const char*>(a.v_cache) + static_cast<size_t>(head) * kBytes);
    k_scales = a.k_scale + head;
    v_scales = a.v_scale + head;
    first = first_;
    stride = stride_;
    count = (seen - first - 1) / stride + 1;
    now = entries(pg, 0, lane);
    next = entries(pg, 1, lane);
  }
  template <int POLICY>
  __device__ __forceinline__ void begin(const Pages& pg, const Bases& at, uint4* slot) {
    now = pg.block(now);
    load_scales(k_first, v_first);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      if (k < count) {
        issue<POLICY, false>(at, k, slot);
        issue<POLICY, true>(at, k, slot);
      }
    }
  }
  // Until K, or V, of the stage has landed: behind it are its V (for K), K and V of
  // the `left` stages behind it that are loaded, and K of the next (for V, where it is).
  template <int LEFT>
  static __device__ __forceinline__ void wait_k(int left) {
    if constexpr (LEFT > 0) {
      if (left < LEFT) return wait_k<LEFT - 1>(left);
    }
    wait_vmcnt<(2 * LEFT + 1) * L>();
  }
  template <int LEFT>
  static __device__ __forceinline__ void wait_v(int left) {
    if constexpr (LEFT > 0) {
      if (left < LEFT) return wait_v<LEFT - 1>(left);
    }
    wait_vmcnt<2 * LEFT * L>();
  }
  template <int POLICY>
  __device__ __forceinline__ void run(E& e, const ChunkArgs& a, const Pages& pg, const Bases& at, int tok_hi, int least, float c, int lane,
                                      bool second, uint4* places) {
    const uint32_t slot = lds_addr(places);
    scales = both(k_first, v_first);
    k_next = v_next = 0;
    for (int k = 0; k < count; ++k) {
      const int tb = first + k * stride, ahead = k + N, left = min(N - 1, count - 1 - k);
      const bool more = ahead < count;
      const uint32_t place = slot + k % N * (E::kStage * 16);
      if (k > 0 && k % kWindow == 0) scales = both(k_next, v_next);
      const auto scale = E::scales_at(scales, k % kWindow * kB, lane);
      wait_k<N - 1>(left);
      e.read_k(place, at);  // (waited for: the half may be written again)
      if (more) {
        if (ahead % kWindow == 0) {
          now = pg.block(next);
          asm volatile("" : "+v"(now));
          next = entries(pg, ahead / kWindow + 1, lane);
          load_scales(k_next, v_next);
        }
        issue<POLICY, false>(at, ahead, places);
      }
      e.softmax(tb, tok_hi, tb + E::kTokens > tok_hi || tb + E::kTokens - 1 > least, c, lane, second, scale);
      if (more) wait_vmcnt<(2 * N - 1) * L>();
      else wait_v<N - 1>(left);
      e.read_v(place, at);
      if (more) issue<POLICY, true>(at, ahead, places);
      e.values(tb, tok_hi, lane, second, scale);
    }
  }
};

// The stages that a workgroup's waves share (chunk_wide.h): each wave loads its part of
// a pair of stages as codes into registers, a period of two stages ahead, and writes
// it as bf16 into a ring of three pairs, a pair ahead of the one that is published. So
// every code is converted once, not by every wave that needs it. (LDS is nearly as
// busy as the matrix cores here: codes that came into LDS first, by direct loads, cost
// 2,048 rows behind 30,000 positions 1.86 ms.)
// Instruction i of wave w takes stage i of a pair, its chunks 64 w .. (64 channels:
// the lower four waves the first stage, the others the second, chunks 64 (w % 4) ..),
// the first half of them K. A chunk of K is two of the ring's: its first and last
// eight channels go to chunks 4 (c / 2) + c % 2 and 2 further, the order in which
// load_q has the queries, or the other way round (StageLayout::step).
template <int D, int BS>
struct CodeLoader {
  using E = StageLayout<D, BS, true>;
  static constexpr bool kCoded = true;
  static constexpr int kRing = 6;         // stages of bf16
  static constexpr int kStageLoads = 1;   // (of a stage's place in the period)
  static constexpr int kPairLoads = D / 64;
  static constexpr int kPerStage = 32 / BS, kWindow = 64 / kPerStage;  // entries of a stage, stages of a window
  static constexpr int kSteps = 3;
  const char* pool;
  const uint8_t* scales;
  Pages pages;
  int first;  // the tile's first entry
  uint32_t block_bytes;  // of all heads
  int hkv;
  int wave, lane;
  int stage, half;  // D = 64: the stage of a pair that the wave loads; which block of a stage
  uint32_t off, dst, other;  // of the lane: in a block of codes, in a stage of the ring; bit in which its second chunk there differs
  uint32_t ring;
  int now, next;         // lane i: block of entry i of the window that is loaded; entry of the next one
  uint32_t scale_now, scale_next;
  // of a period
  const char* from[kPairLoads];
  float scale[kPairLoads];
  uint32_t to[kPairLoads];  // stages of the ring
  u32x4 w[kPairLoads];  // the codes

  __device__ __forceinline__ int entries(int st) const { return pages.entry(first + st * kPerStage + lane); }
  __device__ __forceinline__ uint32_t scales_of(int block) const { return scales[static_cast<size_t>(block) * hkv]; }
  __device__ __forceinline__ void init(const ChunkArgs& a, const Pages& pg, int kv_head, int tb0, int wave_, int lane_, uint4* smem) {
    wave = wave_;
    lane = lane_;
    pages = pg;
    first = tb0 / BS;
    hkv = a.hkv;
    block_bytes = alone_in_scalars(static_cast<uint32_t>(hkv) * (BS * D));
    const int part = D == 128 ? wave : wave & 3;  // of a stage, 64 chunks each
    constexpr int kParts = D / 32;                // of K, and of V
    stage = D == 128 ? 0 : wave >> 2;
    const bool values = part >= kParts;
    const int chunk = (values ? part - kParts : part) * 64 + lane;
    pool = alone_in_scalars(static_cast<const char*>(values ? a.v_cache : a.k_cache) + static_cast<size_t>(kv_head) * (BS * D));
    scales = (values ? a.v_scale : a.k_scale) + kv_head;
    if (!values) {
      constexpr int kPerToken = D / 16;
      const int t = chunk / kPerToken, c = chunk % kPerToken;
      half = uniform(BS == 16 ? t / 16 : 0);
      off = (t % BS) * D + 16 * c;
      dst = 16u * (t * E::kChunksPerToken + ((4 * (c >> 1) + 2 * (D == 128 ? c >> 2 : 0) + (c & 1)) ^ E::kswz(t)));
      other = 32;
    } else {
      const int d = BS == 16 ? chunk % D : chunk >> 1, h = BS == 16 ? chunk / D : chunk & 1;
      half = uniform(BS == 16 ? h : 0);
      off = d * BS + (BS == 16 ? 0 : 16 * h);
      dst = 16u * (E::kHalf + (BS == 16 ? E::kHalf / 2 * h + 2 * d + E::vswz(d) : 4 * d + ((2 * h) ^ E::vswz(d))));
      other = 16;
    }
    ring = lds_addr(smem);
    now = pages.block(entries(0));
    next = entries(kWindow);
    scale_now = scales_of(now);
    scale_next = 0;
  }
  // What a period needs to know: the pair of stages from st on is loaded, that from st on converted.
  __device__ __forceinline__ void will_load(int st) {
#pragma unroll
    for (int i = 0; i < kPairLoads; ++i) {
      const int s = D == 128 ? i : stage;
      const int block = __builtin_amdgcn_readlane(now, (st + s) % kWindow * kPerStage + half);
      from[i] = pool + static_cast<uint64_t>(static_cast<uint32_t>(block)) * block_bytes;
    }
  }
  __device__ __forceinline__ void will_convert(int conv) {
#pragma unroll
    for (int i = 0; i < kPairLoads; ++i) {
      const int s = D == 128 ? i : stage;
      scale[i] = scale_of(__builtin_amdgcn_readlane(scale_now, (conv + s) % kWindow * kPerStage + half));
      to[i] = ring + static_cast<uint32_t>((conv + s) % kRing) * (8 * D * 16);
    }
  }
  __device__ __forceinline__ void load(int i) {
    typedef const __attribute__((address_space(1))) char* global;
    typedef const __attribute__((address_space(1))) u32x4* global_u32x4;
    w[i] = *(global_u32x4)((global)from[i] + off);
  }
  __device__ __forceinline__ void convert(int i, int b) const {
    const bf16x8 x = widen(w[i][2 * b], w[i][2 * b + 1], scale[i]);
    asm volatile("ds_write_b128 %0, %1" : : "v"(to[i] + (b == 0 ? dst : dst ^ other)), "v"(x) : "memory");
  }
  // Pairs 0 and 1 loaded; then converted, and pair 2 loaded.
  u32x4 second[kPairLoads];
  __device__ __forceinline__ void begin() {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      will_load(2 * p);
#pragma unroll
      for (int i = 0; i < kPairLoads; ++i) {
        load(i);
        if (p == 0) second[i] = w[i];
      }
    }
  }
  __device__ __forceinline__ void first_pairs() {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      will_convert(2 * p);
#pragma unroll
      for (int i = 0; i < kPairLoads; ++i) {
        const u32x4 later = w[i];
        if (p == 0) w[i] = second[i];
        convert(i, 0);
        convert(i, 1);
        if (p == 0) w[i] = later;
      }
    }
    will_load(4);
#pragma unroll
    for (int i = 0; i < kPairLoads; ++i) load(i);
  }
  // Stage st begins a period: stages st + 4 and st + 5 are converted, st + 6 and st + 7 loaded.
  __device__ __forceinline__ void publish(int st) {
    if ((st + 6) % kWindow == 0) {
      now = pages.block(next);
      asm volatile("" : "+v"(now));
      next = entries(st + 6 + kWindow);
      scale_next = scales_of(now);
    }
    if ((st + 4) % kWindow == 0) {
      scale_now = scale_next;
      asm volatile("" : "+v"(scale_now));
    }
    will_load(st + 6);
    will_convert(st + 4);
  }
  // Step t of the period's stage I.
  template <int I>
  __device__ __forceinline__ void step(int t) {
    if (I >= kPairLoads) return;
    if (t < 2) convert(I, t);
    else load(I);
  }
};

struct Scale2 {
  float k, v;
};

// WIDE: tiles of many row tiles share their stages. A call whose rows cannot make such a
// tile runs the engine without: its registers need not hold both.
template <typename T, int D, int BS, bool WIDE>
struct CodeEngine;

template <int D, int BS, bool WIDE>
struct CodeEngine<__bf16, D, BS, WIDE> {
  using Elem = __bf16;
  using Stages = DeepStages<CodeEngine>;
  static constexpr bool kShifts = true;
  // A tile's start-up: chunks beside 60 tokens, 64 heads, 292 us at 600, 281 at 1,000,
  // 271 at 1,600; 24 prompts of up to 777 tokens with 16 heads of 64 61, 54, 52.5; 96
  // single tokens 152.5, 148, 148.5.
  static constexpr int kTile = 1600;
  static constexpr bool kWide = WIDE;
  // Row tiles of a tile that isn't wide: 16 sequences of 9 rows over 8,000 positions, 64
  // heads in groups of 8 (three row tiles) 111 us with stages of each wave's own, 98 with
  // shared ones; in groups of 4 (two) 74 and 88. Wide tiles are of one KV head; where the
  // batch has tiles enough for two heads each (chunk_tile_heads), tiles of three and four
  // row tiles could take them instead, with stages of each wave's own. With one wide and with
  // two, us: 64 such sequences 330 and 380 (two heads a tile at most), 128 over 4,000 341 and
  // 385 (four); 64 verify rows of 9 beside 128 tokens over 8,000, 32 heads in groups of 8, 379
  // and 386; 192 forks of 8 to 50 rows 342 and 433; 128 chunks of 32 rows over 3,000, groups
  // of 4, 309 and 319; 64 of 96 rows over 2,000, 16 heads of 64, 129 and 143. Short contexts
  // alone lose: 128 of 16 rows over 100 58 and 38, 64 of 128 rows over 200 47 and 38.
  static constexpr int kNarrowTiles = 2;
  static constexpr int kD = D, kBlock = BS;
  static constexpr int kTokens = 32;             // of a stage
  static constexpr int kUnits = 1;               // rows of a lane
  static constexpr int kBlocks = kTokens / BS;   // of a stage
  static constexpr int kPerToken = D / 16;       // 16-byte chunks
  static constexpr int kHalf = kTokens * D / 16; // chunks of K, and of V
  static constexpr int kLoads = kHalf / 64;
  // (64 channels, whose stages have half the bytes: eight tokens over up to 1,500 positions
  // 15.8 us with two in flight, 16.5 with three, 17.0 with four; 96 over up to 8,190 150,
  // 149, 152.)
  static constexpr int kStage = 2 * kHalf, kDepth = 2;
  static constexpr int kSlot = kDepth * kStage;
  static_assert(kWaves * kSlot >= CodeLoader<D, BS>::kRing * 8 * D, "the slots hold the ring");
  static constexpr int kSteps = D / 16, kCt = D / 32;
  bf16x8 q[kSteps];
  f32x16 o[kCt];
  float m[1], l[1];
  int hz[1];  // last visible position of the lane's row

  // The line's unit is what a token of 128 channels takes where HBM bounds it, about 6
  // ns on one compute unit, until the products weigh more. (Three chunks beside 29
  // tokens 190 us at a price of 2 for more than one row tile, 182 at 4, 222 at 8 from
  // five row tiles on.)
  static __device__ __forceinline__ int token_cost(const ChunkArgs&, int row_tiles, int heads) {
    return max(D == 128 ? heads : (heads + 1) / 2, row_tiles <= 1 ? 1 : 4);
  }
  static __device__ __forceinline__ int row(int lane, int) { return lane & 31; }
  static __device__ __forceinline__ int out_row(int lane, int) { return lane & 31; }
  static __device__ __forceinline__ int out_channel(int lane, int i) { return 32 * (i / 4) + 8 * (i % 4) + 4 * (lane >> 5); }
  __device__ __forceinline__ f32x4 get(int i) const {
    const f32x16& v = o[i / 4];
    const int e = 4 * (i % 4);
    return f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]};
  }
  __device__ __forceinline__ float row_sum(int) const { return l[0] + __shfl_xor(l[0], 32); }

  // K: chunk t * kPerToken + (c ^ kswz(t)) holds channels 16c .. of token t. V: chunk
  // d of half h (16-token blocks: a block each) or 2d + (h ^ vswz(d)), tokens 16h .. of
  // channel d. The swizzles spread the lanes of an operand read over the banks.
  static __device__ __forceinline__ int kswz(int t) { return (D == 128 ? t >> 1 : t >> 2) & (kPerToken - 1); }
  static __device__ __forceinline__ int vswz(int d) { return BS == 16 ? 0 : (d >> 3) & 1; }

  __device__ __forceinline__ void load_q(const __bf16* p, int lane, int) {
    const int g = lane >> 5;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) q[s] = as_bf16x8(*reinterpret_cast<const uint4*>(p + 32 * (s / 2) + 16 * g + 8 * (s % 2)));
  }
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
    const int tl = lane / kPerToken, c = lane % kPerToken, r = lane & 31, g = lane >> 5;
    const int t = 16 * ((r >> 2) & 1) + 4 * (r >> 3) + (r & 3);
    Bases x;
    x.kload = tl * D + 16 * (c ^ kswz(tl));
    x.vload = BS == 16 ? 16 * lane : 32 * (lane >> 1) + 16 * ((lane & 1) ^ vswz(lane >> 1));
    x.kread = 16 * (t * kPerToken + (g ^ kswz(t)));
    x.vread = 16 * (kHalf + (BS == 16 ? g * D + r : 2 * r + (g ^ vswz(r))));
    return x;
  }
  // K or V of a stage from its blocks into a place.
  template <int POLICY, bool kValues>
  static __device__ __forceinline__ void load(const char* const (&from)[kBlocks], const Bases& x, int, uint4* to) {
    const uint32_t off = anew(kValues ? x.vload : x.kload);
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      if constexpr (kValues) {  // channels dk .. of a half, or of all 32 tokens
        const int dk = BS == 16 ? 64 * k % D : 32 * k;
        load_lds<POLICY>(from[BS == 16 ? 64 * k / D : 0], BS * D, off, dk * BS, to + kHalf + 64 * k);
      } else {  // tokens tk .. of the stage
        const int tk = 64 * k / kPerToken;
        load_lds<POLICY>(from[tk / BS], BS * D, off ^ (16u * kswz(tk)), (tk % BS) * D, to + 64 * k);
      }
    }
  }
  // The scales that a lane's operands need: of its token's block (K), of its half's (V).
  static __device__ __forceinline__ Scale2 scales_at(uint32_t scales, int i, int lane) {
    const uint32_t s0 = __builtin_amdgcn_readlane(scales, i);
    if constexpr (kBlocks == 1) return Scale2{scale_of(s0 & 0xFF), scale_of(s0 >> 16)};
    const uint32_t s1 = __builtin_amdgcn_readlane(scales, i + 1);
    return Scale2{scale_of((lane & 4 ? s1 : s0) & 0xFF), scale_of((lane & 32 ? s1 : s0) >> 16)};
  }

  u32x4 kop[kSteps / 2], vop[kCt];
  __device__ __forceinline__ void read_k(uint32_t slot, const Bases& b) {
    const uint32_t kr = anew(b.kread);
#pragma unroll
    for (int s = 0; s < kSteps / 2; ++s) kop[s] = lds_read_b128(slot + (kr ^ (32u * s)), 0);
    lds_wait(kop);
  }
  __device__ __forceinline__ void read_v(uint32_t slot, const Bases& b) {
    const uint32_t vr = anew(b.vread);
#pragma unroll
    for (int ct = 0; ct < kCt; ++ct) vop[ct] = lds_read_b128(slot + vr, (BS == 16 ? 512 : 1024) * ct);
    lds_wait(vop);
  }

  uint32_t pw[8];  // the stage's probabilities, as bf16 pairs

  // Scores and softmax of the stage at tb; positions from `end` on are not there,
  // `masked`: a row of the wave doesn't see all of the stage.
  __device__ __forceinline__ void softmax(int tb, int end, bool masked, float c, int lane, bool, const Scale2& scale) {
    f32x16 sc;
#pragma unroll
    for (int e = 0; e < 16; ++e) sc[e] = 0.0f;
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(kop[s / 2][s % 2 * 2], kop[s / 2][s % 2 * 2 + 1], scale.k), q[s], sc, 0, 0, 0);
    float sv[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) sv[e] = sc[e];
    if (masked) {
      const int hi = min(end - 1, hz[0]) - tb - 16 * (lane >> 5);  // the last visible one, from the lane's first
      const float none = c < 0.0f ? -kNegInf : kNegInf;
#pragma unroll
      for (int e = 0; e < 16; ++e) sv[e] = e > hi ? none : sv[e];
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
  __device__ __forceinline__ void values(int tb, int end, int lane, bool, const Scale2& scale) {
    if (tb + kTokens > end) {  // what lies behind the end may be anything: 0 * NaN
#pragma unroll
      for (int i = 0; i < kCt; ++i)
#pragma unroll
        for (int w = 0; w < 4; ++w) vop[i][w] = zero_past4(vop[i][w], tb + 16 * (lane >> 5) + 4 * w, end);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int ct = 0; ct < kCt; ++ct)
        o[ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            widen(vop[ct][2 * i], vop[ct][2 * i + 1], scale.v),
            __builtin_bit_cast(bf16x8, u32x4{pw[4 * i], pw[4 * i + 1], pw[4 * i + 2], pw[4 * i + 3]}), o[ct], 0, 0, 0);
  }
  static __device__ __forceinline__ void wide_tile(const ChunkArgs& a, const Tile& w, const Pages& pg, uint4 (*smem)[kSlot], int lane,
                                                   int wave, CodeEngine& e) {
    spork::wide_tile<D, BS, CodeLoader<D, BS>>(a, w, pg, reinterpret_cast<uint4(*)[D * 8]>(smem), lane, wave, e);
  }
};

template <int D, int BS>
struct CodeEngine<float, D, BS, false> {
  using Elem = float;
  using Stages = DeepStages<CodeEngine>;
  static constexpr bool kShifts = true;
  // 64 single tokens over up to 4,000 positions with 4 query and 2 KV heads of 64 take 30.5
  // us at 500, 28.9 at 1,000, 32.0 at 2,000; of 128 45.6, 41.1, 41.9.
  static constexpr int kTile = kTileCost;
  static constexpr bool kWide = false;
  static constexpr int kNarrowTiles = kWaves;
  static constexpr int kD = D, kBlock = BS;
  static constexpr int kTokens = 16;
  static constexpr int kUnits = 2;
  static constexpr int kBlocks = 1;
  static constexpr int kPerToken = D / 16;
  static constexpr int kHalf = kTokens * D / 16;  // chunks of K, and of V
  static constexpr int kLoads = kHalf / 64;
  // (four stages are what the accumulator's place at a tile's end has)
  static constexpr int kStage = 2 * kHalf, kDepth = 4, kSlot = kDepth * kStage;
  static constexpr int kDt = D / 16;
  f32x4 q[2][kDt];  // [4s + j]: channels 64s + 16g + 4j ..
  f32x4 o[2][kDt];
  float m[2], l[2];
  int hz[2];

  // (Half of it: the same 64 tokens 35.0 and 42.5 us, three chunks of up to 200 rows 22.0
  // against 23.3 and 34.2 against 36.9.)
  static __device__ __forceinline__ int token_cost(const ChunkArgs&, int row_tiles, int heads) {
    return (D == 128 ? 4 : 2) * heads << (row_tiles > 4 ? 3 : row_tiles > 2 ? 2 : row_tiles - 1);
  }
  static __device__ __forceinline__ int row(int lane, int u) { return 16 * u + (lane & 15); }
  static __device__ __forceinline__ int out_row(int lane, int i) { return 16 * (i / kDt) + (lane & 15); }
  static __device__ __forceinline__ int out_channel(int lane, int i) { return 16 * (i % kDt) + 4 * (lane >> 4); }
  __device__ __forceinline__ f32x4 get(int i) const { return o[i / kDt][i % kDt]; }
  __device__ __forceinline__ float row_sum(int u) const {
    const float x = l[u] + __shfl_xor(l[u], 16);
    return x + __shfl_xor(x, 32);
  }
  // K: chunk t * kPerToken + (c ^ kswz(t)); V: chunk d, the stage's 16 tokens of channel d.
  static __device__ __forceinline__ int kswz(int t) { return (D == 128 ? t >> 1 : t >> 2) & (kPerToken - 1); }

  __device__ __forceinline__ void load_q(const float* p, int lane, int u) {
    const int g = lane >> 4;
#pragma unroll
    for (int j = 0; j < kDt; ++j) q[u][j] = *reinterpret_cast<const f32x4*>(p + 64 * (j / 4) + 16 * g + 4 * (j % 4));
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
    const int tl = lane / kPerToken, c = lane % kPerToken, r = lane & 15, g = lane >> 4;
    Bases x;
    x.kload = tl * D + 16 * (c ^ kswz(tl));
    x.vload = lane * BS;
    x.kread = 16 * (r * kPerToken + (g ^ kswz(r)));
    x.vread = 16 * (kHalf + r) + 4 * g;
    return x;
  }
  template <int POLICY, bool kValues>
  static __device__ __forceinline__ void load(const char* const (&from)[1], const Bases& x, int first, uint4* to) {
    const uint32_t off = anew(kValues ? x.vload : x.kload) + (kValues ? first : first * D);
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      if constexpr (kValues) {  // channels 64k ..
        load_lds<POLICY>(from[0], BS * D, off, 64 * k * BS, to + kHalf + 64 * k);
      } else {  // tokens tk ..
        const int tk = 64 * k / kPerToken;
        load_lds<POLICY>(from[0], BS * D, off ^ (16u * kswz(tk)), tk * D, to + 64 * k);
      }
    }
  }
  static __device__ __forceinline__ Scale2 scales_at(uint32_t scales, int i, int) {
    const uint32_t s = __builtin_amdgcn_readlane(scales, i);
    return Scale2{scale_of(s & 0xFF), scale_of(s >> 16)};
  }

  u32x4 kop[kDt / 4];
  uint32_t vop[kDt];
  float p[2][4];  // the stage's probabilities
  __device__ __forceinline__ void read_k(uint32_t slot, const Bases& b) {
    const uint32_t kr = anew(b.kread);
#pragma unroll
    for (int s = 0; s < kDt / 4; ++s) kop[s] = lds_read_b128(slot + (kr ^ (64u * s)), 0);
    lds_wait(kop);
  }
  __device__ __forceinline__ void read_v(uint32_t slot, const Bases& b) {
    const uint32_t vr = anew(b.vread);
#pragma unroll
    for (int j = 0; j < kDt; ++j) vop[j] = lds_read_b32(slot + vr, 256 * j);
    lds_wait(vop);
  }
  // Four codes as fp32 times the scale.
  static __device__ __forceinline__ f32x4 widen4(uint32_t w, float scale) {
    const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, true);
    return f32x4{lo[0], lo[1], hi[0], hi[1]};
  }

  // second: the wave's rows 16 .. 31 are there.
  __device__ __forceinline__ void softmax(int tb, int end, bool masked, float c, int lane, bool second, const Scale2& scale) {
    const int g = lane >> 4;
    f32x4 sc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int j = 0; j < kDt; ++j) {
      const f32x4 k4 = widen4(kop[j / 4][j % 4], scale.k);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sc[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(k4[i], q[0][j][i], sc[0], 0, 0, 0);
        if (second) sc[1] = __builtin_amdgcn_mfma_f32_16x16x4f32(k4[i], q[1][j][i], sc[1], 0, 0, 0);
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (u == 1 && !second) break;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[u][i] = sc[u][i] * c;
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

  __device__ __forceinline__ void values(int tb, int end, int lane, bool second, const Scale2& scale) {
    if (tb + kTokens > end) {
#pragma unroll
      for (int j = 0; j < kDt; ++j) vop[j] = zero_past4(vop[j], tb + 4 * (lane >> 4), end);
    }
#pragma unroll
    for (int j = 0; j < kDt; ++j) {
      const f32x4 v4 = widen4(vop[j], scale.v);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        o[0][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(v4[i], p[0][i], o[0][j], 0, 0, 0);
        if (second) o[1][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(v4[i], p[1][i], o[1][j], 0, 0, 0);
      }
    }
  }
  static __device__ __forceinline__ void wide_tile(const ChunkArgs&, const Tile&, const Pages&, uint4 (*)[kSlot], int, int, CodeEngine&) {}
};

template <typename T, bool WIDE>
hipError_t launch(const ChunkArgs& a, hipStream_t stream) {
  const auto k = a.head_dim == 128 ? (a.block_size == 16 ? chunk_attn_kernel<CodeEngine<T, 128, 16, WIDE>> : chunk_attn_kernel<CodeEngine<T, 128, 32, WIDE>>)
                                   : (a.block_size == 16 ? chunk_attn_kernel<CodeEngine<T, 64, 16, WIDE>> : chunk_attn_kernel<CodeEngine<T, 64, 32, WIDE>>);
  hipLaunchKernelGGL(k, dim3(kChunkSlices), dim3(64 * kWaves), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kvq_attn(const ChunkArgs& a, hipStream_t stream) {
  if (a.dtype == 0) return launch<float, false>(a, stream);
  // (all rows in one sequence would make at most this many packed rows)
  constexpr int kNarrow = CodeEngine<__bf16, 128, 16, true>::kNarrowTiles;
  const bool wide = static_cast<int64_t>(a.n_rows) * a.group > 32 * kNarrow;
  return wide ? launch<__bf16, true>(a, stream) : launch<__bf16, false>(a, stream);
}

}  // namespace spork
