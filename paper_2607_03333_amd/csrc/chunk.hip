// gfx950 attention of the new tokens of a ragged batch, prompt chunks and single
// tokens alike, over the paged cache of bf16 or fp32 values. Lengths, offsets and
// block tables are read on the device; nothing of the work split comes from the
// host (chunk_tiles.h).
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
#include "chunk_wide.h"

#include <algorithm>

namespace spork {
namespace {

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

template <typename T, int D, int BS>
struct Engine;

// A wave's loads of the shared stages: instruction k of wave w fills chunks
// (kStageLoads * w + k) * 64 + lane of a stage (the lower four waves K, the upper
// four V), from one block, at a scalar base plus the lane's fixed offset. The
// table goes through registers: lane i holds entry i of the window of 64 that the
// loads are in, and of the next one.
template <int D, int BS>
struct RingLoader {
  using E = StageLayout<D, BS, false>;
  static constexpr bool kCoded = false;
  static constexpr int kRing = 8;  // stages
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
  __device__ __forceinline__ void init(const ChunkArgs& a, const Pages& pg, int kv_head, int tb0, int wave_, int lane_, uint4*) {
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

template <int D, int BS>
struct Engine<__bf16, D, BS> : StageLayout<D, BS, false> {
  using Layout = StageLayout<D, BS, false>;
  using Layout::kChunksPerToken;
  using Layout::kHalf;
  using Layout::kswz;
  using Layout::vswz;
  using Layout::zero_past;
  using Elem = __bf16;
  using Stages = int;
  static constexpr int kDepth = 1;
  static constexpr bool kShifts = false;
  static constexpr int kTile = kTileCost;
  static constexpr bool kWide = true;
  static constexpr int kNarrowTiles = kWaves / 2;  // row tiles of a tile that isn't wide
  static constexpr int kD = D, kBlock = BS;
  static constexpr int kTokens = 32;                // of a stage
  static constexpr int kUnits = 1;                  // rows of a lane
  static constexpr int kSlot = 2 * kHalf;
  static constexpr int kLoads = kHalf / 64;         // instructions of K, and of V
  static constexpr int kSteps = D / 16, kCt = D / 32;
  bf16x8 q[kSteps];
  f32x16 o[kCt];
  float m[1], l[1];
  int hz[1];  // last visible position of the lane's row

  static __device__ __forceinline__ int token_cost(const ChunkArgs& a, int row_tiles, int heads) {
    return spork::token_cost(a, row_tiles, heads);
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

  static __device__ __forceinline__ void wide_tile(const ChunkArgs& a, const Tile& w, const Pages& pg, uint4 (*smem)[D * 8], int lane,
                                                   int wave, Engine& e) {
    spork::wide_tile<D, BS, RingLoader<D, BS>>(a, w, pg, smem, lane, wave, e);
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
  using Elem = float;
  using Stages = int;
  static constexpr int kDepth = 1;
  static constexpr bool kShifts = false;
  static constexpr int kTile = kTileCost;
  static constexpr bool kWide = false;
  static constexpr int kNarrowTiles = kWaves;
  static constexpr int kD = D, kBlock = BS;
  static constexpr int kTokens = 16;
  static constexpr int kUnits = 2;
  static constexpr int kChunksPerToken = D / 4;
  static constexpr int kHalf = kTokens * D / 4;
  static constexpr int kSlot = 2 * kHalf;
  static constexpr int kLoads = kHalf / 64;
  static constexpr int kDt = D / 16;
  f32x4 q[2][kDt];  // channels 16j + 4g + i
  f32x4 o[2][kDt];
  float m[2], l[2];
  int hz[2];

  static __device__ __forceinline__ int token_cost(const ChunkArgs& a, int row_tiles, int heads) {
    return spork::token_cost(a, row_tiles, heads);
  }
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

// Log-sum-exp merge of a split tile: D / 4 lanes per packed row, four channels a
// lane. What bounds it is the way of a load, so many are in flight: with up to
// four pieces (most tiles that a cut goes through have two) a wave takes its next
// rows together, their weights beside their outputs; with more, lane i of a row
// takes the maximum and sum of pieces i, i + D / 4, ..., and the pieces' rows come
// in eight or sixteen at a time, the first of them beside the weights. (Three long
// chunks beside 29 tokens, nearly every tile in two pieces: 19 us when a wave took
// its rows one after the other, 12 so; one token over 1,000 positions in 8 pieces:
// 16.5 us of both launches when the rows came behind the weights, 15.6 so.)
constexpr int kMergeWaves = 4, kMergeGroups = 16;  // of a workgroup; workgroups of a slice, at most

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
  const int first = blockIdx.y * kMergeWaves + static_cast<int>(threadIdx.x >> 6), step = static_cast<int>(gridDim.y) * kMergeWaves;
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
  if (d == 64) return bs == 16 ? chunk_attn_kernel<Engine<T, 64, 16>> : chunk_attn_kernel<Engine<T, 64, 32>>;
  if (d == 128) return bs == 16 ? chunk_attn_kernel<Engine<T, 128, 16>> : chunk_attn_kernel<Engine<T, 128, 32>>;
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
  // No more workgroups of a slice than a tile can have rows for (one token over 1,000
  // positions of 8-bit codes 14.3 us with all 16, 13.95 with one).
  const int64_t rows = std::min(static_cast<int64_t>(a.n_rows) * a.group * a.most_heads, static_cast<int64_t>(kChunkTileRows));
  const int per_group = kMergeWaves * 64 / (a.head_dim / 4);
  const int groups = static_cast<int>(std::min((rows + per_group - 1) / per_group, static_cast<int64_t>(kMergeGroups)));
  hipLaunchKernelGGL(k, dim3(kChunkSlices, groups), dim3(64 * kMergeWaves), 0, stream, a);
  return hipGetLastError();
}

}  // namespace spork
