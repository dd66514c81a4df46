// gfx950 writes into the cache of 8-bit codes, and its block copies.
//
// A block and head has one scale for its keys and one for its values, 2^e: the
// least e with max|x| <= 448 * 2^e over the tokens that it holds, 448 being the
// largest code. A code is x / 2^e, rounded to nearest (ties to even); since the
// scale is a power of two the division is exact, and a code means the same value
// whatever the scale, but for the smallest. A step's tokens of a block raise e
// where they need it; the codes of the tokens in front of them are then written
// anew (again exact, but for those that fall below 2^-6 of the scale).
//
// A run is the step's consecutive tokens of a block. Three kinds of workgroups share
// the launch: keys and values of four KV heads, a head a wave, of the runs that begin
// in a window of rows; and query heads. Nothing is left to atomics.
//   keys     16 bytes a lane and load, D / 16 lanes a token (turn.h). Norm and
//            rotation are in 64 bits: 32 would put values that lie near the middle
//            of two codes on the wrong side. What is kept of the result is 16 bits
//            rounded to odd, from which the 8 bits come out as from the 64.
//   values   four tokens of eight channels a lane, packed by channel and turned
//            through LDS: the pool is channel-major. A run that doesn't fill its
//            block is put into the 16 bytes of each channel that the block holds.
//   queries  in 32 bits, as in rope.hip.
// Rows read once and codes written once bound it: a prompt of 4,096 tokens with 32
// query and 8 KV heads of 128, normed and turned, 92 MB, takes 22.8 us (4.05 TB/s; a
// large copy has 5.1, which would be 18). The keys' arithmetic in 64 bits and their two
// barriers a run go beside the queries' rows, two thirds of the bytes; registers
// decide how many workgroups do (166 of them 24.4 us, 125 22.8; 101 with heads of 64, and
// 161 and 125 in blocks of 32, where the prompt takes 3% longer; fp32 rows 129 to 213;
// keys that come ready 64 to 125). A step of few tokens costs a launch and the waits for
// slots, rows and old codes: 96 tokens 9.9 us. With fewer than four KV heads the waves of
// keys and values that have none only find runs and wait: a prompt of 4,096 tokens with 16
// query heads and one KV head 11.8 us for 37 MB (7.2 at a copy's rate).
#include <algorithm>

#include "turn.h"

namespace spork {
namespace {

constexpr int kWriteWaves = 4;
constexpr int kLeastExp = -100, kMostExp = 120;  // of a scale: far from where 32 bits end
constexpr int kBias = 127;

// Least e with top <= 448 * 2^e, from the bits of a finite top >= 0.
__device__ __forceinline__ int scale_exp(uint32_t top) {
  const int e = static_cast<int>(top >> 23) - 127 - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return min(max(e, kLeastExp), kMostExp);
}
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

// The magnitude's bits; what is no finite number counts as nothing (its code is NaN).
__device__ __forceinline__ uint32_t top_bits(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7FFFFFFFu;
  return u < 0x7F800000u ? u : 0u;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  const auto with = [&](float y) __attribute__((always_inline)) { x = max(x, __float_as_uint(y)); };
  with(dpp_mov<0xB1>(__uint_as_float(x)));  // of two, four, eight, and all 16 lanes of a row
  with(dpp_mov<0x4E>(__uint_as_float(x)));
  with(dpp_mov<0x141>(__uint_as_float(x)));
  with(dpp_mov<0x140>(__uint_as_float(x)));
  const auto row = [&](int r) { return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(x), 16 * r)); };
  return max(max(row(0), row(1)), max(row(2), row(3)));
}

// 64 bits to bf16's 16, rounded to odd: the last of the 8 places is set where anything
// was cut off, so that a later rounding to 6 places or fewer sees on which side of a
// middle the value lies: a code has 4, and so has the largest code's multiple that a
// scale is found by. (Below 2^-126, far under the least code: zero.)
__device__ __forceinline__ uint32_t round_odd(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t hi = static_cast<uint32_t>(u >> 32), sign = hi >> 16 & 0x8000u;
  const int e = static_cast<int>(hi >> 20 & 0x7FF) - 1023;
  if (e >= 128) return sign | 0x7F80u | (x == x ? 0u : 0x40u);  // infinities and NaN, and what bf16 doesn't hold
  if (e < -126) return sign;
  return sign | static_cast<uint32_t>(e + 127) << 7 | (hi >> 13 & 0x7Fu) | (((hi & 0x1FFFu) | static_cast<uint32_t>(u)) != 0 ? 1u : 0u);
}

// Eight values as bf16's 16 bits.
struct Odd8 {
  uint32_t w[4];
  __device__ __forceinline__ void set(int i, uint32_t bits) { w[i / 2] = i % 2 == 0 ? bits : w[i / 2] | bits << 16; }
  __device__ __forceinline__ float get(int i) const { return __uint_as_float(i % 2 == 0 ? w[i / 2] << 16 : w[i / 2] & 0xFFFF0000u); }
};

// Four codes. (Infinities are coded as NaN: the codes have none.)
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}
// Four codes at a scale 2^by times theirs.
__device__ __forceinline__ uint32_t recode4(uint32_t w, float by) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), false);
  const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), true);
  return codes4(lo[0] * by, lo[1] * by, hi[0] * by, hi[1] * by);
}
__device__ __forceinline__ uint4 recode16(uint4 w, float by) {
  return make_uint4(recode4(w.x, by), recode4(w.y, by), recode4(w.z, by), recode4(w.w, by));
}

// The lane's run of 8 codes.
template <typename X>
__device__ __forceinline__ uint2 codes8(const X& x, float by) {
  return make_uint2(codes4(x.get(0) * by, x.get(1) * by, x.get(2) * by, x.get(3) * by),
                    codes4(x.get(4) * by, x.get(5) * by, x.get(6) * by, x.get(7) * by));
}

// A run: its first row, its block, the tokens of the block in front of it, and its length.
struct Run {
  int row, tokens, kept;
  int64_t block;
};

// Bytes [lo, hi) of a dword that holds bytes first .. first + 3.
__device__ __forceinline__ uint32_t byte_mask(int first, int lo, int hi) {
  const int l = min(max(lo - first, 0), 4), h = min(max(hi - first, 0), 4);
  const uint64_t m = (uint64_t{1} << (8 * h)) - (uint64_t{1} << (8 * min(l, h)));
  return static_cast<uint32_t>(m);
}

// Dwords of the LDS tile that turns a head's values: a channel's block of codes
// lies in BS / 4 of them, with a gap behind every eight channels, which spreads
// the writes of a wave over the banks.
template <int D, int BS>
constexpr int kTileWords = D * BS / 4 + (D / 8) * (BS / 4);

// What a wave makes of a head of a run, D / 16 lanes a token (keys) or four tokens of
// eight channels a lane (values).
template <typename T, int D, int BS, bool kTurn>
struct Heads {
  static constexpr int kLanes = D / 16, kRows = 64 / kLanes;  // lanes of a token, tokens that a wave holds in two runs
  static constexpr int kKeyPasses = (BS + kRows - 1) / kRows;
  static constexpr int kChunks = D / 8, kQuads = 64 / kChunks, W = BS / 4;
  static constexpr int kValuePasses = (W + kQuads - 1) / kQuads;
  static constexpr int kOld = D * W / 4 / 64;  // 16-byte pieces of a head's block of values, of a lane

  static __device__ __forceinline__ int exponent(uint8_t byte) { return min(max(byte - kBias, kLeastExp), kMostExp); }

  // The run's keys, as they are loaded, and the scale of the tokens in front of them. (Lanes
  // without a token have the last one's: it changes no largest magnitude.)
  struct Keys {
    Raw<T> raw[kKeyPasses][2];
    uint8_t before;
    __device__ __forceinline__ void load(const KvqWriteArgs& a, const Run& run, int head, const Runs& at, int lane) {
      const T* src = static_cast<const T*>(a.k) + run.row * a.k_stride + head * D;
#pragma unroll
      for (int p = 0; p < kKeyPasses; ++p) {
        if (p * kRows >= run.tokens) break;
        const int t = min(p * kRows + lane / kLanes, run.tokens - 1);
        raw[p][0].load(src + t * a.k_stride + at.a);
        raw[p][1].load(src + t * a.k_stride + at.b);
      }
      before = a.pools.k_scale[run.block * a.hkv + head];
    }
  };

  static __device__ __forceinline__ void write_keys(const KvqWriteArgs& a, const Run& run, int head, const Runs& at, const Keys& k,
                                                    const Raw<T> (&weight)[2], const double2* table, int lane) {
    const int c = lane % kLanes;
    std::conditional_t<kTurn, Odd8, Raw<T>> x[kKeyPasses][2];
    uint32_t top = 0;
#pragma unroll
    for (int p = 0; p < kKeyPasses; ++p) {
      if (p * kRows >= run.tokens) break;
      const int t = min(p * kRows + lane / kLanes, run.tokens - 1);
      if constexpr (!kTurn) {
        x[p][0] = k.raw[p][0];
        x[p][1] = k.raw[p][1];
      } else {
        // One pair at a time, from what was loaded to 16 bits: kept in 64, a run's would
        // fill the registers.
        __builtin_amdgcn_sched_barrier(0);
        Raw<T> w[2] = {weight[0], weight[1]};
        w[0].anew();  // (or all of them would be kept in 64 bits over the passes)
        w[1].anew();
        double r = 1.0;
        if (a.turn.k_weight != nullptr) {
          double s = 0.0;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const double v = k.raw[p][i / 8].get(i % 8);
            s += v * v;
          }
          r = norm_factor<D>(s, a.turn.eps);
        }
        Raw<T> raw[2] = {k.raw[p][0], k.raw[p][1]};
        raw[0].anew();  // (as above)
        raw[1].anew();
        const auto value = [&](int i) __attribute__((always_inline)) {
          const double v = raw[i / 8].get(i % 8);
          return a.turn.k_weight != nullptr ? v * (r * w[i / 8].get(i % 8)) : v;
        };
        const auto pairs = [&](auto interleaved) __attribute__((always_inline)) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int lo = interleaved ? 2 * j : j, hi = interleaved ? 2 * j + 1 : 8 + j;
            double u = value(lo), v = value(hi);
            if (at.turns) {
              const double2 cs = table[t * (D / 2) + 8 * c + j];
              const double y = u * cs.x - v * cs.y;
              v = v * cs.x + u * cs.y;
              u = y;
            }
            x[p][lo / 8].set(lo % 8, round_odd(u));
            x[p][hi / 8].set(hi % 8, round_odd(v));
            __builtin_amdgcn_sched_barrier(0);
          }
        };
        if (a.turn.interleaved) pairs(std::true_type{});
        else pairs(std::false_type{});
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) top = max(top, top_bits(x[p][i / 8].get(i % 8)));
    }
    const int before = run.kept > 0 ? exponent(k.before) : kLeastExp;
    const int e = max(before, scale_exp(wave_max(top)));
    const int64_t bh = run.block * a.hkv + head;
    uint8_t* codes = a.pools.k_codes + bh * (BS * D);
    const float by = exp2_int(-e);
#pragma unroll
    for (int p = 0; p < kKeyPasses; ++p) {
      const int t = p * kRows + lane / kLanes;
      if (t >= run.tokens) continue;
      uint8_t* dst = codes + (run.kept + t) * D;
      *reinterpret_cast<uint2*>(dst + at.a) = codes8(x[p][0], by);
      *reinterpret_cast<uint2*>(dst + at.b) = codes8(x[p][1], by);
    }
    if (run.kept > 0 && e > before) {
      const float again = exp2_int(max(before - e, -126));
      for (int i = lane; i < run.kept * (D / 16); i += 64) {
        uint4* p = reinterpret_cast<uint4*>(codes) + i;
        *p = recode16(*p, again);
      }
    }
    if (lane == 0) a.pools.k_scale[bh] = static_cast<uint8_t>(e + kBias);
  }

  static __device__ __forceinline__ void write_values(const KvqWriteArgs& a, const Run& run, int head, uint32_t* tile, int lane) {
    const int chunk = lane % kChunks;
    const int64_t bh = run.block * a.hkv + head;
    uint4* dst = reinterpret_cast<uint4*>(a.pools.v_codes + bh * (BS * D));
    const T* src = static_cast<const T*>(a.v) + run.row * a.v_stride + head * D + 8 * chunk;
    const auto there = [&](int p, int i) {
      const int t = 4 * (p * kQuads + lane / kChunks) + i - run.kept;
      return t >= 0 && t < run.tokens;
    };
    Raw<T> raw[kValuePasses][4];
#pragma unroll
    for (int p = 0; p < kValuePasses; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (there(p, i)) raw[p][i].load(src + (4 * (p * kQuads + lane / kChunks) + i - run.kept) * a.v_stride);
    uint4 old[kOld];
    if (run.tokens < BS) {
#pragma unroll
      for (int i = 0; i < kOld; ++i) old[i] = dst[i * 64 + lane];
    }
    const int before = run.kept > 0 ? exponent(a.pools.v_scale[bh]) : kLeastExp;
    uint32_t top = 0;
#pragma unroll
    for (int p = 0; p < kValuePasses; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) top = there(p, i) ? max(top, top_bits(raw[p][i].get(j))) : top;
    const int e = max(before, scale_exp(wave_max(top)));
    const float by = exp2_int(-e);
#pragma unroll
    for (int p = 0; p < kValuePasses; ++p) {
      const int quad = p * kQuads + lane / kChunks;
      if (quad >= W) continue;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = there(p, i) ? raw[p][i].get(j) * by : 0.0f;
        tile[(8 * chunk + j) * W + chunk * W + quad] = codes4(x[0], x[1], x[2], x[3]);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const float again = exp2_int(max(before - e, -126));
#pragma unroll
    for (int i = 0; i < kOld; ++i) {
      const int at = i * 64 + lane, d = at / (W / 4), part = at % (W / 4);
      uint4 w = *reinterpret_cast<const uint4*>(tile + d * W + d / 8 * W + 4 * part);
      if (run.tokens < BS) {
        uint32_t n[4] = {w.x, w.y, w.z, w.w}, o[4] = {old[i].x, old[i].y, old[i].z, old[i].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int first = 16 * part + 4 * k;
          const uint32_t mine = byte_mask(first, run.kept, run.kept + run.tokens), front = byte_mask(first, 0, run.kept);
          uint32_t rest = o[k];
          if (e > before && front != 0) rest = (recode4(o[k], again) & front) | (o[k] & ~front);
          n[k] = (n[k] & mine) | (rest & ~mine);
        }
        w = make_uint4(n[0], n[1], n[2], n[3]);
      }
      dst[at] = w;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();  // the tile is read: the wave's next run may write it
    if (lane == 0) a.pools.v_scale[bh] = static_cast<uint8_t>(e + kBias);
  }
};

// Rows of a window, at most: with the row in front of it and the longest run that
// begins in it they fit the lanes of a wave.
constexpr int kMostWindow = 16;

// The runs that begin in a window of rows, found by all lanes at once: lane i has the
// slot of row row0 - 1 + i.
template <int BS>
struct Window {
  int64_t slot;
  uint64_t ends, leaders;
  int row0, bad;
  __device__ __forceinline__ Window(const KvqWriteArgs& a, int first_row, int lane) {
    static_assert(1 + kMostWindow + BS <= 64, "a window's rows in a wave's lanes");
    row0 = first_row;
    const int mine = row0 - 1 + lane;
    slot = mine >= 0 && mine < a.n_rows ? a.slots[mine] : -1;
    const bool sound = slot >= 0 && slot < static_cast<int64_t>(a.pools.num_blocks) * BS;
    const int64_t before = __shfl_up(slot, 1);  // (of all lanes: not behind a condition)
    const bool begins = !sound || slot % BS == 0 || before != slot - 1;
    const uint64_t rows = ((uint64_t{1} << min(a.window, a.n_rows - row0)) - 1) << 1, good = __ballot(sound);
    ends = __ballot(begins);
    leaders = ends & good & rows;
    bad = static_cast<int>(__popcll(rows & ~good));
  }
  __device__ __forceinline__ Run next() {
    const int l = __builtin_ctzll(leaders);
    leaders &= leaders - 1;
    const int64_t begin = __shfl(slot, l);
    return Run{row0 - 1 + l, __builtin_ctzll(ends >> (l + 1)) + 1, static_cast<int>(begin % BS), begin / BS};  // (a run ends within BS rows)
  }
};

constexpr int64_t kMostRunGroups = 1536;  // of keys and values, as far as windows can (launch_kvq_write)

// A wave's query heads of one token, twice qk_rope_kernel's (rope.hip): a prompt of 4,096
// tokens 24.1 us with as many, 22.8 with twice, 23.2 with four times as many.
constexpr int kQueryGroups = 2;

template <typename T, int D>
__device__ __forceinline__ void write_queries(const KvqWriteArgs& a, int64_t num_slots, int64_t unit, float2* table, int lane) {
  constexpr int kLanes = D / 16, kHeads = 64 / kLanes;
  const int parts = (a.hq + kQueryGroups * kHeads - 1) / (kQueryGroups * kHeads);
  if (unit >= static_cast<int64_t>(a.n_rows) * parts) return;
  const int row = static_cast<int>(unit / parts), first = static_cast<int>(unit % parts) * (kQueryGroups * kHeads) + lane / kLanes;
  const int64_t slot = a.slots[row];
  const int position = a.turn.rotary_dim > 0 ? a.positions[row] : 0;
  const int c = lane % kLanes;
  const Runs at(a.turn, c);
  const T* src = static_cast<const T*>(a.q) + row * a.q_stride;
  Raw<T> raw[kQueryGroups][2], weight[2];
#pragma unroll
  for (int u = 0; u < kQueryGroups; ++u) {
    const int head = first + u * kHeads;
    if (head < a.hq) {
      raw[u][0].load(src + head * D + at.a);
      raw[u][1].load(src + head * D + at.b);
    }
  }
  if (a.turn.q_weight != nullptr) {
    weight[0].load(static_cast<const T*>(a.turn.q_weight) + at.a);
    weight[1].load(static_cast<const T*>(a.turn.q_weight) + at.b);
  }
  if (slot < 0 || slot >= num_slots) return;
  float2 cs[8];
  if (a.turn.rotary_dim > 0) lane_turns(a.turn, position, table, lane, c, cs);
  T* dst = static_cast<T*>(a.q_out) + row * a.q_out_stride;
#pragma unroll
  for (int u = 0; u < kQueryGroups; ++u) {
    const int head = first + u * kHeads;
    if (head >= a.hq) continue;  // (whole heads: the lanes that reduce together stay together)
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = raw[u][i / 8].get(i % 8);
    if (a.turn.q_weight != nullptr) {
      float w[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) w[i] = weight[i / 8].get(i % 8);
      norm_head<D>(x, w, a.turn.eps);
    }
    if (at.turns) {
      if (a.turn.interleaved) turn_pairs(x, cs, true);
      else turn_pairs(x, cs, false);
    }
    store_run(dst + head * D + at.a, x);
    store_run(dst + head * D + at.b, x + 8);
  }
}

template <typename T, int D, int BS, bool kTurn>
__global__ void __launch_bounds__(64 * kWriteWaves) kvq_write_kernel(KvqWriteArgs a) {
  using H = Heads<T, D, BS, kTurn>;
  constexpr int kTableBytes = kTurn ? BS * (D / 2) * sizeof(double2) : 0, kTilesBytes = kWriteWaves * kTileWords<D, BS> * 4;
  __shared__ __align__(16) char memory[kTableBytes > kTilesBytes ? kTableBytes : kTilesBytes];  // of keys, values or queries
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head_groups = (a.hkv + kWriteWaves - 1) / kWriteWaves;
  const int64_t groups = static_cast<int64_t>(a.phases) * a.stretch * head_groups;  // of keys, and of values
  const int64_t group = blockIdx.x;
  if (kTurn && group >= 2 * groups) {  // (there are none without)
    write_queries<T, D>(a, static_cast<int64_t>(a.pools.num_blocks) * BS, (group - 2 * groups) * kWriteWaves + wave,
                        reinterpret_cast<float2*>(memory) + 64 * wave, lane);
    return;
  }
  const bool values = group >= groups;
  const int at_group = static_cast<int>(values ? group - groups : group);
  const int head = at_group % head_groups * kWriteWaves + wave, place = at_group / head_groups;
  const int64_t row = (static_cast<int64_t>(place % a.stretch) * a.phases + place / a.stretch) * a.window;
  if (row >= a.n_rows) return;
  const int row0 = static_cast<int>(row);
  Window<BS> window(a, row0, lane);
  if (values) {
    uint32_t* tile = reinterpret_cast<uint32_t*>(memory) + wave * kTileWords<D, BS>;
    if (head >= a.hkv) return;
    while (window.leaders != 0) H::write_values(a, window.next(), head, tile, lane);
    return;
  }
  if (head == 0 && lane == 0 && a.bad_slots != nullptr && window.bad > 0) atomicAdd(a.bad_slots, window.bad);
  const Runs at(a.turn, lane % H::kLanes);
  Raw<T> weight[2];
  if constexpr (kTurn) {
    if (a.turn.k_weight != nullptr) {
      weight[0].load(static_cast<const T*>(a.turn.k_weight) + at.a);
      weight[1].load(static_cast<const T*>(a.turn.k_weight) + at.b);
    }
  }
  double2* table = reinterpret_cast<double2*>(memory);
  while (window.leaders != 0) {
    const Run run = window.next();
    typename H::Keys keys;
    if (head < a.hkv) keys.load(a, run, head, at, lane);
    if constexpr (kTurn) {
      const int half = a.turn.rotary_dim / 2;
      if (half > 0) {
        __syncthreads();  // the last run's are read
        for (int i = tid; i < run.tokens * half; i += 64 * kWriteWaves) {
          const int t = i / half, pair = i - t * half;
          table[t * (D / 2) + pair] = pair_turn(a.turn, pair, a.positions[run.row + t]);
        }
        __syncthreads();
      }
    }
    if (head < a.hkv) H::write_keys(a, run, head, at, keys, weight, table, lane);
  }
}

template <typename T, int D, int BS>
hipError_t launch_write(const KvqWriteArgs& a, hipStream_t stream) {
  const bool turn = a.turn.rotary_dim > 0 || a.turn.q_weight != nullptr || a.turn.k_weight != nullptr;
  const auto k = turn ? kvq_write_kernel<T, D, BS, true> : kvq_write_kernel<T, D, BS, false>;
  constexpr int kTaskHeads = kQueryGroups * 64 / (D / 16);
  const int64_t windows = static_cast<int64_t>(a.phases) * a.stretch;
  const int64_t queries = a.q == nullptr ? 0 : static_cast<int64_t>(a.n_rows) * ((a.hq + kTaskHeads - 1) / kTaskHeads);
  const int64_t groups = 2 * windows * ((a.hkv + kWriteWaves - 1) / kWriteWaves) + (queries + kWriteWaves - 1) / kWriteWaves;
  hipLaunchKernelGGL(k, dim3(static_cast<unsigned>(groups)), dim3(64 * kWriteWaves), 0, stream, a);
  return hipGetLastError();
}

// A copy's block and head a wave at a time: the first tokens' codes, both scales.
template <int D, int BS>
__global__ void __launch_bounds__(64) kvq_copy_kernel(KvqPools p, int hkv, const int32_t* copies, const int32_t* n_copies,
                                                      int max_copies) {
  const int i = static_cast<int>(blockIdx.x / static_cast<unsigned>(hkv)), h = static_cast<int>(blockIdx.x % static_cast<unsigned>(hkv));
  if (i >= min(*n_copies, max_copies)) return;
  const int src = copies[3 * i], dst = copies[3 * i + 1], n = copies[3 * i + 2], lane = threadIdx.x;
  if (src < 0 || src >= p.num_blocks || dst < 0 || dst >= p.num_blocks || src == dst || n < 1 || n > BS) return;
  const size_t from = static_cast<size_t>(src) * hkv + h, to = static_cast<size_t>(dst) * hkv + h;
  const uint4* ks = reinterpret_cast<const uint4*>(p.k_codes + from * (BS * D));
  uint4* kd = reinterpret_cast<uint4*>(p.k_codes + to * (BS * D));
  for (int k = lane; k < n * (D / 16); k += 64) kd[k] = ks[k];
  const uint4* vs = reinterpret_cast<const uint4*>(p.v_codes + from * (BS * D));
  uint4* vd = reinterpret_cast<uint4*>(p.v_codes + to * (BS * D));
#pragma unroll
  for (int k = 0; k < D * BS / 16 / 64; ++k) {
    const int at = k * 64 + lane, first = at % (BS / 16) * 16;
    uint4 w = vs[at];
    if (n < BS) {
      const uint4 old = vd[at];
      const auto pick = [&](uint32_t x, uint32_t y, int q) {
        const uint32_t m = byte_mask(first + 4 * q, 0, n);
        return (x & m) | (y & ~m);
      };
      w = make_uint4(pick(w.x, old.x, 0), pick(w.y, old.y, 1), pick(w.z, old.z, 2), pick(w.w, old.w, 3));
    }
    vd[at] = w;
  }
  if (lane == 0) {
    p.k_scale[to] = p.k_scale[from];
    p.v_scale[to] = p.v_scale[from];
  }
}

}  // namespace

bool kvq_supported(int32_t dtype, int32_t head_dim, int32_t block_size) {
  return (dtype == 0 || dtype == 1) && (head_dim == 64 || head_dim == 128) && (block_size == 16 || block_size == 32);
}

hipError_t launch_kvq_write(const KvqWriteArgs& given, hipStream_t stream) {
  KvqWriteArgs a = given;
  // Windows are as narrow as leaves the workgroups of keys and values at most kMostRunGroups:
  // fewer would wait for each other's runs, more find none where runs are long. A workgroup's
  // rows and the time with 8 KV heads of 128, us: 300 single tokens one 10.4, two 10.7, four
  // 14.7; 1,000 one 25.7, four 22.3, eight 28.4; a prompt of 4,096 four 29.2, eight 26.5, 16
  // 25.4. With 4 KV heads: 1,000 single tokens one 15.8, two 14.4, four 16.7; 192 forks' 8 to
  // 50 tokens two 12.7, four 10.7, eight 10.8, 16 11.7.
  const int64_t head_groups = (a.hkv + kWriteWaves - 1) / kWriteWaves;
  a.window = 1;
  while (a.window < kMostWindow && 2 * head_groups * ((a.n_rows + a.window - 1) / a.window) > kMostRunGroups) a.window *= 2;
  // A prompt's runs begin a block apart, in every block_size / window-th window, and every
  // eighth workgroup is on the same XCD: windows go by their phase in a block first (in the
  // rows' order 1,024 tokens took 14.8 us, with 8 KV heads of 128, now 10.7).
  const int windows = (a.n_rows + a.window - 1) / a.window;
  a.phases = std::min(std::max(a.block_size / a.window, 1), windows);
  a.stretch = (windows + a.phases - 1) / a.phases;
  if (a.dtype == 1) {
    if (a.head_dim == 128) return a.block_size == 16 ? launch_write<__bf16, 128, 16>(a, stream) : launch_write<__bf16, 128, 32>(a, stream);
    return a.block_size == 16 ? launch_write<__bf16, 64, 16>(a, stream) : launch_write<__bf16, 64, 32>(a, stream);
  }
  if (a.head_dim == 128) return a.block_size == 16 ? launch_write<float, 128, 16>(a, stream) : launch_write<float, 128, 32>(a, stream);
  return a.block_size == 16 ? launch_write<float, 64, 16>(a, stream) : launch_write<float, 64, 32>(a, stream);
}

hipError_t launch_kvq_copy_batch(const KvqPools& p, int32_t hkv, int32_t head_dim, int32_t block_size, const int32_t* copies,
                                 const int32_t* n_copies, int32_t max_copies, hipStream_t stream) {
  const auto k = head_dim == 128 ? (block_size == 16 ? kvq_copy_kernel<128, 16> : kvq_copy_kernel<128, 32>)
                                 : (block_size == 16 ? kvq_copy_kernel<64, 16> : kvq_copy_kernel<64, 32>);
  hipLaunchKernelGGL(k, dim3(static_cast<unsigned>(max_copies) * static_cast<unsigned>(hkv)), dim3(64), 0, stream, p, hkv, copies,
                     n_copies, max_copies);
  return hipGetLastError();
}

}  // namespace spork
