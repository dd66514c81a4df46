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
// A run is the step's consecutive tokens of a block. A workgroup takes the runs
// that begin in its window of rows, one after the other; `parts` workgroups share
// a window and deal its tasks among their waves: a KV head's keys, a KV head's
// values, a token's query heads. Nothing is left to atomics.
//   keys     16 bytes a lane and load, D / 16 lanes a token (turn.h). Norm and
//            rotation are in 64 bits: 32 would put values that lie near the middle
//            of two codes on the wrong side. What is kept of the result is 32 bits
//            rounded to odd, from which the 8 bits come out as from the 64.
//   values   four tokens of eight channels a lane, packed by channel and turned
//            through LDS: the pool is channel-major. A run that doesn't fill its
//            block is put into the 16 bytes of each channel that the block holds.
//   queries  in 32 bits, as in rope.hip.
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
#pragma unroll
  for (int by = 32; by >= 1; by >>= 1) x = max(x, static_cast<uint32_t>(__shfl_xor(static_cast<int>(x), by)));
  return x;
}

// 64 bits to 32, rounded to odd: the last place is set where anything was cut off,
// so that a later rounding to fewer places (22 or less) sees on which side of a
// middle the value lies. (Below 2^-126, far under the least code: zero.)
__device__ __forceinline__ float round_odd(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t sign = static_cast<uint32_t>(u >> 32) & 0x80000000u;
  const int e = static_cast<int>(u >> 52 & 0x7FF) - 1023;
  if (e >= 128) return static_cast<float>(x);  // infinities and NaN, and what 32 bits don't hold
  if (e < -126) return __uint_as_float(sign);
  const uint32_t m = static_cast<uint32_t>(u >> 29) & 0x7FFFFFu;
  return __uint_as_float(sign | static_cast<uint32_t>(e + 127) << 23 | m | ((u & 0x1FFFFFFFu) != 0 ? 1u : 0u));
}

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

// A run: its first row and slot, the tokens of its block in front of it, and its length.
struct Run {
  int row, tokens, kept;
  int64_t block;
};

// The lane's run of 8 codes.
__device__ __forceinline__ uint2 codes8(const float* x, float by) {
  return make_uint2(codes4(x[0] * by, x[1] * by, x[2] * by, x[3] * by), codes4(x[4] * by, x[5] * by, x[6] * by, x[7] * by));
}

// A KV head's keys of a run.
template <typename T, int D, int BS, bool kTurn>
__device__ __forceinline__ void write_keys(const KvqWriteArgs& a, const Run& run, int head, const double2* table, int lane) {
  constexpr int kLanes = D / 16, kTokens = 64 / kLanes, kPasses = (BS + kTokens - 1) / kTokens;
  const int c = lane % kLanes;
  const Runs at(a.turn, c);
  const size_t bh = static_cast<size_t>(run.block) * a.hkv + head;
  const int before = run.kept > 0 ? a.pools.k_scale[bh] - kBias : kLeastExp;
  Raw<T> raw[kPasses][2];
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int t = p * kTokens + lane / kLanes;
    if (t < run.tokens) {
      const T* src = static_cast<const T*>(a.k) + (run.row + t) * a.k_stride + head * D;
      raw[p][0].load(src + at.a);
      raw[p][1].load(src + at.b);
    }
  }
  float x[kPasses][16];
  uint32_t top = 0;
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int t = p * kTokens + lane / kLanes;
    if (t >= run.tokens) continue;
    if constexpr (!kTurn) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[p][i] = raw[p][i / 8].get(i % 8);
    } else {
      double y[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) y[i] = raw[p][i / 8].get(i % 8);
      if (a.turn.k_weight != nullptr) {
        Raw<T> wr[2];
        wr[0].load(static_cast<const T*>(a.turn.k_weight) + at.a);
        wr[1].load(static_cast<const T*>(a.turn.k_weight) + at.b);
        double w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = wr[i / 8].get(i % 8);
        norm_head<D>(y, w, a.turn.eps);
      }
      if (at.turns) {
        double2 cs[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) cs[j] = table[t * (D / 2) + 8 * c + j];
        if (a.turn.interleaved) turn_pairs(y, cs, true);
        else turn_pairs(y, cs, false);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) x[p][i] = round_odd(y[i]);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, top_bits(x[p][i]));
  }
  const int e = max(before, scale_exp(wave_max(top)));
  uint8_t* codes = a.pools.k_codes + bh * (BS * D);
  const float by = exp2_int(-e);
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int t = p * kTokens + lane / kLanes;
    if (t >= run.tokens) continue;
    uint8_t* dst = codes + (run.kept + t) * D;
    *reinterpret_cast<uint2*>(dst + at.a) = codes8(x[p], by);
    *reinterpret_cast<uint2*>(dst + at.b) = codes8(x[p] + 8, by);
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

// A KV head's values of a run.
template <typename T, int D, int BS>
__device__ __forceinline__ void write_values(const KvqWriteArgs& a, const Run& run, int head, uint32_t* tile, int lane) {
  constexpr int kChunks = D / 8;                        // runs of 8 channels
  constexpr int kQuads = 64 / kChunks;                  // groups of four tokens that a wave holds at once
  constexpr int kPasses = (BS / 4 + kQuads - 1) / kQuads;
  constexpr int W = BS / 4;
  const int chunk = lane % kChunks;
  const size_t bh = static_cast<size_t>(run.block) * a.hkv + head;
  const int before = run.kept > 0 ? a.pools.v_scale[bh] - kBias : kLeastExp;
  Raw<T> raw[kPasses][4];
  bool there[kPasses][4];
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = 4 * (p * kQuads + lane / kChunks) + i - run.kept;
      there[p][i] = t >= 0 && t < run.tokens;
      if (there[p][i]) raw[p][i].load(static_cast<const T*>(a.v) + (run.row + t) * a.v_stride + head * D + 8 * chunk);
    }
  }
  uint32_t top = 0;
#pragma unroll
  for (int p = 0; p < kPasses; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) top = there[p][i] ? max(top, top_bits(raw[p][i].get(j))) : top;
  const int e = max(before, scale_exp(wave_max(top)));
  const float by = exp2_int(-e);
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int quad = p * kQuads + lane / kChunks;
    if (quad >= W) continue;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = there[p][i] ? raw[p][i].get(j) * by : 0.0f;
      const int d = 8 * chunk + j;
      tile[d * W + chunk * W + quad] = codes4(x[0], x[1], x[2], x[3]);
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  uint4* dst = reinterpret_cast<uint4*>(a.pools.v_codes + bh * (BS * D));
  const bool whole = run.tokens == BS;
  const float again = exp2_int(max(before - e, -126));
#pragma unroll
  for (int i = 0; i < D * W / 4 / 64; ++i) {
    const int at = i * 64 + lane, d = at / (W / 4), part = at % (W / 4);
    uint4 w = *reinterpret_cast<const uint4*>(tile + d * W + d / 8 * W + 4 * part);
    if (!whole) {
      const uint4 old = dst[at];
      uint32_t n[4] = {w.x, w.y, w.z, w.w}, o[4] = {old.x, old.y, old.z, old.w};
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
  __builtin_amdgcn_wave_barrier();  // the tile is read: the wave's next task may write it
  if (lane == 0) a.pools.v_scale[bh] = static_cast<uint8_t>(e + kBias);
}

// A token's query heads.
template <typename T, int D, bool kTurn>
__device__ __forceinline__ void write_queries(const KvqWriteArgs& a, int row, const double2* table, int lane) {
  constexpr int kLanes = D / 16, kHeads = 64 / kLanes;
  const int c = lane % kLanes;
  const Runs at(a.turn, c);
  float2 cs[8];
  if (at.turns) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const double2 t = table[8 * c + j];
      cs[j] = make_float2(static_cast<float>(t.x), static_cast<float>(t.y));
    }
  }
  float w[16];
  if (kTurn && a.turn.q_weight != nullptr) {
    Raw<T> wr[2];
    wr[0].load(static_cast<const T*>(a.turn.q_weight) + at.a);
    wr[1].load(static_cast<const T*>(a.turn.q_weight) + at.b);
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = wr[i / 8].get(i % 8);
  }
  for (int head = lane / kLanes; head < a.hq; head += kHeads) {
    const T* src = static_cast<const T*>(a.q) + row * a.q_stride + head * D;
    Raw<T> raw[2];
    raw[0].load(src + at.a);
    raw[1].load(src + at.b);
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = raw[i / 8].get(i % 8);
    if constexpr (kTurn) {
      if (a.turn.q_weight != nullptr) norm_head<D>(x, w, static_cast<float>(a.turn.eps));
      if (at.turns) {
        if (a.turn.interleaved) turn_pairs(x, cs, true);
        else turn_pairs(x, cs, false);
      }
    }
    T* dst = static_cast<T*>(a.q_out) + row * a.q_out_stride + head * D;
    store_run(dst + at.a, x);
    store_run(dst + at.b, x + 8);
  }
}

template <typename T, int D, int BS, bool kTurn>
__global__ void __launch_bounds__(64 * kWriteWaves) kvq_write_kernel(KvqWriteArgs a) {
  __shared__ double2 table[kTurn ? BS * (D / 2) : 1];
  __shared__ __align__(16) uint32_t tile[kWriteWaves][kTileWords<D, BS>];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int part = blockIdx.x % static_cast<unsigned>(a.parts);
  const int row0 = static_cast<int>(blockIdx.x / static_cast<unsigned>(a.parts)) * a.window;
  const int64_t num_slots = static_cast<int64_t>(a.pools.num_blocks) * BS;
  const int row1 = min(a.n_rows, row0 + a.window);
  for (int row = row0; row < row1; ++row) {
    const int64_t slot = a.slots[row];
    if (slot < 0 || slot >= num_slots) {
      if (part == 0 && tid == 0 && a.bad_slots != nullptr) atomicAdd(a.bad_slots, 1);
      continue;
    }
    Run run;
    run.row = row;
    run.block = slot / BS;
    run.kept = static_cast<int>(slot % BS);
    if (run.kept > 0 && row > 0 && a.slots[row - 1] == slot - 1) continue;  // inside a run
    const int most = min(BS - run.kept, a.n_rows - row);
    const bool goes_on = lane < most && a.slots[row + lane] == slot + lane;
    const uint64_t ends = ~__ballot(goes_on);
    run.tokens = __builtin_ctzll(ends);  // (most <= BS < 64: a bit is set)
    if constexpr (kTurn) {
      const int half = a.turn.rotary_dim / 2;
      if (half > 0) {
        __syncthreads();  // the last run's are read
        for (int i = tid; i < run.tokens * half; i += 64 * kWriteWaves) {
          const int t = i / half, pair = i - t * half;
          table[t * (D / 2) + pair] = pair_turn(a.turn, pair, a.positions[row + t]);
        }
        __syncthreads();
      }
    }
    const int tasks = 2 * a.hkv + (a.q != nullptr ? run.tokens : 0);
    for (int task = part * kWriteWaves + wave; task < tasks; task += a.parts * kWriteWaves) {
      if (task < a.hkv) write_keys<T, D, BS, kTurn>(a, run, task, table, lane);
      else if (task < 2 * a.hkv) write_values<T, D, BS>(a, run, task - a.hkv, tile[wave], lane);
      else write_queries<T, D, kTurn>(a, row + task - 2 * a.hkv, table + (kTurn ? (task - 2 * a.hkv) * (D / 2) : 0), lane);
    }
  }
}

template <typename T, int D, int BS>
hipError_t launch_write(const KvqWriteArgs& a, hipStream_t stream) {
  const bool turn = a.turn.rotary_dim > 0 || a.turn.q_weight != nullptr || a.turn.k_weight != nullptr;
  const auto k = turn ? kvq_write_kernel<T, D, BS, true> : kvq_write_kernel<T, D, BS, false>;
  const int64_t windows = (static_cast<int64_t>(a.n_rows) + a.window - 1) / a.window;
  hipLaunchKernelGGL(k, dim3(static_cast<unsigned>(windows * a.parts)), dim3(64 * kWriteWaves), 0, stream, a);
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
  a.window = a.n_rows <= 512 ? 1 : 8;
  a.parts = 4;
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
