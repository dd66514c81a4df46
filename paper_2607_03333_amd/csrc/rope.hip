// gfx950 norms and rotations of queries and keys (turn.h has the mathematics).
//
// A wave takes one token and 64 * 16 / D of its heads (16 bytes a lane and load in
// bf16, so that a load covers whole lines of the heads' halves; two or four times as
// many heads take as long). They are loaded before the angles are computed: one pair
// a lane, in 64 bits, exchanged through LDS. HBM bounds it, each row is read and
// written once: 8,192 tokens with 32 query and 4 KV heads of 128, normed and turned,
// 31.1 us for 151 MB (4.85 TB/s); 32,768 with 64 and 8 heads 211 us for 1.21 GB (5.7; a
// copy of 512 MB has 5.1). A few tokens cost a launch: one 8.1 us, 96 with 72 heads 8.7.
// Tokens of fewer heads than a wave takes leave the others' lanes idle: 4 query and 2 KV
// heads of 64 fill 24 of 64, 4,001 such fp32 tokens take 5.8 us on the GPU for 12 MB (2.4
// at a copy's rate); one query and one KV head of 128 fill 16.
#include "turn.h"

namespace spork {
namespace {

constexpr int kRopeWaves = 4;

template <typename T, int D, bool kNorm>
__global__ void __launch_bounds__(64 * kRopeWaves) qk_rope_kernel(RopeArgs a, int parts) {
  constexpr int kLanes = D / 16, kHeads = 64 / kLanes;  // of a head; heads of a group
  __shared__ float2 table[kRopeWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * kRopeWaves + wave;
  if (unit >= static_cast<int64_t>(a.n_rows) * parts) return;
  const int row = static_cast<int>(unit / parts), part = static_cast<int>(unit % parts);
  const int position = a.positions != nullptr ? a.positions[row] : 0;
  if (position < 0) return;
  const int c = lane % kLanes, heads = a.hq + a.hkv;
  const Runs at(a.turn, c);
  Raw<T> raw[2];
  const int head = part * kHeads + lane / kLanes;
  const bool is_q = head < a.hq;
  if (head < heads) {
    const T* p = is_q ? static_cast<const T*>(a.q) + row * a.q_stride + head * D
                      : static_cast<const T*>(a.k) + row * a.k_stride + (head - a.hq) * D;
    raw[0].load(p + at.a);
    raw[1].load(p + at.b);
  }
  float2 cs[8];
  if (a.turn.rotary_dim > 0) lane_turns(a.turn, position, table[wave], lane, c, cs);
  if (head >= heads) return;  // (whole heads: the lanes that reduce together stay together)
  float x[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = raw[i / 8].get(i % 8);
  if constexpr (kNorm) {
    const T* weight = static_cast<const T*>(is_q ? a.turn.q_weight : a.turn.k_weight);
    Raw<T> wr[2];
    wr[0].load(weight + at.a);
    wr[1].load(weight + at.b);
    float w[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = wr[i / 8].get(i % 8);
    norm_head<D>(x, w, a.turn.eps);
  }
  if (at.turns) {
    if (a.turn.interleaved) turn_pairs(x, cs, true);
    else turn_pairs(x, cs, false);
  }
  T* p = is_q ? static_cast<T*>(a.q_out) + row * a.q_out_stride + head * D
              : static_cast<T*>(a.k_out) + row * a.k_out_stride + (head - a.hq) * D;
  store_run(p + at.a, x);
  store_run(p + at.b, x + 8);
}

template <typename T, int D>
hipError_t launch(const RopeArgs& a, hipStream_t stream) {
  constexpr int kHeads = 64 / (D / 16);
  const int parts = (a.hq + a.hkv + kHeads - 1) / kHeads;
  const int64_t groups = (static_cast<int64_t>(a.n_rows) * parts + kRopeWaves - 1) / kRopeWaves;
  const auto k = a.turn.q_weight != nullptr || a.turn.k_weight != nullptr ? qk_rope_kernel<T, D, true> : qk_rope_kernel<T, D, false>;
  hipLaunchKernelGGL(k, dim3(static_cast<unsigned>(groups)), dim3(64 * kRopeWaves), 0, stream, a, parts);
  return hipGetLastError();
}

}  // namespace

bool rows_supported(int32_t dtype, int32_t head_dim) {
  return (dtype == 0 || dtype == 1) && (head_dim == 64 || head_dim == 128);
}

hipError_t launch_qk_rope(const RopeArgs& a, hipStream_t stream) {
  if (a.dtype == 1) return a.head_dim == 128 ? launch<__bf16, 128>(a, stream) : launch<__bf16, 64>(a, stream);
  return a.head_dim == 128 ? launch<float, 128>(a, stream) : launch<float, 64>(a, stream);
}

}  // namespace spork
