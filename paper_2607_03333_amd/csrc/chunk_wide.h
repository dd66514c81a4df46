// Tiles of many row tiles: a workgroup's waves, each with a row tile of its own,
// share the stages of keys and values, bf16 in LDS. So all of them are of one KV head
// (chunk_heads, chunk_kernels.h). How the stages come there is the including file's (a
// Loader).
#pragma once
#include "chunk_tiles.h"

namespace spork {
namespace {

// --------------------------------------------------------------------------
// The wide path: tiles of bf16 queries with more row tiles than an engine's
// kNarrowTiles (four over bf16 pools, two over codes). Each wave owns one row tile of 32
// and all of them share every 32-token stage (16 KB for 128 channels), which goes
// through a ring in LDS (Loader::kRing, eight stages, or six of converted codes); a
// barrier publishes two stages at a time and frees the two that were read. The matrix cores bound a stage (D / 8
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
constexpr int kPer = 2;  // stages that a barrier publishes

// How a stage lies in the ring, in 16-byte chunks. K: chunk t * kChunksPerToken + (c ^
// kswz(t)) of token t. V: chunk 2d + q of half h (16-token blocks) or 4d + (q ^
// vswz(d)), tokens 8q .. of channel d. The swizzles spread the lanes of an operand
// read over the banks. CODED: also those of a write of converted codes, which serves
// eight lanes at a time (lane bit 2 is what would bring two of them together: it
// decides which of its two chunks a lane writes first).
template <int D, int BS, bool CODED>
struct StageLayout {
  static constexpr int kChunksPerToken = D / 8;
  static constexpr int kHalf = 32 * D / 8;  // chunks of K, and of V
  static __device__ __forceinline__ int kswz(int t) {
    if constexpr (CODED && D == 64) return (t & 1) << 1 | (t >> 1 & 1) | (t & 4);
    return ((t & 7) | ((t >> 1) & 8)) & (kChunksPerToken - 1);
  }
  static __device__ __forceinline__ int vswz(int d) {
    const int x = BS == 16 ? (d >> 3) & 1 : (d >> 3) & 3;
    return CODED ? x ^ (BS == 16 ? (d >> 2) & 1 : (d >> 1) & 1) : x;
  }
  // Product of the queries that the scores' product s takes: with codes of 128 channels
  // the two halves of a 16-channel piece change places from channel 64 on.
  static constexpr int step(int s) { return CODED && D == 128 && s >= 4 ? s ^ 1 : s; }
  // Zero the elements of an 8-token chunk from position `first` on that lie at or
  // past `end`.
  static __device__ __forceinline__ u32x4 zero_past(u32x4 w, int first, int end) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] &= (first + 2 * i < end ? 0x0000FFFFu : 0u) | (first + 2 * i + 1 < end ? 0xFFFF0000u : 0u);
    return w;
  }
};

// Every wave of the workgroup runs this for the same tile, w.head the same in all of
// them: each loads a part of its keys and values for all; on return e holds the
// wave's row tile (nothing where wave * 32 >= n_packed), and its rows' loads are
// done. Loader: how stages come into the ring.
template <int D, int BS, typename Loader, typename Rows>
__device__ __forceinline__ void wide_tile(const ChunkArgs& a, const Tile& w, const Pages& pg, uint4 (*smem)[D * 8], int lane,
                                          int wave, Rows& e) {
  using E = StageLayout<D, BS, Loader::kCoded>;
  constexpr int kRing = Loader::kRing, kAhead = kRing - kPer, kStageLoads = Loader::kStageLoads;
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
    ld.init(a, pg, w.head, tb0, wave, lane, &smem[0][0]);
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
      sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kr[s]), e.q[E::step(s)], acc, 0, 0, 0);
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
    [[maybe_unused]] const char* src[kPer] = {nullptr, nullptr};
    [[maybe_unused]] int st_load = 0;
    [[maybe_unused]] auto load = [&](int i) __attribute__((always_inline)) {
      if constexpr (!Loader::kCoded) ld.load(src[i / kStageLoads], smem[(st_load + i / kStageLoads) % kRing], i % kStageLoads);
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
        if constexpr (Loader::kCoded) {
          barrier_lds();  // this wave's writes of the stages are done, and every wave's
          ld.publish(st);
        } else {
          wait_vmcnt<3 * kStageLoads>();
          barrier_only();
          st_load = st + kAhead;
          if (st_load % Loader::kWindow == 0) ld.enter(st_load);
#pragma unroll
          for (int i = 0; i < kPer; ++i) src[i] = ld.block(st_load + i);
        }
      }
      if constexpr (!OWNS) {
        if constexpr (Loader::kCoded) {
          if constexpr (LOAD >= 0) {
#pragma unroll
            for (int t = 0; t < Loader::kSteps; ++t) ld.template step<LOAD / kStageLoads>(t);
          }
        } else if constexpr (LOAD >= 0) {
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
          if constexpr (Loader::kCoded) {
            if constexpr (LOAD >= 0) {
              if (t < Loader::kSteps) ld.template step<LOAD / kStageLoads>(t);
            }
          }
          if (!LAST && t >= NP) {
            lds_wait(kr[t - NP], kSince[t - NP]);
            score_product(x.sc, t - NP, kr);
          }
          if (!LAST && t >= NP - kLate && t < 2 * NP - kLate) read_k(kr, t - (NP - kLate), k_off);
          if (t >= kFirstV && t < NP + kFirstV) read_v(x.vr, t - kFirstV, v_off);
          if (!Loader::kCoded && LOAD >= 0 && t % 8 == 4) load(LOAD + t / 8);
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
    [[maybe_unused]] auto prologue = [&](auto lo_c, auto hi_c) __attribute__((always_inline)) {
      constexpr int LO = decltype(lo_c)::value, N = decltype(hi_c)::value - LO;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if constexpr (!Loader::kCoded) {
          const char* from = ld.block(LO + i);
#pragma unroll
          for (int k = 0; k < kStageLoads; ++k) ld.load(from, smem[LO + i], k);
        }
      }
    };
    if constexpr (Loader::kCoded) {
      ld.begin();
      e.settle_q();
      ld.first_pairs();
    } else {
      prologue(std::integral_constant<int, 0>{}, std::integral_constant<int, 4>{});
      e.settle_q();
      prologue(std::integral_constant<int, 4>{}, std::integral_constant<int, kAhead>{});
    }

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
      if constexpr (Loader::kCoded) {
        barrier_lds();  // stages 0 to 3 are readable
      } else {
        wait_vmcnt<(kAhead - 1) * kStageLoads>();
        barrier_only();  // stage 0 is readable
      }
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

}  // namespace
}  // namespace spork
