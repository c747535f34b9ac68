// The head's matrix products: logits of a piece of the vocabulary with their row statistics (and their probabilities, kept as bf16 for the
// piece only), and the sums E = P W over a piece.
//
// For many tokens a workgroup of eight waves owns 256 rows x 256 tokens, a wave 128 x 64 of them.  Stages of 64 inputs: both operands go
// from memory to LDS directly, row slabs two stages ahead (they come from HBM), token slabs one (they sit in the caches).  The workgroup
// meets once a stage, before its last quarter, when the next slabs are needed; the requests that refill what was read go out between
// that quarter's matrix instructions, so that the pipe has work right behind the barrier (issued before them: 5.3 ms in place of 4.9 for
// 4096 tokens, 152064 x 5120).
//
// What bounds it, at that size: the chip's power.  1.26..1.32 PFLOP/s by card with the statistics; the library's product that writes the
// logits 1.34..1.41.  The matrix pipe is busy 66 % of the cycles, at 1.5..1.9 GHz; leaving out the statistics gains 2 %.  The sums reach
// 1.29.  Four waves of 128 x 128 take 7.1 ms, eight of 64 x 128 5.2.  Up to 128 tokens it is the head's bytes: 5.8 TB/s at 1 token of
// 152064 x 3584 (188 us).
//
// Operand layout in LDS: rows of 64 inputs as eight 16-byte chunks, chunk c of row r at r * 8 + (c ^ ((r >> 1) & 7)).
#include "lm_head.hpp"
#include "lds_dma.hpp"

namespace qerl {

// RT row tiles and TT token tiles of 32 per wave, WR x WT waves, SA and SB slabs of the operands in LDS
template <int RT_, int TT_, int WR_, int WT_, int SA_, int SB_>
struct HeadCfg {
  static constexpr int RT = RT_, TT = TT_, WR = WR_, WT = WT_, SA = SA_, SB = SB_;
  static constexpr int kWaves = WR * WT, kThreads = 64 * kWaves, kRows = 32 * RT * WR, kTokens = 32 * TT * WT;
  static constexpr int kSlabA = kRows * 8, kSlabB = kTokens * 8;                // 16-byte chunks
  static constexpr int IA = kSlabA / kThreads, IB = kSlabB / kThreads;          // requests per wave and stage
  static_assert(IA * kThreads == kSlabA && IB * kThreads == kSlabB, "whole requests");
  static constexpr int kLds = (SA * kSlabA + SB * kSlabB) * 16;
  static_assert(kLds <= 160 * 1024, "LDS of a compute unit");
  // requests that may be outstanding when stage s + 1 is needed: those behind its own, batches being (token slab, row slab)
  static constexpr int kAfterB = IA + (SB - 2) * (IA + IB), kAfterA = (SA - 2) * (IA + IB);
  static constexpr int kAhead = kAfterA < kAfterB ? kAfterA : kAfterB;
  static constexpr int kDeep = SA > SB ? SA : SB;
};

// Stages [s0, s1) of a tile's product, added to acc.  rows_a / rows_b: byte offsets of the lane's rows for each request.
template <class C>
struct HeadLoop {
  u32x4* lds;
  uint32_t lds0;
  int lane, wave, wr, wt, n32, kg;
  const uint8_t* base_a; const uint8_t* base_b;
  uint32_t off_a[C::IA], off_b[C::IB];
  int64_t k;
  bool active;                                   // the wave has tokens (uniform)

  __device__ __forceinline__ void init(u32x4* memory, int tid) {
    lds = memory; lds0 = lds_address(memory);
    lane = tid & 63; wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    wr = wave % C::WR; wt = wave / C::WR;
    n32 = lane & 31; kg = lane >> 5;
  }
  // row and byte inside it that a lane's request i fetches (rows further by whole requests have the same swizzle)
  static_assert(C::kThreads % 128 == 0, "swizzle of later requests");
  __device__ __forceinline__ int slab_row(int i) const { return wave * 8 + (lane >> 3) + 8 * C::kWaves * i; }
  __device__ __forceinline__ uint32_t slab_col() const { return (uint32_t)(((lane & 7) ^ ((slab_row(0) >> 1) & 7)) * 16); }
  template <int N>
  __device__ __forceinline__ void request(const uint8_t* base, const uint32_t (&off)[N], int slab_chunks, int stage) {
    const uint32_t dst = lds0 + (uint32_t)((slab_chunks + wave * 64) * 16);
    const uint8_t* p = base + (int64_t)stage * 128;
#pragma unroll
    for (int i = 0; i < N; ++i) lds_request(dst + (uint32_t)(i * C::kThreads * 16), p, off[i]);
  }
  // the last stage of a k that is no multiple of 64: through registers, zeros behind k (which is a multiple of 8)
  template <int N>
  __device__ __forceinline__ void copy_tail(const uint8_t* base, const uint32_t (&off)[N], int slab_chunks, int stage) {
    const int64_t at = (int64_t)stage * 128;
    const bool inside = at + slab_col() < k * 2;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(base + off[i] + (inside ? at : -(int64_t)slab_col()));
      lds[slab_chunks + i * C::kThreads + wave * 64 + lane] = inside ? v : u32x4{0u, 0u, 0u, 0u};
    }
  }
  __device__ __forceinline__ int chunk_a(int slot, int j, int t) const {
    const int r = n32;
    return slot + (wr * C::RT * 32 + r) * 8 + ((2 * j + kg) ^ ((r >> 1) & 7)) + t * 256;
  }
  __device__ __forceinline__ int chunk_b(int slot, int j, int t) const {
    const int r = n32;
    return slot + C::SA * C::kSlabA + (wt * C::TT * 32 + r) * 8 + ((2 * j + kg) ^ ((r >> 1) & 7)) + t * 256;
  }
  __device__ __forceinline__ bf16x8 frag(int chunk) const { return __builtin_bit_cast(bf16x8, lds[chunk]); }

  int s1, next_a, next_b, put_a, put_b;          // end of the stages, next ones to fetch and their slots
  __device__ __forceinline__ void fetch_a() {
    if (next_a >= s1) return;
    if (next_a < (int)(k >> 6)) request(base_a, off_a, put_a, next_a); else copy_tail(base_a, off_a, put_a, next_a);
    ++next_a;
    put_a = put_a + C::kSlabA == C::SA * C::kSlabA ? 0 : put_a + C::kSlabA;
  }
  __device__ __forceinline__ void fetch_b() {
    if (next_b >= s1) return;
    const int at = C::SA * C::kSlabA + put_b;
    if (next_b < (int)(k >> 6)) request(base_b, off_b, at, next_b); else copy_tail(base_b, off_b, at, next_b);
    ++next_b;
    put_b = put_b + C::kSlabB == C::SB * C::kSlabB ? 0 : put_b + C::kSlabB;
  }
  // Requests ahead of the first stage: SB - 1 token slabs and SA - 1 row slabs, the last batch (token, row).  Nobody reads LDS meanwhile.
  __device__ __forceinline__ void start(int from, int to) {
    next_a = next_b = from; s1 = to;
    put_a = put_b = 0;
#pragma unroll
    for (int i = 0; i < C::kDeep - 1; ++i) {
      if (i >= C::kDeep - C::SB) fetch_b();
      if (i >= C::kDeep - C::SA) fetch_a();
    }
  }
  // Stages from s0 on (as start was told), added to acc.  SHORT: chains of four stages, their sums added up with what each addition
  // rounds off (see Head32).
  template <bool SHORT>
  __device__ __forceinline__ void run(f32x16 (&acc)[C::RT][C::TT], int s0) {
    float high[SHORT ? C::RT * C::TT * 16 : 1], low[SHORT ? C::RT * C::TT * 16 : 1];
    if constexpr (SHORT) {
#pragma unroll
      for (int i = 0; i < C::RT * C::TT * 16; ++i) high[i] = low[i] = 0.f;
    }
    auto add_up = [&] {
      if constexpr (SHORT) {
#pragma unroll
        for (int i = 0; i < C::RT * C::TT * 16; ++i) {
          const float x = acc[i / 16 / C::TT][i / 16 % C::TT][i % 16], h = high[i], sum = h + x, part = sum - h;
          low[i] += (h - (sum - part)) + (x - part);
          high[i] = sum;
          acc[i / 16 / C::TT][i / 16 % C::TT][i % 16] = 0.f;
        }
      }
    };
    const int full = (int)(k >> 6);              // stages from here on take the tail's way
    auto meet = [&](int s) {                     // everybody has read stage s - 1, and stage s is in LDS
      if (s + C::kDeep - 2 < (s1 < full ? s1 : full)) lds_wait_barrier<C::kAhead>();
      else lds_wait_barrier<0>();
    };
    meet(s0);
    fetch_b();
    fetch_a();
    if (!active) {                               // no tokens for this wave: it fetches and meets only
      for (int s = s0 + 1; s < s1; ++s) {
        meet(s);
        fetch_b();
        fetch_a();
      }
      return;
    }
    int slot_a = 0, slot_b = 0;
    bf16x8 fa[C::RT], fb[C::TT];
#pragma unroll
    for (int t = 0; t < C::TT; ++t) fb[t] = frag(chunk_b(slot_b, 0, t));
#pragma unroll
    for (int t = 0; t < C::RT; ++t) fa[t] = frag(chunk_a(slot_a, 0, t));
    // One step's matrix instructions, the next step's fragments read between them, `between(i)` behind instruction i
    auto step = [&](int ca, int cb, int jn, auto between) {
      bf16x8 na[C::RT], nb[C::TT];
#pragma unroll
      for (int i = 0; i < C::RT * C::TT; ++i) {
        const int t = i / C::TT, tt = i % C::TT;
        acc[t][tt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[t], fb[tt], acc[t][tt], 0, 0, 0);
#pragma unroll
        for (int r = i * (C::RT + C::TT) / (C::RT * C::TT); r < (i + 1) * (C::RT + C::TT) / (C::RT * C::TT); ++r)
          if (r < C::TT) nb[r] = frag(chunk_b(cb, jn, r)); else na[r - C::TT] = frag(chunk_a(ca, jn, r - C::TT));
        between(i);
      }
#pragma unroll
      for (int t = 0; t < C::RT; ++t) fa[t] = na[t];
#pragma unroll
      for (int t = 0; t < C::TT; ++t) fb[t] = nb[t];
    };
    int s = s0, after_a, after_b;
    auto three_steps = [&] {
      after_a = slot_a + C::kSlabA == C::SA * C::kSlabA ? 0 : slot_a + C::kSlabA;
      after_b = slot_b + C::kSlabB == C::SB * C::kSlabB ? 0 : slot_b + C::kSlabB;
#pragma unroll
      for (int j = 0; j < 3; ++j) {
        step(slot_a, slot_b, j + 1, [](int) {});
#pragma unroll
        for (int i = 0; i < C::RT + C::TT; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    const int limit = s1 < full ? s1 : full;
    for (; next_a < limit && next_b < limit; ++s) {       // whole slabs to fetch: their requests go out between the matrix instructions
      three_steps();
      lds_wait_barrier<C::kAhead>();
      const uint32_t dst_b = lds0 + (uint32_t)((C::SA * C::kSlabA + put_b + wave * 64) * 16), dst_a = lds0 + (uint32_t)((put_a + wave * 64) * 16);
      const uint8_t* from_b = base_b + (int64_t)next_b * 128;
      const uint8_t* from_a = base_a + (int64_t)next_a * 128;
      step(after_a, after_b, 0, [&](int i) {
        constexpr int kAll = C::IA + C::IB, kSteps = C::RT * C::TT;
#pragma unroll
        for (int r = i * kAll / kSteps; r < (i + 1) * kAll / kSteps; ++r) {
          if (r < C::IB) lds_request(dst_b + (uint32_t)(r * C::kThreads * 16), from_b, off_b[r < C::IB ? r : 0]);
          else lds_request(dst_a + (uint32_t)((r - C::IB) * C::kThreads * 16), from_a, off_a[r < C::IB ? 0 : r - C::IB]);
        }
        __builtin_amdgcn_sched_barrier(0);
      });
      ++next_a;
      ++next_b;
      put_a = put_a + C::kSlabA == C::SA * C::kSlabA ? 0 : put_a + C::kSlabA;
      put_b = put_b + C::kSlabB == C::SB * C::kSlabB ? 0 : put_b + C::kSlabB;
      slot_a = after_a;
      slot_b = after_b;
      if (SHORT && ((s - s0) & 3) == 3) add_up();
    }
    for (; s < s1; ++s) {
      three_steps();
      if (s + 1 < s1) {
        meet(s + 1);
        fetch_b();
        fetch_a();
        __builtin_amdgcn_sched_barrier(0);
      }
      step(after_a, after_b, 0, [](int) {});     // (behind the last stage the fragments are whatever the slots hold, and not used)
      __builtin_amdgcn_sched_barrier(0);
      slot_a = after_a;
      slot_b = after_b;
      if (SHORT && ((s - s0) & 3) == 3) add_up();
    }
    if constexpr (SHORT) {
      add_up();
#pragma unroll
      for (int i = 0; i < C::RT * C::TT * 16; ++i) acc[i / 16 / C::TT][i / 16 % C::TT][i % 16] = high[i] + low[i];
    }
  }
};

// Row statistics of a wave's tile, from the products in acc; with PROBS acc becomes 2^(s - ref).
// lane l holds of token 32 tt + l % 32 the rows 32 t + 8 q + 4 (l / 32) + 0..3 as elements 4 q .. 4 q + 3
struct HeadLane { int own; float ref; };         // of a lane's token: its own row in the wave's tile, less 4 (l / 32) (or -1); its reference
template <class C, bool PROBS, bool ENTROPY>
__device__ __forceinline__ void head_statistics(f32x16 (&acc)[C::RT][C::TT], const HeadArgs& a, const HeadLane (&of)[C::TT], int M, int64_t r0, int m0, int part,
                                                int lane) {
  const int n32 = lane & 31, kg = lane >> 5;
  const float scale = a.scale;
#pragma unroll
  for (int tt = 0; tt < C::TT; ++tt) {
    const int token = m0 + tt * 32 + n32;
    const bool live = token < M;
    const int own = of[tt].own;
    const bool mine = own >= 0;
    if (__any(mine)) {
      float logit = 0.f;
#pragma unroll
      for (int t = 0; t < C::RT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const bool hit = own == t * 32 + 8 * (i >> 2) + (i & 3);
          logit = hit ? acc[t][tt][i] : logit;
          acc[t][tt][i] = hit ? kNegInf : acc[t][tt][i];
        }
      if (mine && live) a.target_logit[token] = logit * scale;
    }
    if (r0 + 32 * C::RT > a.rows) {
      const int end = (int)(a.rows - r0) - 4 * kg;
#pragma unroll
      for (int t = 0; t < C::RT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[t][tt][i] = t * 32 + 8 * (i >> 2) + (i & 3) < end ? acc[t][tt][i] : kNegInf;
    }
    float top = kNegInf;
#pragma unroll
    for (int t = 0; t < C::RT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, acc[t][tt][i]);
    top = fmaxf(top, __shfl_xor(top, 32, 64)) * scale;
    const float ref = PROBS ? of[tt].ref : top;
    const float base = PROBS ? ref : top == kNegInf ? 0.f : top;
    float sum[2] = {0.f, 0.f}, weighted[2] = {0.f, 0.f};
#pragma unroll
    for (int t = 0; t < C::RT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float d = fmaf(acc[t][tt][i], scale, -base), e = __builtin_amdgcn_exp2f(d);
        sum[i & 1] += e;
        if (ENTROPY) weighted[i & 1] = fmaf(e, fmaxf(d, -1e30f), weighted[i & 1]);     // (0 at rows that do not count, where d is -inf)
        if (PROBS) acc[t][tt][i] = e;
      }
    float s = sum[0] + sum[1], w = weighted[0] + weighted[1];
    s += __shfl_xor(s, 32, 64);
    if (ENTROPY) w += __shfl_xor(w, 32, 64);
    if (live && kg == 0) {
      a.part[(int64_t)token * a.part_ld + part] = HeadPart{ref, s, w, top};
      if (PROBS && !a.again && top > ref + kRaise) {
        atomicMax(a.raise + token, order_key(top));
        a.flag[token / C::kTokens] = 1;          // (several may write the same)
      }
    }
  }
}

// The probabilities in acc as bf16 to p, row-major by token: a lane and its partner 32 further hold rows 4 kg + 0..3 of each eight; two
// swaps per sixteen rows give each of them eight in a row, 16 bytes.
template <class C>
__device__ __forceinline__ void store_probs(const f32x16 (&acc)[C::RT][C::TT], const HeadArgs& a, int M, int64_t r0, int m0, int lane) {
  const int n32 = lane & 31, kg = lane >> 5;
  const int64_t end = (a.rows + 63) & ~(int64_t)63;
#pragma unroll
  for (int tt = 0; tt < C::TT; ++tt) {
    const int token = m0 + tt * 32 + n32;
    uint16_t* out = a.p + (int64_t)token * a.ldp + r0 + 8 * kg;
#pragma unroll
    for (int t = 0; t < C::RT; ++t)
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const f32x16& v = acc[t][tt];
        const auto lo = __builtin_amdgcn_permlane32_swap(pack_bf16x2(v[8 * g], v[8 * g + 1]), pack_bf16x2(v[8 * g + 4], v[8 * g + 5]), false, false);
        const auto hi = __builtin_amdgcn_permlane32_swap(pack_bf16x2(v[8 * g + 2], v[8 * g + 3]), pack_bf16x2(v[8 * g + 6], v[8 * g + 7]), false, false);
        if (token < M && r0 + t * 32 + 16 * g < end) *reinterpret_cast<u32x4*>(out + t * 32 + 16 * g) = u32x4{lo[0], hi[0], lo[1], hi[1]};
      }
  }
}

template <class C, bool PROBS, bool ENTROPY>
__global__ __launch_bounds__(C::kThreads, C::kWaves >= 4 ? C::kWaves / 4 : 1) void head_gemm_kernel(const HeadArgs a, int row_blocks, int blocks_per_xcd) {
  extern __shared__ __attribute__((aligned(256))) u32x4 head_lds[];
  HeadLoop<C> loop;
  loop.init(head_lds, threadIdx.x);
  loop.k = a.k;
  const int M = head_tokens(a), token_blocks = (M + C::kTokens - 1) / C::kTokens;
  const int stages = (int)((a.k + 63) >> 6), total = 8 * blocks_per_xcd * token_blocks;
  int rb = 0, mb = 0;
  HeadLane of[C::TT];
  // The next tile from `tile` on that there is anything to do for; its operands.  Workgroup ids go round-robin to the eight XCDs, each of
  // which takes a contiguous eighth of the row blocks; four of them and all token blocks, rows first, make a group, so that what is in
  // flight on an XCD shares its slabs.
  auto find = [&](int tile) {
    for (; tile < total; tile += (int)gridDim.x) {
      const int xcd = tile & 7, local = tile >> 3, group = local / (4 * token_blocks), in = local - group * 4 * token_blocks;
      const int width = blocks_per_xcd - 4 * group < 4 ? blocks_per_xcd - 4 * group : 4;
      mb = in / width;
      rb = xcd * blocks_per_xcd + 4 * group + in - mb * width;
      if (rb < row_blocks && !(PROBS && a.again && !a.flag[mb])) break;
    }
    return tile;
  };
  auto prepare = [&] {
    const int64_t r0 = (int64_t)rb * C::kRows;
    const int m0 = mb * C::kTokens;
    loop.base_a = uniform_pointer(a.a + r0 * a.lda);
    loop.base_b = uniform_pointer(a.b);
#pragma unroll
    for (int i = 0; i < C::IA; ++i) {
      const int64_t r = r0 + loop.slab_row(i) < a.rows ? loop.slab_row(i) : a.rows - 1 - r0;
      loop.off_a[i] = (uint32_t)(r * a.lda * 2) + loop.slab_col();
    }
#pragma unroll
    for (int i = 0; i < C::IB; ++i) {
      const int token = m0 + loop.slab_row(i);
      loop.off_b[i] = (uint32_t)((int64_t)head_row(a, token < M ? token : M - 1) * a.ldb * 2) + loop.slab_col();
    }
    const int wm0 = m0 + loop.wt * C::TT * 32;
    loop.active = wm0 < M;
#pragma unroll
    for (int tt = 0; tt < C::TT; ++tt) {
      const int token = wm0 + tt * 32 + loop.n32, at = token < M ? token : M - 1;
      const int64_t far = a.targets[head_row(a, at)] - a.row0 - (r0 + loop.wr * C::RT * 32);
      of[tt].own = far >= 0 && far < 32 * C::RT && (((int)far >> 2) & 1) == loop.kg ? (int)far - 4 * loop.kg : -1;
      if constexpr (PROBS) of[tt].ref = a.again ? head_raised_ref(a, at) : a.ref[at];
    }
    loop.start(0, stages);
  };
  int tile = find(blockIdx.x);
  if (tile >= total) return;
  prepare();
  while (true) {
    f32x16 acc[C::RT][C::TT];
#pragma unroll
    for (int t = 0; t < C::RT; ++t)
#pragma unroll
      for (int tt = 0; tt < C::TT; ++tt)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[t][tt][i] = 0.f;
    loop.template run<C::kTokens <= 64>(acc, 0);
    const int64_t wr0 = (int64_t)rb * C::kRows + loop.wr * C::RT * 32;
    const int wm0 = mb * C::kTokens + loop.wt * C::TT * 32, part = a.part0 + rb * C::WR + loop.wr;
    const bool results = loop.active && wr0 < a.rows;
    tile = find(tile + (int)gridDim.x);
    // the next tile's first slabs are on their way while this one's statistics are formed, which need no LDS
    HeadLane now[C::TT];
#pragma unroll
    for (int tt = 0; tt < C::TT; ++tt) now[tt] = of[tt];
    if (tile < total) {
      lds_wait_barrier<0>();
      prepare();
    }
    if (results) {
      head_statistics<C, PROBS, ENTROPY>(acc, a, now, M, wr0, wm0, part, loop.lane);
      if constexpr (PROBS) store_probs<C>(acc, a, M, wr0, wm0, loop.lane);
    }
    if (tile >= total) return;
  }
}

// ---- sums: [tokens, piece] x [piece, H] ----------------------------------------------------------------------------------
// Unit u of `split` x tiles: which K-part, row block and token block.  The eight XCDs share the K-parts out (several of them to a part
// where there are fewer than eight), and inside a part the tiles, so that an XCD's caches see few slabs.
struct HeadUnit { int part, rb, mb; bool any; };
struct HeadShare { int rows, tokens; };          // log2 of how many ways 2^(3 - log_split) XCDs share the row blocks and the token blocks of a part
__host__ __device__ inline HeadShare head_share(int log_split) {
  const int rows = log_split == 0 ? 2 : log_split == 3 ? 0 : 1;
  return HeadShare{rows, 3 - log_split - rows};
}
__device__ __forceinline__ HeadUnit head_unit(int xcd, int local, int log_split, int row_blocks, int token_blocks) {
  if (log_split >= 3) {
    const int tiles = row_blocks * token_blocks, turn = local / tiles, in = local - turn * tiles, part = turn * 8 + xcd;
    return HeadUnit{part, in % row_blocks, in / row_blocks, part < 1 << log_split};
  }
  const HeadShare h = head_share(log_split);
  const int part = xcd >> (3 - log_split), x = xcd & ((8 >> log_split) - 1);
  const int nr = (row_blocks + (1 << h.rows) - 1) >> h.rows, nt = (token_blocks + (1 << h.tokens) - 1) >> h.tokens;
  const int r = local % nr, rb = (x & ((1 << h.rows) - 1)) * nr + r, mb = (x >> h.rows) * nt + local / nr;
  return HeadUnit{part, rb, mb, local < nr * nt && rb < row_blocks && mb < token_blocks};
}
__host__ __device__ inline int head_units_per_xcd(int log_split, int row_blocks, int token_blocks) {
  if (log_split >= 3) return (row_blocks * token_blocks) << (log_split - 3);
  const HeadShare h = head_share(log_split);
  return ((row_blocks + (1 << h.rows) - 1) >> h.rows) * ((token_blocks + (1 << h.tokens) - 1) >> h.tokens);
}

// log2 of how many parts K is split into: rounds of units over the chip's compute units (two at a time for the smallest tile) at 0.4 us a
// stage and 1.2 per 256 x 256 of it, or what the row slab takes from memory (32 KB per unit at 6 TB/s over the chip: 1.4 us), 2 us to start a unit, and the
// partial sums at 5 TB/s, which every piece reads and writes.  Whole nanoseconds: the host sizes the sums by the same function that the
// kernels evaluate for the rows that have a loss.
struct HeadSplit { int log_split; int64_t ns; };
template <int ROWS, int TOKENS>
__host__ __device__ inline HeadSplit head_split(int row_blocks, int token_blocks, int stages) {
  constexpr int kAtOnce = TOKENS == 64 ? 64 : 32, kStage = TOKENS == 256 ? 400 + 1200 * ROWS / 256 : 1400 * ROWS / 256 * kAtOnce / 32,
                kTile = 2 * ROWS * TOKENS * 4 / 5000;
  HeadSplit best = {0, INT64_MAX};
  for (int l = 0; l <= 6 && (l == 0 || 1 << l <= stages); ++l) {
    const int rounds = (head_units_per_xcd(l, row_blocks, token_blocks) + kAtOnce - 1) / kAtOnce;
    const int64_t ns = rounds * (2000 + (int64_t)((stages + (1 << l) - 1) >> l) * kStage) + ((int64_t)(row_blocks * token_blocks) << l) * kTile;
    if (ns < best.ns) best = HeadSplit{l, ns};
  }
  return best;
}

template <class C>
__global__ __launch_bounds__(C::kThreads, C::kWaves >= 4 ? C::kWaves / 4 : 1) void head_sums_kernel(const HeadArgs a, int row_blocks) {
  extern __shared__ __attribute__((aligned(256))) u32x4 head_lds[];
  HeadLoop<C> loop;
  loop.init(head_lds, threadIdx.x);
  loop.k = a.k;
  const int M = head_tokens(a), token_blocks = (M + C::kTokens - 1) / C::kTokens;
  if (M == 0) return;
  const int stages = (int)((a.k + 63) >> 6);
  const int xcd = blockIdx.x & 7, local = blockIdx.x >> 3;
  const int split = head_split<C::kRows, C::kTokens>(row_blocks, token_blocks, a.piece_stages).log_split;
  const HeadUnit u = head_unit(xcd, local, split, row_blocks, token_blocks);
  if (!u.any) return;
  const int s0 = (int)((int64_t)stages * u.part >> split), s1 = (int)((int64_t)stages * (u.part + 1) >> split);
  const int64_t r0 = (int64_t)u.rb * C::kRows;
  const int m0 = u.mb * C::kTokens;
  loop.base_a = uniform_pointer(a.a + r0 * a.lda);
  loop.base_b = uniform_pointer(a.b + (int64_t)m0 * a.ldb);
#pragma unroll
  for (int i = 0; i < C::IA; ++i) {
    const int64_t r = r0 + loop.slab_row(i) < a.rows ? loop.slab_row(i) : a.rows - 1 - r0;
    loop.off_a[i] = (uint32_t)(r * a.lda * 2) + loop.slab_col();
  }
#pragma unroll
  for (int i = 0; i < C::IB; ++i) {
    const int token = m0 + loop.slab_row(i) < M ? loop.slab_row(i) : M - 1 - m0;
    loop.off_b[i] = (uint32_t)((int64_t)token * a.ldb * 2) + loop.slab_col();
  }
  f32x16 acc[C::RT][C::TT];
#pragma unroll
  for (int t = 0; t < C::RT; ++t)
#pragma unroll
    for (int tt = 0; tt < C::TT; ++tt)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[t][tt][i] = 0.f;
  loop.active = m0 + loop.wt * C::TT * 32 < M;
  if (s1 > s0) {
    loop.start(s0, s1);
    loop.template run<false>(acc, s0);
  }
  if (!loop.active) return;
  // partial sums stay in the registers' order: lane after lane, four rows of a token each
  f32x4* out = reinterpret_cast<f32x4*>(a.acc) + (((int64_t)u.part * token_blocks + u.mb) * row_blocks + u.rb) * (C::kRows * C::kTokens / 4) +
               loop.wave * (C::RT * C::TT * 4 * 64) + loop.lane;
#pragma unroll
  for (int tt = 0; tt < C::TT; ++tt) {
    int token = m0 + (loop.wt * C::TT + tt) * 32 + loop.n32;
    const bool live = token < M;
    token = live ? token : M - 1;
    const float r = a.ref[token], rn = head_raised_ref(a, token), alpha = r == rn ? 1.f : __builtin_amdgcn_exp2f(r - rn);
    if (u.part == 0 && u.rb == 0 && loop.wr == 0 && loop.kg == 0 && live) a.ref_next[token] = rn;
#pragma unroll
    for (int t = 0; t < C::RT; ++t)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f32x4* o = out + (int64_t)((tt * C::RT + t) * 4 + q) * 64;
        f32x4 v = {acc[t][tt][4 * q], acc[t][tt][4 * q + 1], acc[t][tt][4 * q + 2], acc[t][tt][4 * q + 3]};
        if (!a.first) {
          const f32x4 old = *o;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = fmaf(alpha, old[e], v[e]);
        }
        *o = v;
      }
  }
}

// slope = (1/T) [ (1 - p_t) W_t - sums e_scale - large ones' weights W_v ]; a workgroup takes one row tile of a wave's part of a tile, a wave of it one token tile
template <class C>
__global__ __launch_bounds__(64 * C::TT) void head_tile_slope_kernel(const HeadArgs a, const uint16_t* W, int64_t ldw, int row_blocks, float inv_temperature,
                                                                     const float* rest, const float* e_scale, const HeadLargeArgs large, float* slope,
                                                                     int64_t ld_slope) {
  const int M = head_tokens(a);
  const int t = blockIdx.x % C::RT, wave = blockIdx.x / C::RT % C::kWaves, tile = blockIdx.x / (C::RT * C::kWaves), rb = tile % row_blocks, mb = tile / row_blocks;
  const int wr = wave % C::WR, wt = wave / C::WR, lane = threadIdx.x & 63, tt = threadIdx.x >> 6;
  const int token = mb * C::kTokens + (wt * C::TT + tt) * 32 + (lane & 31);
  const int64_t h0 = (int64_t)rb * C::kRows + (wr * C::RT + t) * 32 + 4 * (lane >> 5);
  if (token >= M || h0 >= a.rows) return;
  const int row = head_row(a, token);
  if (!a.index && (a.targets[row] < 0 || a.targets[row] >= a.V)) return;
  const float r = rest[row] * inv_temperature, es = e_scale[row] * inv_temperature;
  const uint16_t* w = W + a.targets[row] * ldw;
  float* out = slope + (int64_t)row * ld_slope;
  const int token_blocks = (M + C::kTokens - 1) / C::kTokens, split = 1 << head_split<C::kRows, C::kTokens>(row_blocks, token_blocks, a.piece_stages).log_split;
  const f32x4* in = reinterpret_cast<const f32x4*>(a.acc) + (int64_t)tile * (C::kRows * C::kTokens / 4) + wave * (C::RT * C::TT * 4 * 64) + (tt * C::RT + t) * 4 * 64 + lane;
  const int64_t slab = (int64_t)token_blocks * row_blocks * (C::kRows * C::kTokens / 4);
  f32x4 s[4] = {};
#pragma unroll 4
  for (int z = 0; z < split; ++z)
#pragma unroll
    for (int q = 0; q < 4; ++q) s[q] += in[z * slab + q * 64];
  f32x4 back[4] = {};                            // what the large probabilities' roundings cut off
  for (int i = 0, n = large.count[token]; i < n; ++i) {
    const HeadLarge l = large.slot[(int64_t)token * kLargeSlots + i];
    const uint16_t* wl = W + l.v * ldw + h0;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (h0 + 8 * q < a.rows) {
        const u32x2 wv = *reinterpret_cast<const u32x2*>(wl + 8 * q);
        back[q] += l.off * f32x4{bf16_bits_to_f32(wv[0] & 0xffffu), __uint_as_float(wv[0] & 0xffff0000u), bf16_bits_to_f32(wv[1] & 0xffffu),
                                 __uint_as_float(wv[1] & 0xffff0000u)};
      }
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int64_t h = h0 + 8 * q;
    if (h >= a.rows) break;                      // H is a multiple of 8: four rows are inside or beyond
    const u32x2 wv = *reinterpret_cast<const u32x2*>(w + h);
    f32x4 o;
    o[0] = bf16_bits_to_f32(wv[0] & 0xffffu) * r - s[q][0] * es - back[q][0] * inv_temperature;
    o[1] = __uint_as_float(wv[0] & 0xffff0000u) * r - s[q][1] * es - back[q][1] * inv_temperature;
    o[2] = bf16_bits_to_f32(wv[1] & 0xffffu) * r - s[q][2] * es - back[q][2] * inv_temperature;
    o[3] = __uint_as_float(wv[1] & 0xffff0000u) * r - s[q][3] * es - back[q][3] * inv_temperature;
    *reinterpret_cast<f32x4*>(out + h) = o;
  }
}

// ---- host ----------------------------------------------------------------------------------------------------------------
// Up to 64 tokens the logits' products are in chains of 256 inputs: a row whose token is nearly certain has a log-probability that is off, relative
// to itself, by what its logit is off, and with few rows no other hides it (one chain over 3584 inputs: 3e-6 of a log-probability near 0,
// in chains 1e-6; the kernels stream the weights either way).
using Head32 = HeadCfg<2, 1, 2, 1, 4, 4>;        // 128 rows x 32 tokens, two workgroups of two waves per compute unit
using Head64 = HeadCfg<2, 2, 2, 1, 3, 3>;        // 128 rows x 64 tokens
using Head128 = HeadCfg<2, 2, 4, 2, 3, 2>;       // 256 rows x 128 tokens
using Head256 = HeadCfg<4, 2, 2, 4, 3, 2>;       // 256 rows x 256 tokens
using HeadHalf = HeadCfg<2, 2, 2, 4, 3, 2>;      // 128 rows x 256 tokens
using Head320 = HeadCfg<5, 2, 2, 4, 2, 2>;       // 320 rows x 256 tokens (six registers in scratch): sums whose tiles of 256 would leave a round of workgroups half empty

// The smallest tile that holds all tokens, so that few tokens stream the weights through small workgroups; beyond 128 tokens 256 rows, or 128
// where those would leave half of the compute units without a tile (200 rows of 32001 x 1024: 35 -> 25 us).
HeadGemmPlan plan_head_gemm(int64_t M, int64_t V, bool gradient) {
  if (M <= 32 && !gradient) return HeadGemmPlan{Head32::kTokens, Head32::kRows, 32 * Head32::RT};
  if (M <= 64) return HeadGemmPlan{Head64::kTokens, Head64::kRows, 32 * Head64::RT};
  if (M <= 128) return HeadGemmPlan{Head128::kTokens, Head128::kRows, 32 * Head128::RT};
  if (ceil_div(V, Head256::kRows) * ceil_div(M, Head256::kTokens) <= 128) return HeadGemmPlan{HeadHalf::kTokens, HeadHalf::kRows, 32 * HeadHalf::RT};
  return HeadGemmPlan{Head256::kTokens, Head256::kRows, 32 * Head256::RT};
}

template <class K>
static int allow_lds(K kernel, int bytes) {
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != hipSuccess) { set_last_hip_error((int)e); return QERL_ERR_LAUNCH; }
  return QERL_OK;
}

template <class C, bool PROBS, bool ENTROPY>
static int launch_products(const HeadArgs& a, hipStream_t st) {
  if (const int e = allow_lds(head_gemm_kernel<C, PROBS, ENTROPY>, C::kLds)) return e;
  const int row_blocks = (int)ceil_div(a.rows, C::kRows), per_xcd = (int)ceil_div(row_blocks, 8);
  int64_t grid = 8 * (int64_t)per_xcd * ceil_div(a.M, C::kTokens);
  // as many workgroups as fit at once: each goes on to its next tile while it finishes the last
  const int64_t at_once = 256 * (160 * 1024 / C::kLds);
  if (grid > at_once) grid = at_once;
  head_gemm_kernel<C, PROBS, ENTROPY><<<dim3((unsigned)grid), dim3(C::kThreads), C::kLds, st>>>(a, row_blocks, per_xcd);
  return launch_status();
}
template <class C>
static int launch_sums(const HeadArgs& a, hipStream_t st) {
  if (const int e = allow_lds(head_sums_kernel<C>, C::kLds)) return e;
  const int row_blocks = (int)ceil_div(a.rows, C::kRows), token_blocks = (int)ceil_div(a.M, C::kTokens);
  int units = 0;                                 // of an XCD, at most, whatever number of rows has a loss
  for (int tb = a.count ? 1 : token_blocks; tb <= token_blocks; ++tb) {
    const int n = head_units_per_xcd(head_split<C::kRows, C::kTokens>(row_blocks, tb, a.piece_stages).log_split, row_blocks, tb);
    units = n > units ? n : units;
  }
  head_sums_kernel<C><<<dim3((unsigned)(8 * units)), dim3(C::kThreads), C::kLds, st>>>(a, row_blocks);
  return launch_status();
}
template <class C, bool PROBS>
static int launch_mode(bool entropy, const HeadArgs& a, hipStream_t st) {
  return entropy ? launch_products<C, PROBS, true>(a, st) : launch_products<C, PROBS, false>(a, st);
}
int launch_head_logits(const HeadGemmPlan& p, bool entropy, const HeadArgs& a, hipStream_t st) {
  switch (p.tokens) {
    case 32: return launch_mode<Head32, false>(entropy, a, st);
    case 64: return launch_mode<Head64, false>(entropy, a, st);
    case 128: return launch_mode<Head128, false>(entropy, a, st);
    default: return p.rows == 128 ? launch_mode<HeadHalf, false>(entropy, a, st) : launch_mode<Head256, false>(entropy, a, st);
  }
}
int launch_head_probs(const HeadGemmPlan& p, bool entropy, const HeadArgs& a, hipStream_t st) {
  switch (p.tokens) {
    case 64: return launch_mode<Head64, true>(entropy, a, st);
    case 128: return launch_mode<Head128, true>(entropy, a, st);
    default: return p.rows == 128 ? launch_mode<HeadHalf, true>(entropy, a, st) : launch_mode<Head256, true>(entropy, a, st);
  }
}

// The tile that costs least, and what its partial sums take for up to M rows with a loss
template <class C>
static void consider_sums(HeadSumsPlan& q, int64_t& best, int64_t M, int64_t H, int64_t piece) {
  const int token_blocks = (int)ceil_div(M, C::kTokens), row_blocks = (int)ceil_div(H, C::kRows), stages = (int)(piece / 64);
  const int64_t ns = head_split<C::kRows, C::kTokens>(row_blocks, token_blocks, stages).ns;
  if (ns >= best) return;
  best = ns;
  q = HeadSumsPlan{C::kRows, 0};
  for (int tb = 1; tb <= token_blocks; ++tb) {
    const size_t bytes = ((size_t)(row_blocks * tb) << head_split<C::kRows, C::kTokens>(row_blocks, tb, stages).log_split) * 4 * C::kRows * C::kTokens;
    q.bytes = bytes > q.bytes ? bytes : q.bytes;
  }
}
HeadSumsPlan plan_head_sums(const HeadGemmPlan& p, int64_t M, int64_t H, int64_t piece) {
  HeadSumsPlan q = {};
  int64_t best = INT64_MAX;
  if (p.tokens == 64) consider_sums<Head64>(q, best, M, H, piece);
  else if (p.tokens == 128) consider_sums<Head128>(q, best, M, H, piece);
  else {
    consider_sums<HeadHalf>(q, best, M, H, piece);
    consider_sums<Head256>(q, best, M, H, piece);
    consider_sums<Head320>(q, best, M, H, piece);
  }
  return q;
}

template <class C>
static int launch_slope(const HeadArgs& sums, const HeadArgs& head, float inv_temperature, const float* rest, const float* e_scale, const HeadLargeArgs& large,
                        float* slope, int64_t ld_slope, hipStream_t st) {
  const int row_blocks = (int)ceil_div(sums.rows, C::kRows);
  head_tile_slope_kernel<C><<<dim3((unsigned)(row_blocks * ceil_div(sums.M, C::kTokens) * C::kWaves * C::RT)), dim3(64 * C::TT), 0, st>>>(
      sums, head.a, head.lda, row_blocks, inv_temperature, rest, e_scale, large, slope, ld_slope);
  return launch_status();
}
int launch_head_sums(const HeadGemmPlan& p, const HeadSumsPlan& q, const HeadArgs& a, hipStream_t st) {
  return p.tokens == 64    ? launch_sums<Head64>(a, st)
         : p.tokens == 128 ? launch_sums<Head128>(a, st)
         : q.rows == 128   ? launch_sums<HeadHalf>(a, st)
         : q.rows == 320   ? launch_sums<Head320>(a, st)
                           : launch_sums<Head256>(a, st);
}
int launch_head_slope(const HeadGemmPlan& p, const HeadSumsPlan& q, const HeadArgs& sums, const HeadArgs& head, float inv_temperature, const float* rest,
                      const float* e_scale, const HeadLargeArgs& large, float* slope, int64_t ld_slope, hipStream_t st) {
  return p.tokens == 64    ? launch_slope<Head64>(sums, head, inv_temperature, rest, e_scale, large, slope, ld_slope, st)
         : p.tokens == 128 ? launch_slope<Head128>(sums, head, inv_temperature, rest, e_scale, large, slope, ld_slope, st)
         : q.rows == 128   ? launch_slope<HeadHalf>(sums, head, inv_temperature, rest, e_scale, large, slope, ld_slope, st)
         : q.rows == 320   ? launch_slope<Head320>(sums, head, inv_temperature, rest, e_scale, large, slope, ld_slope, st)
                           : launch_slope<Head256>(sums, head, inv_temperature, rest, e_scale, large, slope, ld_slope, st);
}

}  // namespace qerl
