// lm_head_logprob*: log-probability of one token per row under the language-model head, entropy, and the gradient with respect to
// the hidden states, without keeping the logits.
//
// With z_v = x . W_v / T, t the row's token, o = sum_{v != t} e^(z_v - z_t):
//   logprob = -ln(1 + o)                       exact near 0, where z_t - lse would have cancelled
//   lse     = z_t + ln(1 + o)
//   entropy = lse - sum_v p_v z_v
//   d logprob / dx = (1/T) [ (1 - p_t) W_t - sum_{v != t} p_v W_v ],   1 - p_t = o / (1 + o)
// Everything runs on s = z log2(e) with exp2; logits come from bf16 matrix instructions into fp32, all sums are fp32.
#include <math.h>
#include "common.hpp"
#include "lm_head.hpp"

namespace qerl {

constexpr float kLn2 = 0.693147180559945309f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// (m, s, w) <- both, sums relative to the larger m; an m of -inf goes with sums of 0 (or NaN, which has to stay)
__device__ __forceinline__ void merge_sums(float& m, float& s, float& w, float m2, float s2, float w2) {
  const float top = fmaxf(m, m2);
  const float d1 = m == kNegInf ? 0.f : m - top, d2 = m2 == kNegInf ? 0.f : m2 - top;
  const float e1 = exp2_fast(d1), e2 = exp2_fast(d2);
  w = (w + d1 * s) * e1 + (w2 + d2 * s2) * e2;
  s = s * e1 + s2 * e2;
  m = top;
}

// Rows with a loss, in order: index[0 .. *count), and each row's place among them (-1: none)
constexpr int kCompactThreads = 1024;
__global__ __launch_bounds__(kCompactThreads) void head_compact_kernel(const int64_t* targets, int64_t V, int M, int* index, int* place, int* count) {
  __shared__ int waves[kCompactThreads / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int before = 0;
  for (int m0 = 0; m0 < M; m0 += kCompactThreads) {
    const int m = m0 + threadIdx.x;
    const bool in = m < M && targets[m] >= 0 && targets[m] < V;
    const uint64_t votes = __ballot(in);
    if (lane == 0) waves[wave] = __popcll(votes);
    __syncthreads();
    int at = before, all = 0;
    for (int w = 0; w < kCompactThreads / 64; ++w) {
      if (w < wave) at += waves[w];
      all += waves[w];
    }
    at += __popcll(votes & (((uint64_t)1 << lane) - 1));
    if (in) index[at] = m;
    if (m < M) place[m] = in ? at : -1;
    before += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) *count = before;
}

// logit of a vocabulary row, by a wave: x . w
__device__ __forceinline__ float wave_logit(const uint16_t* x, const uint16_t* w, int64_t H, int lane) {
  float sum = 0.f;
  for (int64_t k = lane * 8; k < H; k += 512) {
    const u32x4 xv = *reinterpret_cast<const u32x4*>(x + k), wv = *reinterpret_cast<const u32x4*>(w + k);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      sum += bf16_bits_to_f32(xv[j] & 0xffffu) * bf16_bits_to_f32(wv[j] & 0xffffu);
      sum += __uint_as_float(xv[j] & 0xffff0000u) * __uint_as_float(wv[j] & 0xffff0000u);
    }
  }
  return wave_sum(sum);
}

// Reference of the first piece: the logit of the token's own row (a lower bound of the largest).  A row without a loss, where such are not
// left out, gets +inf, which makes its probabilities 0.  Clears the pieces' flags and what
// raises references.
__global__ __launch_bounds__(256) void head_first_ref_kernel(const HeadArgs a, float* ref, uint32_t* clear, int64_t n_clear) {
  for (int64_t i = blockIdx.x * 256 + threadIdx.x; i < n_clear; i += gridDim.x * 256) clear[i] = 0u;
  const int token = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (token >= head_tokens(a)) return;
  const int64_t row = head_row(a, token), target = a.targets[row];
  if (target < 0 || target >= a.V) {
    if (lane == 0) ref[token] = kInf;
    return;
  }
  const float sum = wave_logit(a.b + row * a.ldb, a.a + target * a.lda, a.k, lane);
  if (lane == 0) ref[token] = sum * a.scale;
}

// Large probabilities.  The second product takes probabilities as bf16.  Over a sum of many their roundings, half a step each at most and
// independent, cancel to a small part of it; where few tokens hold what the row's own token leaves, nothing cancels, and the slope would be off
// by up to 2^-8 of itself, as much as dx by its own rounding.  So all that hold kLargeShare of what all others hold together, 32 at most, are looked
// up again where the parts' largest logits say that there are some: the logit formed once more in fp32, and what the rounding cut off kept for the
// slope.  The rest is off by 2^-8 / sqrt(32) of the slope at most, in the root mean square.  Measured on rows whose mass one or five other tokens
// share, slope against 64 bits: 9e-4 of itself without, 2e-6 and 2e-5 with; time for 4096 rows of 152064 x 5120 9.95 ms without, 10.00 with where no
// probability is large, 10.10 and 10.23 with one and five per row; 200 rows of 32001 x 1024 74 us, 76, 80 and 83.
// Of a piece, by a workgroup for its token: those of at least `least` (relative to ref), 33 at most as it is a share of their sum; lane i of the first
// wave holds slot i in `mine`.  The first wave lists them, all four form their logits (five of them, 64 rows of 32000 x 2048: by one wave 98 us, 95),
// and the first takes them up: where the slots do not suffice (earlier pieces' sums were smaller) the largest stay.
constexpr int kLargeWords = (int)(((int64_t)1 << 22) / 64 / 64);   // a bit for each part of the largest vocabulary
struct LargeShared { uint64_t marks[kLargeWords]; int64_t at[kLargeSlots]; float kept[kLargeSlots], s[kLargeSlots]; int n; };
__device__ __forceinline__ void collect_large(const HeadArgs& a, const HeadLargeArgs& g, int token, int64_t row, float ref, float least, LargeShared& sh,
                                              HeadLarge& mine, int& count) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const HeadPart* part = a.part + (int64_t)token * a.part_ld + a.part0;
  for (int b0 = 0; b0 < g.parts; b0 += 256) {
    const int b = b0 + threadIdx.x;
    const uint64_t votes = __ballot(b < g.parts && exp2_fast(part[b < g.parts ? b : 0].top - ref) >= least);
    if (lane == 0) sh.marks[b0 / 64 + wave] = votes;
  }
  __syncthreads();
  if (wave == 0) {
    const uint16_t* p = a.p + (int64_t)token * a.ldp;
    const int words = (g.parts + 63) / 64;
    int n = 0;
    for (int w0 = 0; w0 < words; w0 += 64) {
      const uint64_t word = w0 + lane < words ? sh.marks[w0 + lane] : 0;
      for (uint64_t some = __ballot(word != 0); some; some &= some - 1) {
        const int from = __ffsll((unsigned long long)some) - 1;
        for (uint64_t bits = __shfl((unsigned long long)word, from, 64); bits; bits &= bits - 1) {
          const int64_t r0 = ((int64_t)(w0 + from) * 64 + __ffsll((unsigned long long)bits) - 1) * g.part_rows;
          for (int64_t r = r0; r < r0 + g.part_rows; r += 64) {
            const float value = r + lane < a.rows ? bf16_bits_to_f32(p[r + lane]) : 0.f;
            const uint64_t hits = __ballot(value >= least);
            const int to = n + __popcll(hits & (((uint64_t)1 << lane) - 1));
            if (value >= least && to < kLargeSlots) { sh.at[to] = r + lane; sh.kept[to] = value; }
            n += __popcll(hits);
          }
        }
      }
    }
    if (lane == 0) sh.n = n < kLargeSlots ? n : kLargeSlots;
  }
  __syncthreads();
  const int n = sh.n;
  for (int i = wave; i < n; i += 4) {
    const float s = wave_logit(a.b + row * a.ldb, a.a + sh.at[i] * a.lda, a.k, lane) * a.scale;
    if (lane == 0) sh.s[i] = s;
  }
  __syncthreads();
  if (wave != 0) return;
  for (int i = 0; i < n; ++i) {
    const float s = sh.s[i];
    int slot = count;
    if (count == kLargeSlots) {
      float lowest = mine.s;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) lowest = fminf(lowest, __shfl_xor(lowest, o, 64));
      slot = s > lowest ? __ffsll((unsigned long long)__ballot(mine.s == lowest)) - 1 : kLargeSlots;
    } else {
      ++count;
    }
    if (lane == slot) mine = HeadLarge{(int)(a.row0 + sh.at[i]), ref, exp2_fast(s - ref) - sh.kept[i], s};
  }
}
// least: the share of all that the others hold, a little less, so that roundings exclude nothing; NaN, which nothing reaches, where that is not finite
__device__ __forceinline__ float large_from(float others) {
  return others > 0.f && others < kInf ? others * (kLargeShare * (1.f - 0x1p-6f)) : __uint_as_float(0x7fc00000u);
}

// Large probabilities of a piece that is not the last one (whose are looked up with the row results)
__global__ __launch_bounds__(256) void head_large_kernel(const HeadArgs a, const HeadLargeArgs g) {
  __shared__ LargeShared large;
  __shared__ float sm[4];
  const int token = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (token >= head_tokens(a)) return;
  const int64_t row = head_row(a, token);
  if (a.targets[row] < 0 || a.targets[row] >= a.V) return;
  const float ref = head_raised_ref(a, token);
  const HeadPart* part = a.part + (int64_t)token * a.part_ld + a.part0;
  const float before = g.first ? 0.f : g.running[2 * token] * exp2_fast(g.running[2 * token + 1] - ref);
  float sum = 0.f;
  for (int b = threadIdx.x; b < g.parts; b += 256) sum += part[b].sum;
  sum = wave_sum(sum);
  if (lane == 0) sm[wave] = sum;
  __syncthreads();                               // (also: the running sum is read)
  sum = before + ((sm[0] + sm[1]) + (sm[2] + sm[3]));
  HeadLarge* slot = g.slot + (int64_t)token * kLargeSlots;
  int count = g.first ? 0 : g.count[token];
  HeadLarge mine = lane < count ? slot[lane] : HeadLarge{0, 0.f, 0.f, kNegInf};
  collect_large(a, g, token, row, ref, large_from(sum), large, mine, count);
  if (wave != 0) return;
  if (lane < count) slot[lane] = mine;
  if (lane == 0) {
    g.count[token] = count;
    g.running[2 * token] = sum;
    g.running[2 * token + 1] = ref;
  }
}

// Row results from all parts; for the gradient also 1 - p_t, what turns the sums E into sum p W, the weights of the large probabilities' roundings, and
// the slopes of rows without a loss
__global__ __launch_bounds__(256) void head_finish_kernel(const HeadArgs a, int parts, const int* place, const float* ref_last, float* logprob, float* lse,
                                                          float* entropy, float* rest, float* e_scale, const HeadLargeArgs g, float* slope, int64_t ld_slope,
                                                          int64_t H) {
  __shared__ float sm[3][4];
  __shared__ LargeShared large;
  const int row = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t target = a.targets[row];
  if (target < 0 || target >= a.V) {
    const float v = target < 0 ? 0.f : __uint_as_float(0x7fc00000u);
    if (threadIdx.x == 0) {
      logprob[row] = v;
      if (lse) lse[row] = v;
      if (entropy) entropy[row] = v;
    }
    if (slope)
      for (int64_t h = threadIdx.x; h < H; h += 256) slope[(int64_t)row * ld_slope + h] = v;
    return;
  }
  const int token = place ? place[row] : row;
  float m = kNegInf, s = 0.f, w = 0.f;
  const HeadPart* part = a.part + (int64_t)token * a.part_ld;
  int b = threadIdx.x;
  for (; b + 3 * 256 < parts; b += 4 * 256) {    // four on their way at a time
    HeadPart p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = part[b + 256 * i];
#pragma unroll
    for (int i = 0; i < 4; ++i) merge_sums(m, s, w, p[i].ref, p[i].sum, p[i].weighted);
  }
  for (; b < parts; b += 256) {
    const HeadPart p = part[b];
    merge_sums(m, s, w, p.ref, p.sum, p.weighted);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const float m2 = __shfl_xor(m, o, 64), s2 = __shfl_xor(s, o, 64), w2 = __shfl_xor(w, o, 64);
    merge_sums(m, s, w, m2, s2, w2);
  }
  if (lane == 0) { sm[0][wave] = m; sm[1][wave] = s; sm[2][wave] = w; }
  __syncthreads();
  if (!rest && threadIdx.x != 0) return;
  m = sm[0][0]; s = sm[1][0]; w = sm[2][0];
  for (int i = 1; i < 4; ++i) merge_sums(m, s, w, sm[0][i], sm[1][i], sm[2][i]);
  const float st = a.target_logit[token];
  float base, total, logp, l;
  if (!(st < m - 30.f)) {
    base = st;                                   // relative to the token itself: nothing cancels
    const float d = m == kNegInf ? 0.f : m - st, f = exp2_fast(d);
    w = (w + d * s) * f;
    s *= f;
    total = 1.f + s;
    l = log1pf(s);
    logp = -l;
  } else {
    base = m;
    const float et = exp2_fast(st - m);
    total = s + et;
    w += et * (st - m);
    l = logf(total);
    logp = kLn2 * (st - m) - l;
  }
  if (threadIdx.x == 0) {
    logprob[row] = logp;
    if (lse) lse[row] = kLn2 * base + l;
    if (entropy) entropy[row] = l - kLn2 * w / total;
    if (rest) {
      rest[row] = s / total;
      e_scale[row] = exp2_fast(ref_last[token] - base) / total;
    }
  }
  if (!rest) return;
  const float ref = ref_last[token];
  HeadLarge* slot = g.slot + (int64_t)token * kLargeSlots;
  int count = g.first ? 0 : g.count[token];
  HeadLarge mine = lane < count ? slot[lane] : HeadLarge{0, 0.f, 0.f, kNegInf};
  collect_large(a, g, token, row, ref, large_from(s * exp2_fast(base - ref)), large, mine, count);
  if (wave != 0) return;
  const bool stays = lane < count && exp2_fast(mine.s - base) >= large_from(s);   // what earlier pieces found may be small now
  const uint64_t all = __ballot(stays);
  if (stays) slot[__popcll(all & (((uint64_t)1 << lane) - 1))] = HeadLarge{mine.v, 0.f, mine.off * exp2_fast(mine.ref - base) / total, 0.f};
  if (lane == 0) g.count[token] = __popcll(all);
}

// dx = bf16(g slope)
__global__ __launch_bounds__(256) void head_backward_kernel(const float* g, const float* slope, int64_t ld_slope, int M, int64_t H, uint16_t* dx, int64_t lddx) {
  const int token = blockIdx.y;
  const int64_t h = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (h >= H) return;
  const float gm = g[token];
  const f32x4 a = *reinterpret_cast<const f32x4*>(slope + token * ld_slope + h), b = *reinterpret_cast<const f32x4*>(slope + token * ld_slope + h + 4);
  *reinterpret_cast<u32x4*>(dx + token * lddx + h) =
      u32x4{pack_bf16x2(gm * a[0], gm * a[1]), pack_bf16x2(gm * a[2], gm * a[3]), pack_bf16x2(gm * b[0], gm * b[1]), pack_bf16x2(gm * b[2], gm * b[3])};
}

// W [V, ldw] -> Wt [H, ldt], ldt = V rounded up to 64, zeros behind the vocabulary.  Tiles of 64 x 64, 16 bytes a lane on both sides; the
// swizzle of the 16-byte columns keeps the column reads off each other's banks.
__global__ __launch_bounds__(256) void head_transpose_kernel(const uint16_t* w, int64_t V, int64_t H, int64_t ldw, uint16_t* out, int64_t ldt) {
  __shared__ __attribute__((aligned(16))) uint16_t tile[64 * 64];
  const int64_t v0 = (int64_t)blockIdx.x * 64, h0 = (int64_t)blockIdx.y * 64;
  const int r = threadIdx.x >> 3, c = threadIdx.x & 7;
#pragma unroll
  for (int i = 0; i < 64; i += 32) {
    const int row = r + i;
    u32x4 v = {0u, 0u, 0u, 0u};
    if (v0 + row < V && h0 + 8 * c < H) v = *reinterpret_cast<const u32x4*>(w + (v0 + row) * ldw + h0 + 8 * c);   // H is a multiple of 8
    *reinterpret_cast<u32x4*>(tile + row * 64 + 8 * (c ^ (row >> 3))) = v;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 64; i += 32) {
    const int h = r + i;                          // a row of the output, its vocabulary rows 8 c .. 8 c + 7
    if (h0 + h >= H) continue;
    uint32_t o[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      o[j] = tile[(8 * c + 2 * j) * 64 + 8 * ((h >> 3) ^ c) + (h & 7)] | (uint32_t)tile[(8 * c + 2 * j + 1) * 64 + 8 * ((h >> 3) ^ c) + (h & 7)] << 16;
    *reinterpret_cast<u32x4*>(out + (h0 + h) * ldt + v0 + 8 * c) = u32x4{o[0], o[1], o[2], o[3]};
  }
}

// ---- host ----------------------------------------------------------------------------------------------------------------
constexpr int64_t kMaxLd = 1 << 18, kMaxVocab = 1 << 22;  // (exclusive, inclusive) offsets inside the GEMM's operands have 32 bits
constexpr int64_t kTokenBlock = 8192;                     // tokens that are taken through the whole vocabulary together
constexpr int64_t kPieceBytes = (int64_t)192 << 20;       // probabilities of a piece: they stay in the last-level cache until they are used

struct HeadPlan {
  HeadGemmPlan gemm;
  HeadSumsPlan sums;
  bool compact;                                           // rows without a loss are left out of the products
  int64_t tokens, parts, pieces, piece, flags;            // tokens at a time; parts of a row; pieces and their rows, flags of a piece
  size_t part, target, index, ref, clear, rest, large, p, acc, bytes;  // offsets; clear: of each piece the flags, then what raises references
};

// Rows of a piece in blocks of `unit`: at most `most`, as few rounds of workgroups as possible over the vocabulary, then as few pieces
static int64_t piece_blocks(int64_t blocks, int64_t most, int64_t token_blocks) {
  most = most < 1 ? 1 : most;
  if (most >= blocks) return blocks;
  int64_t best = most, best_rounds = INT64_MAX;
  for (int64_t n = most; n >= 1 && n > most / 2; --n) {
    const int64_t last = blocks % n, rounds = blocks / n * ceil_div(n * token_blocks, 256) + ceil_div(last * token_blocks, 256);
    if (rounds < best_rounds) { best = n; best_rounds = rounds; }
  }
  return best;
}

static HeadPlan plan_head(int64_t M, int64_t V, int64_t H, bool gradient) {
  HeadPlan q = {};
  q.tokens = M < kTokenBlock ? M : kTokenBlock;
  q.gemm = plan_head_gemm(q.tokens, V, gradient);
  q.compact = q.tokens > 128;                             // fewer are one token block whatever they are
  q.parts = ceil_div(V, q.gemm.part_rows);
  auto up = [](size_t b) { return (b + 255) & ~(size_t)255; };
  size_t at = 0;
  q.part = at; at += up((size_t)(q.tokens * q.parts) * sizeof(HeadPart));
  q.target = at; at += up((size_t)q.tokens * 4);
  q.index = at; at += q.compact ? up((size_t)(2 * q.tokens + 1) * 4) : 0;
  if (gradient) {
    q.flags = ceil_div(q.tokens, q.gemm.tokens);
    q.piece = piece_blocks(ceil_div(V, q.gemm.rows), kPieceBytes / (2 * q.flags * q.gemm.tokens * q.gemm.rows), q.flags) * q.gemm.rows;
    q.pieces = ceil_div(V, q.piece);
    q.sums = plan_head_sums(q.gemm, q.tokens, H, q.piece);
    q.ref = at; at += up((size_t)(q.tokens * (q.pieces + 1)) * 4);
    q.clear = at; at += up((size_t)((q.flags + q.tokens) * q.pieces) * 4);
    q.rest = at; at += up((size_t)(2 * q.tokens) * 4);
    q.large = at; at += up((size_t)q.tokens * (kLargeSlots * sizeof(HeadLarge) + 3 * 4));
    q.p = at; at += up((size_t)(q.tokens * q.piece) * 2);
    q.acc = at; at += up(q.sums.bytes);
  }
  q.bytes = at;
  return q;
}

struct HeadCall {
  const uint16_t* x; int64_t M, H, ldx;
  const uint16_t* W; int64_t V, ldw;
  const uint16_t* Wt;
  const int64_t* targets; float inv_temperature;
  float* logprob; float* lse; float* entropy; float* slope; int64_t ld_slope;
  uint8_t* ws; size_t ws_bytes; hipStream_t st;
};

static int run_tokens(const HeadCall& c, const HeadPlan& q, int64_t m0, int64_t M) {
  const bool entropies = c.entropy != nullptr;
  HeadArgs a = {};
  a.a = c.W; a.lda = c.ldw; a.rows = c.V; a.b = c.x + m0 * c.ldx; a.ldb = c.ldx; a.k = c.H; a.M = (int)M;
  a.targets = c.targets + m0; a.V = c.V; a.scale = c.inv_temperature * 1.44269504088896341f;
  a.part = reinterpret_cast<HeadPart*>(c.ws + q.part); a.part_ld = q.parts; a.target_logit = reinterpret_cast<float*>(c.ws + q.target);
  int* place = nullptr;
  if (q.compact) {
    int* index = reinterpret_cast<int*>(c.ws + q.index);
    place = index + q.tokens;
    head_compact_kernel<<<dim3(1), dim3(kCompactThreads), 0, c.st>>>(a.targets, c.V, (int)M, index, place, place + q.tokens);
    a.index = index; a.count = place + q.tokens;
  }
  float* logprob = c.logprob + m0;
  float* lse = c.lse ? c.lse + m0 : nullptr;
  float* entropy = c.entropy ? c.entropy + m0 : nullptr;
  if (!c.slope) {
    if (const int e = launch_head_logits(q.gemm, entropies, a, c.st)) return e;
    head_finish_kernel<<<dim3((unsigned)M), dim3(256), 0, c.st>>>(a, (int)q.parts, place, nullptr, logprob, lse, entropy, nullptr, nullptr, HeadLargeArgs{},
                                                                  nullptr, 0, 0);
    return launch_status();
  }
  float* ref = reinterpret_cast<float*>(c.ws + q.ref);
  uint32_t* clear = reinterpret_cast<uint32_t*>(c.ws + q.clear);
  float* rest = reinterpret_cast<float*>(c.ws + q.rest);
  float* e_scale = rest + q.tokens;
  float* slope = c.slope + m0 * c.ld_slope;
  HeadLargeArgs large = {};
  large.slot = reinterpret_cast<HeadLarge*>(c.ws + q.large);
  large.running = reinterpret_cast<float*>(large.slot + q.tokens * kLargeSlots);
  large.count = reinterpret_cast<int*>(large.running + 2 * q.tokens);
  large.part_rows = q.gemm.part_rows;
  head_first_ref_kernel<<<dim3((unsigned)ceil_div(M, 4)), dim3(256), 0, c.st>>>(a, ref, clear, (q.flags + q.tokens) * q.pieces);
  HeadArgs e = a;
  e.lda = ceil_div(c.V, 64) * 64; e.rows = c.H; e.b = reinterpret_cast<uint16_t*>(c.ws + q.p); e.ldb = q.piece;
  e.acc = reinterpret_cast<float*>(c.ws + q.acc); e.piece_stages = (int)(q.piece / 64);
  for (int64_t i = 0; i < q.pieces; ++i) {
    const int64_t row0 = i * q.piece, rows = c.V - row0 < q.piece ? c.V - row0 : q.piece;
    a.a = c.W + row0 * c.ldw; a.rows = rows; a.row0 = row0; a.part0 = (int)(row0 / q.gemm.part_rows);
    a.p = reinterpret_cast<uint16_t*>(c.ws + q.p); a.ldp = q.piece;
    a.ref = ref + i * q.tokens; a.ref_next = ref + (i + 1) * q.tokens; a.again = 0;
    a.flag = reinterpret_cast<int*>(clear + i * (q.flags + q.tokens)); a.raise = clear + i * (q.flags + q.tokens) + q.flags;
    if (const int s = launch_head_probs(q.gemm, entropies, a, c.st)) return s;
    a.again = 1;
    if (const int s = launch_head_probs(q.gemm, entropies, a, c.st)) return s;
    large.parts = (int)ceil_div(rows, q.gemm.part_rows); large.first = i == 0;
    if (i + 1 < q.pieces) head_large_kernel<<<dim3((unsigned)M), dim3(256), 0, c.st>>>(a, large);
    e.a = c.Wt + row0; e.k = ceil_div(rows, 64) * 64; e.ref = a.ref; e.raise = a.raise; e.ref_next = a.ref_next; e.first = i == 0;
    if (const int s = launch_head_sums(q.gemm, q.sums, e, c.st)) return s;
  }
  head_finish_kernel<<<dim3((unsigned)M), dim3(256), 0, c.st>>>(a, (int)q.parts, place, ref + q.pieces * q.tokens, logprob, lse, entropy, rest, e_scale, large, slope,
                                                                c.ld_slope, c.H);
  a.a = c.W;
  return launch_head_slope(q.gemm, q.sums, e, a, c.inv_temperature, rest, e_scale, large, slope, c.ld_slope, c.st);
}

static int run_head(const HeadCall& c, bool gradient) {
  if (c.M < 0 || c.V < 1 || c.V > kMaxVocab || c.H < 8 || c.H % 8 != 0 || c.M > 0x7fffffff || c.ldx < c.H || c.ldx >= kMaxLd || c.ldw < c.H ||
      c.ldw >= kMaxLd || (gradient && c.ld_slope < c.H))
    return QERL_ERR_SHAPE;
  if (!(c.inv_temperature > 0.f) || !isfinite(c.inv_temperature * 1.44269504088896341f)) return QERL_ERR_SHAPE;
  if (c.M == 0) return QERL_OK;
  if (!c.x || !c.W || !c.targets || !c.logprob || (gradient && (!c.Wt || !c.slope))) return QERL_ERR_NULL;
  if (!aligned(c.x, 16) || !aligned(c.W, 16) || !aligned(c.Wt, 16) || !aligned(c.slope, 16) || c.ldx % 8 || c.ldw % 8 || (gradient && c.ld_slope % 4) ||
      !aligned(c.targets, 8) || !aligned(c.logprob, 4) || !aligned(c.lse, 4) || !aligned(c.entropy, 4))
    return QERL_ERR_ALIGN;
  const HeadPlan q = plan_head(c.M, c.V, c.H, gradient);
  if (!c.ws || !aligned(c.ws, 256) || c.ws_bytes < q.bytes) return QERL_ERR_WORKSPACE;
  for (int64_t m0 = 0; m0 < c.M; m0 += q.tokens)
    if (const int e = run_tokens(c, q, m0, c.M - m0 < q.tokens ? c.M - m0 : q.tokens)) return e;
  return QERL_OK;
}

}  // namespace qerl

using namespace qerl;

extern "C" size_t lm_head_prepack_t_bytes(int64_t V, int64_t H) {
  return V < 1 || H < 1 ? 0 : (size_t)(ceil_div(V, 64) * 64) * (size_t)H * 2;
}
extern "C" int lm_head_prepack_t(const void* W, int64_t V, int64_t H, int64_t ldw, void* Wt, void* stream) {
  if (V < 0 || H < 0 || V > kMaxVocab || H % 8 != 0 || ldw < H || ldw >= kMaxLd) return QERL_ERR_SHAPE;
  if (V == 0 || H == 0) return QERL_OK;
  if (!W || !Wt) return QERL_ERR_NULL;
  if (!aligned(W, 16) || !aligned(Wt, 16) || ldw % 8) return QERL_ERR_ALIGN;
  const int64_t vb = ceil_div(V, 64);
  head_transpose_kernel<<<dim3((unsigned)vb, (unsigned)ceil_div(H, 64)), dim3(256), 0, (hipStream_t)stream>>>(
      static_cast<const uint16_t*>(W), V, H, ldw, static_cast<uint16_t*>(Wt), vb * 64);
  return launch_status();
}

extern "C" size_t lm_head_logprob_workspace_bytes(int64_t M, int64_t V, int64_t H, int gradient) {
  if (M < 0 || V < 1 || H < 8 || H % 8 != 0 || M > 0x7fffffff || V > kMaxVocab || H >= kMaxLd) return 0;
  size_t most = 256;                             // a smaller call may split its sums further: the largest over all token blocks
  for (int64_t m : {(int64_t)32, (int64_t)64, (int64_t)128}) {
    const size_t b = M > 0 ? plan_head(M < m ? M : m, V, H, gradient != 0).bytes : 0;
    most = b > most ? b : most;
  }
  for (int64_t m = 256; m - 256 < M && m <= kTokenBlock; m += 256) {
    const size_t b = plan_head(M < m ? M : m, V, H, gradient != 0).bytes;
    most = b > most ? b : most;
  }
  return most;
}

extern "C" int lm_head_logprob(const void* x, int64_t M, int64_t H, int64_t ldx, const void* W, int64_t V, int64_t ldw, const int64_t* targets,
                               float inv_temperature, float* logprob, float* lse, float* entropy, void* ws, size_t ws_bytes, void* stream) {
  return run_head(HeadCall{static_cast<const uint16_t*>(x), M, H, ldx, static_cast<const uint16_t*>(W), V, ldw, nullptr, targets, inv_temperature, logprob, lse,
                           entropy, nullptr, 0, static_cast<uint8_t*>(ws), ws_bytes, (hipStream_t)stream}, false);
}
extern "C" int lm_head_logprob_grad(const void* x, int64_t M, int64_t H, int64_t ldx, const void* W, int64_t V, int64_t ldw, const void* Wt,
                                    const int64_t* targets, float inv_temperature, float* logprob, float* lse, float* entropy, float* slope,
                                    int64_t ld_slope, void* ws, size_t ws_bytes, void* stream) {
  return run_head(HeadCall{static_cast<const uint16_t*>(x), M, H, ldx, static_cast<const uint16_t*>(W), V, ldw, static_cast<const uint16_t*>(Wt), targets,
                           inv_temperature, logprob, lse, entropy, slope, ld_slope, static_cast<uint8_t*>(ws), ws_bytes, (hipStream_t)stream}, true);
}
extern "C" int lm_head_logprob_backward(const float* grad, const float* slope, int64_t ld_slope, int64_t M, int64_t H, void* dx, int64_t lddx, void* stream) {
  if (M < 0 || M > 0x7fffffff || H < 8 || H % 8 || H > 0x7fffffff || ld_slope < H || lddx < H) return QERL_ERR_SHAPE;
  if (M == 0) return QERL_OK;
  if (!grad || !slope || !dx) return QERL_ERR_NULL;
  if (!aligned(grad, 4) || !aligned(slope, 16) || !aligned(dx, 16) || ld_slope % 4 || lddx % 8) return QERL_ERR_ALIGN;
  for (int64_t m0 = 0; m0 < M; m0 += 65535) {
    const int n = (int)(M - m0 < 65535 ? M - m0 : 65535);
    head_backward_kernel<<<dim3((unsigned)ceil_div(H, 2048), (unsigned)n), dim3(256), 0, (hipStream_t)stream>>>(
        grad + m0, slope + m0 * ld_slope, ld_slope, n, H, static_cast<uint16_t*>(dx) + m0 * lddx, lddx);
  }
  return launch_status();
}
