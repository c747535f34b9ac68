// Internal interfaces of the language-model head's log-probabilities.
#pragma once
#include "common.hpp"

namespace qerl {

constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kInf = __builtin_huge_valf();
constexpr float kRaise = 60.f;                  // a logit this far (in powers of two) above the reference raises it

// Some rows of the vocabulary seen by one token: with s = logit * log2(e), others = all of these rows but the token's own,
//   ref: what the sums are relative to, sum = sum_others 2^(s - ref), weighted = sum_others 2^(s - ref) (s - ref), top = max_others s
struct HeadPart { float ref, sum, weighted, top; };

// A probability that holds a large share of what its row's other tokens hold together, and what its rounding to bf16 cut off
struct HeadLarge { int v; float ref, off, s; };  // vocabulary row; off = 2^(s - ref) less the bf16 value
constexpr int kLargeSlots = 64;                  // of a token; one per lane
constexpr float kLargeShare = 1.f / 32;
struct HeadLargeArgs {
  HeadLarge* slot; int* count;                   // [tokens][kLargeSlots], [tokens]; once the row results are there, slots hold (v, weight in slope) only
  float* running;                                // [tokens][2] sum over the pieces so far and what it is relative to
  int parts, part_rows;                          // of this piece; rows of a part
  int first;                                     // the piece is the first one
};

struct HeadArgs {
  const uint16_t* a; int64_t lda, rows;         // row operand [rows, k]: W (rows = vocabulary) or its transpose (rows = hidden)
  const uint16_t* b; int64_t ldb;               // token operand [tokens, k]: x, or the piece's probabilities
  int64_t k; int M;                             // contraction length; tokens at most
  const int* index; const int* count;           // rows of x and targets that the tokens stand for, and how many there are; null: all M as they come
  const int64_t* targets; int64_t V;
  float scale;                                  // log2(e) / temperature
  HeadPart* part; int64_t part_ld;              // [tokens][part_ld]
  float* target_logit;                          // [tokens] s of the token's own row
  int64_t row0; int part0;                      // a's first row in the vocabulary, its first part
  // pieces (gradient)
  uint16_t* p; int64_t ldp;                     // probabilities 2^(s - ref) of the piece, 0 at the token's own row and beyond the vocabulary
  const float* ref;                             // [tokens] the references of this piece
  uint32_t* raise;                              // [tokens] order_key of the largest logit that passed the reference by far, 0: none did
  int* flag;                                    // [token blocks] where one did
  float* ref_next;                              // [tokens] references of the next piece, written with the sums
  int again;                                    // the piece is computed again for the token blocks with a flag, with head_raised_ref
  float* acc;                                   // sums E: [K-part][token block][row block][tile]
  int first;                                    // the sums start here
  int piece_stages;                             // of 64 rows in a whole piece
};
__device__ __forceinline__ int head_tokens(const HeadArgs& a) { return a.count ? *a.count : a.M; }
// Unsigned keys in the order of the floats, all above 0: a maximum over them does not depend on the order of its atomics
__device__ __forceinline__ uint32_t order_key(float f) {
  const uint32_t u = __float_as_uint(f);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ float head_raised_ref(const HeadArgs& a, int token) {
  const uint32_t k = a.raise[token];
  return k ? key_value(k) : a.ref[token];
}
__device__ __forceinline__ int head_row(const HeadArgs& a, int token) { return a.index ? a.index[token] : token; }

// the matrix kernels (lm_head_gemm.hip)
struct HeadGemmPlan { int tokens, rows, part_rows; };   // tokens and vocabulary rows of a tile, rows of a part
HeadGemmPlan plan_head_gemm(int64_t M, int64_t V, bool gradient);
int launch_head_logits(const HeadGemmPlan& p, bool entropy, const HeadArgs& a, hipStream_t st);
int launch_head_probs(const HeadGemmPlan& p, bool entropy, const HeadArgs& a, hipStream_t st);
// the sums: rows of a tile, what the partial sums take; and slope = (1/T) [ (1 - p_t) W_t - sums e_scale - large ones' weights W_v ] from them
struct HeadSumsPlan { int rows; size_t bytes; };
HeadSumsPlan plan_head_sums(const HeadGemmPlan& p, int64_t M, int64_t H, int64_t piece);
int launch_head_sums(const HeadGemmPlan& p, const HeadSumsPlan& q, const HeadArgs& a, hipStream_t st);
int launch_head_slope(const HeadGemmPlan& p, const HeadSumsPlan& q, const HeadArgs& sums, const HeadArgs& head, float inv_temperature, const float* rest,
                      const float* e_scale, const HeadLargeArgs& large, float* slope, int64_t ld_slope, hipStream_t st);

}  // namespace qerl
