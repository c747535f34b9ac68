// Internal interfaces of the language-model head's log-probabilities.
#pragma once
#include "common.hpp"

namespace qerl {

// One row block of the vocabulary seen by one token: with s = logit * log2(e), others = every row of the block but the token's own,
//   ref: what the sums are relative to, sum = sum_others 2^(s - ref), weighted = sum_others 2^(s - ref) (s - ref), top = max_others s
struct HeadPart { float ref, sum, weighted, top; };

struct HeadArgs {
  const uint16_t* a; int64_t lda, rows;         // row operand [rows, k]: W (rows = vocabulary), or its transpose (rows = hidden)
  const uint16_t* b; int64_t ldb;               // token operand [tokens, k]: x, or the piece's probabilities
  int64_t k; int M;                             // contraction length; tokens
  const int64_t* targets; int64_t V;
  float scale;                                  // log2(e) / temperature
  HeadPart* part; int64_t part_ld;              // [tokens][part_ld] row blocks
  float* target_logit;                          // [tokens] s of the token's own row
  int64_t row0;                                 // vocabulary row of a's first row (a piece of the vocabulary)
  int block0;                                   // row block of a's first row in `part`
  // pieces (gradient)
  uint16_t* p; int64_t ldp;                     // probabilities 2^(s - ref) of the piece, 0 at the token's own row and beyond the vocabulary
  const float* ref; const float* ref_next;      // [tokens] the references of this piece and of the next (raised where a logit passed it by far)
  const int* flag;                              // [token blocks] piece has to be computed again with ref_next; null: first computation
  float* acc; int64_t ld_acc; int64_t slab;     // sums E [split][tokens][ld_acc]
  int first;                                    // the sums start here
  int split;
};

}  // namespace qerl
