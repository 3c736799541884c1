// Rows of a token policy's logits: what the kernels that read them share.
#pragma once
#include "common.hpp"

namespace pg {

constexpr int LANE_TOKENS = 8;                       // a group: 16 or 32 bytes, two Philox blocks, one byte of a mask
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct LogitArgs {
  pg_logits d;
  int words;                                         // of a mask
  int range;                                         // tokens of a workgroup, a multiple of the counted stretch
  bool count;                                        // there is a history or a bias list
};

// Checks the descriptor alone and fills `a` but for the range; no more than max_rows rows.
pg_status logit_args(const pg_logits* d, const char* who, LogitArgs& a, int32_t max_rows);

// Whether one of `rows` intervals of `b` bytes from q on, each `q_step` after the one before, meets one of `a` bytes from p on (a <= p_step).
bool rows_overlap(uintptr_t p, int64_t p_step, int64_t a, uintptr_t q, int64_t q_step, int64_t b, int64_t rows);

}  // namespace pg
