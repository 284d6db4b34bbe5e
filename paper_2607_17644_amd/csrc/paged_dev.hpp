// What the paged attention's kernels share on the device.
#pragma once
#include "common.hpp"
#include "paged.hpp"

namespace laga {

constexpr float kLn2 = 0.69314718055994530942f;

// bf16: what the call computes on the way (q W_k^T and the turned band, the probabilities, the
// normalised sums before W_v) goes into the products as two bf16 operands, x ~ hi + lo to 16
// bits, so that only the inputs and the result have 8. One operand each would round out three
// more times: against fp64 3.0e-3 of out's norm instead of 1.7e-3, its own rounding.
template <typename T> constexpr bool kTwo = sizeof(T) == 2;

// What the row t may see: positions [0, visible); bad: its request or its position lies
// outside the table (the row's results are NaN, nothing is read for it).
struct RowState {
  int request, visible;
  bool bad;
};
__device__ __forceinline__ RowState row_state(const PagedArgs& a, int t) {
  const int p = a.position[t];
  if (p < 0) return {0, 0, false};
  const int r = a.row_request ? a.row_request[t] : t;
  if ((unsigned)r >= (unsigned)a.R || p >= a.width * a.page) return {0, 0, true};
  return {r, p + 1, false};
}

// Rows that are not read are copied from here (the widest row and its padding).
static __device__ const __attribute__((aligned(16))) unsigned char kZeroRow[4608] = {};

}  // namespace laga
