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

// The lane, formed anew wherever it is asked for: values derived from one kept all the way would fill
// the registers, and a spilled one's reload waits for the copies in flight.
__device__ __forceinline__ int fresh_lane() {
  int l;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
  return l;
}
// What is the same in every lane, in scalar registers.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ const char* uniform(const char* p) {
  return (const char*)((uintptr_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)p) |
                       ((uintptr_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)((uintptr_t)p >> 32)) << 32));
}

// A row that a worker has a share of: its tiles, its request and what it sees of it.
struct Share {
  int t, first, end, request, visible;
};
// where worker w's tiles begin
__device__ __forceinline__ Share first_share(const PagedArgs& a, int w) {
  const int32_t* s = a.sched + sched_shares(a.T) + (int64_t)w * kShareInts;
  return {uniform(s[0]), uniform(s[1]), uniform(s[2]), uniform(s[3]), uniform(s[4])};
}
// the next row that has tiles after t, whose units end at `at`
__device__ __forceinline__ Share next_share(const PagedArgs& a, int t, int at) {
  const int32_t* before = a.sched + kSchedHeader;
  int end;
  do ++t; while ((end = uniform(before[t + 1])) <= at);
  const RowState rs = row_state(a, t);
  return {t, at + uniform(a.sched[3]), end, uniform(rs.request), uniform(rs.visible)};
}

// Rows that are not read are copied from here (the widest row and its padding).
static __device__ const __attribute__((aligned(16))) unsigned char kZeroRow[4608] = {};

}  // namespace laga
