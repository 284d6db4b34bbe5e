// Serving from a paged cache of latents: the arguments of its launchers and the rules, from
// integers alone, that size their grids and workspace (host and device use the same ones).
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "kernels.hpp"

namespace laga {

// ---------------------------------------------------------------- pages
// The step's plan and the release of pages (paged_cache.hip). Both are a scan over the
// requests (one workgroup) and an expansion of its sums to rows and pages.
struct PlanArgs {
  const int32_t* lengths;     // [R] cached tokens
  const int32_t* arg;         // [R] fresh tokens (plan), or != 0 where the request ends (release)
  int32_t* table;             // [R][width]
  int32_t* free_pages;        // [n_pages], a stack
  const int32_t* free_count;  // [1]
  int32_t* lengths_out;       // [R]; may be lengths
  int32_t* free_count_out;    // [1]; may be free_count
  int32_t* row_begin;         // [R + 1]  (plan)
  int32_t* row_request;       // [rows]   (plan)
  int32_t* position;          // [rows]   (plan)
  int32_t* slot;              // [rows]   (plan)
  int32_t* status;            // [1]
  int32_t* ws;                // plan_ws_ints(R)
  int rows, R, width, n_pages, page;
  int release;
  uint32_t page_magic, page_shift;  // key / page = key page_magic >> page_shift
};
// workspace of a plan or release in two launches: [count, pages, rows, -] then pages_before[R + 1] and the lengths as they were [R]
constexpr int kPlanHeader = 4;
inline size_t plan_ws_ints(long long R) { return kPlanHeader + (size_t)(R + 1) + (size_t)R; }
hipError_t launch_plan(const PlanArgs& a, hipStream_t st);

// Items first, first + step, ... below n: n may be 2^31 - 1, past which a signed item would wrap (step: the
// threads of a launch, below 2^31).
template <typename F>
__host__ __device__ __forceinline__ void each_item(int first, int step, int n, F&& f) {
  for (uint32_t k = (uint32_t)first; k < (uint32_t)n; k += (uint32_t)step) f((int)k);
}
// The last r in [0, n) with sums[r] <= k (sums[0] = 0 <= k < the whole sum: the request of item k).
template <typename Sums>
__host__ __device__ __forceinline__ int find_request(const Sums& sums, int n, int k) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = lo + ((hi - lo) >> 1);  // (lo + hi may pass 2^31)
    if (sums[mid] <= k) lo = mid; else hi = mid;
  }
  return lo;
}

struct AppendArgs {
  const void *latent, *kpe, *gamma;  // [T, d_c], [T, d_rope], [d_c] or NULL
  int64_t latent_stride, kpe_stride;  // elements between rows
  const int32_t *position, *slot;     // [T]
  void* cache;
  int64_t page_stride, position_offset;
  int T, d_c, d_rope, n_slots, page;
  float eps;
  double log2_base;
};
template <typename T>
hipError_t launch_append(const AppendArgs& a, hipStream_t st);

// 8 contiguous elements to and from fp32 (bf16 rounds to nearest even)
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  const frag_t<T> x = *reinterpret_cast<const frag_t<T>*>(p);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = to_f32(x[e]);
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
  frag_t<T> x;
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = to_elem<T>(v[e]);
  *reinterpret_cast<frag_t<T>*>(p) = x;
}

// ---------------------------------------------------------------- attention
// Every row t sees the cached positions 0 .. position[t] of its request. Their tiles of
// kTileKeys keys, row after row, are one sequence of tiles; worker w of a head block takes
// tiles [w * per, (w + 1) * per) of it, whatever rows they belong to, so ragged rows load the
// GPU evenly and a long row is split over as many workers as its length asks for. A row that
// one worker takes whole is finished there; of any other row each worker leaves a partial
// (running maximum, sum, unnormalised output) in the one of its two places that the row's end
// of its range owns.
constexpr int kTileKeys = 32;
constexpr int kCus = 256;  // compute units of an MI355X

struct PagedArgs {
  const void* q;               // [T, H, d_nope + d_rope]
  const void* w;               // W_kv_b [d_c, H * (d_nope + d_v)]
  const void* cache;           // pages of [page][d_c + d_rope], page_stride elements apart
  const int32_t* table;        // [R][width]
  const int32_t* row_request;  // [T] or NULL (row t is request t)
  const int32_t* position;     // [T]
  void* out;                   // [T, H, d_v]
  float* lse;                  // [T, H] or NULL
  int64_t page_stride, position_offset;
  int T, R, width, n_pages, page, H, d_c, d_nope, d_rope, d_v;
  uint32_t page_magic, page_shift;  // key / page = key * page_magic >> page_shift for 0 <= key < 2^31
  float scale_log2;  // softmax_scale * log2(e)
  int rotate;        // 1: q_rope is turned by its row's position first
  double log2_base;
  // workspace
  int32_t* sched;    // layout of the tiles (sched_ints)
  void* qa;          // [T][H][d_c + d_rope]: W_k q_nope, then q_rope
  void* qa_lo;       // bf16: what qa's rounding left, rounded
  void* qa_low2;     // and what that left (in the scores of the band alone; of the rest lse has it)
  float* obar;       // [T][H][d_c]: normalised rows that one worker took whole
  float* part_o;     // [2 * workers][H][d_c]
  float* part_ml;    // [2 * workers][H][2]
  int wide;          // paged_wide.hip's
  int heads_per_wg;  // heads of a head block
  int workers;       // of each head block
  int groups;        // of 32 heads in heads_per_wg, for few tiles (wide kernel), or 0
};
// Layout of the tiles: [units per worker, units, groups, units of a row's cost, whether two successive rows have one
// request], units before each row [T + 1], and of
// each worker's first share (kShareInts) the row, its first tile and end, request and visible keys.
constexpr int kSchedHeader = 5, kShareInts = 8;
__host__ __device__ inline int64_t sched_shares(int64_t T) { return (kSchedHeader + T + 1 + 7) / 8 * 8; }
inline size_t sched_ints(long long T, int workers) { return (size_t)sched_shares(T) + (size_t)kShareInts * workers; }

__host__ __device__ inline int tiles_of(int visible) { return (visible + kTileKeys - 1) / kTileKeys; }
// A row's length in the layout: its tiles and, before them, some units of no tile, which stand for what a
// share costs besides its tiles (q in, the first tiles' way from memory, its result out). Us of a call without
// them and with: wide kernel, 20 x up to 3000 keys, 128 heads 80 and 69 (6 units 71, 24 units 70); 300 x up to 150
// keys, 128 heads 214 and 174; 200 x up to 1500 keys, 32 heads 115 and 101 (24 units 114); the others, 64 x
// up to 4000 keys, d_c = 256, 46 and 43, with 9 units 44; d_c = 1024 120 and 114, 117.
constexpr int kRowCost = 2, kWideRowCost = 9;
__host__ __device__ inline int units_of(int visible, int cost) { return visible > 0 ? cost + tiles_of(visible) : 0; }
// Units per worker: even shares.
__host__ __device__ inline int units_per_worker(int total, int workers) {
  return total > workers ? (int)(((int64_t)total + workers - 1) / workers) : 1;
}
// How the wide kernel's workgroups go about their tiles. With few of them, or rows of about one tile, a workgroup takes
// 32 of its heads (groups of them: one after the other on the workgroups of an XCD) in the general form, in
// which a share starts sooner and more workgroups divide a row; groups 0: the wide way. Both hold the same
// precision. Us of a call this way and wide: 20000 keys, 64 heads 41 and 48; 20 x up to 300 keys, 128 heads 43 and 46;
// 1000 x up to 32 keys, 16 heads 77 and 82; but 600 x up to 150 keys, 64 heads 187 and 178, 64 x up to 2000,
// 16 heads 49 and 43, 20 x up to 3000, 128 heads 77 and 65.
constexpr int kFewTiles = 8;   // units of a worker
constexpr int kShortRows = 2;  // tiles, in the mean
struct Shares { int per, workers, groups, cost, total; };
__host__ __device__ inline Shares shares_of(int tiles, int rows, int workers, int groups) {
  const int few = groups > 0 ? workers / (8 * groups) * 8 : 0;
  if (few > 0) {
    const int total = tiles + rows * kRowCost, per = units_per_worker(total, few);
    if (per <= kFewTiles || tiles < (int64_t)kShortRows * rows) return {per, few, groups, kRowCost, total};
  }
  const int cost = groups > 0 ? kWideRowCost : kRowCost, total = tiles + rows * cost;
  return {units_per_worker(total, workers), workers, 0, cost, total};
}
// The partial place of worker w's share of the row whose tiles begin at unit row_first: a row whose tiles
// begin before the worker's range (or with it) is its first, any other its last.
__host__ __device__ inline int partial_place(int w, int per, int row_first) {
  return 2 * w + (row_first > (int64_t)w * per ? 1 : 0);
}

// With s = ceil(log2(page)) and M = ceil(2^(31 + s) / page) < 2^32: M page = 2^(31 + s) + e with
// e < page <= 2^s, so key M / 2^(31 + s) = key / page + key e / (page 2^(31 + s)), and the second
// term is below 1 / page for key < 2^31: it never carries over to the next whole number.
inline void page_division(int page, uint32_t* magic, uint32_t* shift) {
  uint32_t s = 0;
  while (((int64_t)1 << s) < page) ++s;
  *shift = 31 + s;
  *magic = (uint32_t)((((uint64_t)1 << (31 + s)) + page - 1) / page);
}

struct PagedPlan {
  bool wide;  // paged_wide.hip: bf16 with d_c = 512 and d_rope = 64
  int heads_per_wg, head_blocks, workers, groups;
};
inline PagedPlan paged_plan(int H, int d_c, int d_rope, int elem_size) {
  PagedPlan p;
  p.wide = elem_size == 2 && d_c == 512 && d_rope == 64;
  const int most = p.wide ? 64 : 32;  // heads of a workgroup (all parts of q W_k^T of more would not fit in registers)
  p.head_blocks = (H + most - 1) / most;
  p.heads_per_wg = p.wide ? (H + p.head_blocks - 1) / p.head_blocks : most;
  const int wgs = (elem_size == 2 && d_c <= 256 ? 2 : 1) * kCus;  // what runs at once
  const int w = wgs / p.head_blocks / 8 * 8;  // whole rounds over the 8 XCDs
  p.workers = w > 8 ? w : 8;
  p.groups = p.wide ? (p.heads_per_wg + 31) / 32 : 0;
  return p;
}

void launch_paged_wide(const PagedArgs& a, int head_blocks, hipStream_t st);
template <typename T>
hipError_t launch_paged_attn(const PagedArgs& a, hipStream_t st);

}  // namespace laga
