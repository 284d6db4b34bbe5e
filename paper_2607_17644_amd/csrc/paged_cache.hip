// Pages and rows of a paged cache of latents: the plan of a step (which pages its tokens get,
// which slots they go to), the release of pages, and the rows of new tokens.
#include <math.h>
#include <stdint.h>

#include "laga.h"
#include "paged.hpp"
#include "rope.hpp"

namespace laga {
namespace {

// ---------------------------------------------------------------- plan and release
// Two sums over the requests (rows and pages before each), then one thread per row and per
// page that finds its request in them by bisection. Nothing is decided by the order of
// threads: page k of the step is the k-th from the top of the stack, in request order.
constexpr int kScanThreads = 1024, kScanPer = 4;         // requests per thread and turn
constexpr int kScanChunk = kScanThreads * kScanPer;
constexpr int kFillThreads = 256;
constexpr int kSearchLds = 4096;  // sums of this many requests are searched in LDS

__device__ __forceinline__ int page_of(const PlanArgs& a, int key) {
  return (int)((uint64_t)(uint32_t)key * a.page_magic >> a.page_shift);
}
__device__ __forceinline__ int pages_of(const PlanArgs& a, int n) { return page_of(a, n + a.page - 1); }

// Exclusive sums over the workgroup of (rows, pages) per thread; total[] gets the workgroup's. (Pages are at
// most requests x table width, below 2^31.)
__device__ void block_scan(int64_t& rows, int& pages, int64_t (&total)[2], int64_t (*sm)[2]) {
  const int l = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t r = rows;
  int p = pages;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t r1 = __shfl_up(r, o);
    const int p1 = __shfl_up(p, o);
    if (l >= o) { r += r1; p += p1; }
  }
  if (l == 63) { sm[wave][0] = r; sm[wave][1] = p; }
  __syncthreads();
  int64_t rb = 0, pb = 0, rt = 0, pt = 0;
#pragma unroll
  for (int w = 0; w < kScanThreads / 64; ++w) {
    if (w == wave) { rb = rt; pb = pt; }
    rt += sm[w][0];
    pt += sm[w][1];
  }
  __syncthreads();
  total[0] = rt; total[1] = pt;
  rows = rb + r - rows;
  pages = (int)pb + p - pages;
}

// What a plan or release hands out, and where to find it: sums and the lengths before the step, by request.
struct Handout {
  const int32_t *pages_before, *row_begin, *lengths;
  int count, pages, rows;
};
// Rows and pages first, first + step, ... of it.
__device__ __forceinline__ void expand(const PlanArgs& a, const Handout& x, int first, int step) {
  each_item(first, step, x.pages, [&](int k) {
    const int r = find_request(x.pages_before, a.R, k), j = k - x.pages_before[r];
    int32_t* entry = a.table + (int64_t)r * a.width + j;
    if (a.release) a.free_pages[x.count + k] = *entry;
    else entry[pages_of(a, x.lengths[r])] = a.free_pages[x.count - 1 - k];
  });
  if (a.release) return;
  each_item(first, step, a.rows, [&](int t) {
    int request = -1, position = -1, slot = -1;
    if (t < x.rows) {
      request = find_request(x.row_begin, a.R, t);
      const int len = x.lengths[request];
      position = len + t - x.row_begin[request];
      // the entry in the table, or the page that this step puts there
      const int j = page_of(a, position), have = pages_of(a, len);
      const int32_t* from = j < have ? a.table + (int64_t)request * a.width + j
                                     : a.free_pages + (x.count - 1 - (x.pages_before[request] + j - have));
      const int id = *from;
      if ((unsigned)id < (unsigned)a.n_pages) slot = id * a.page + (position - j * a.page);
    }
    a.row_request[t] = request;
    a.position[t] = position;
    a.slot[t] = slot;
  });
}

// FILL: this workgroup also expands the sums (small steps: one launch), from LDS up to kSearchLds requests.
template <bool FILL>
__global__ __launch_bounds__(kScanThreads) void plan_scan_kernel(PlanArgs a) {
  __shared__ int64_t sm[kScanThreads / 64][2];
  __shared__ int bad;
  __shared__ int32_t s_pages[FILL ? kSearchLds : 1], s_rows[FILL ? kSearchLds : 1], s_lengths[FILL ? kSearchLds : 1];
  int32_t* pages_before = a.ws + kPlanHeader;
  int32_t* lengths = pages_before + a.R + 1;
  const bool lds = FILL && a.R <= kSearchLds;
  const int tid = threadIdx.x, count = a.free_count[0];
  const int64_t room = (int64_t)a.width * a.page;
  if (tid == 0) bad = 0;

  int64_t rows0 = 0, pages0 = 0;
  int len[kScanPer], arg[kScanPer];
  for (int64_t base = 0; base < a.R; base += kScanChunk) {
    int64_t rows = 0;
    int f[kScanPer], n[kScanPer], pages = 0, err = 0;
#pragma unroll
    for (int i = 0; i < kScanPer; ++i) {
      const int64_t r = base + tid * kScanPer + i;
      len[i] = arg[i] = 0;
      if (r < a.R) len[i] = a.lengths[r], arg[i] = a.arg[r];
    }
#pragma unroll
    for (int i = 0; i < kScanPer; ++i) {
      f[i] = n[i] = 0;
      if (len[i] < 0 || (!a.release && arg[i] < 0)) err |= LAGA_PLAN_INVALID;
      else if (len[i] + (a.release ? 0 : (int64_t)arg[i]) > room) err |= LAGA_PLAN_TABLE;
      else if (a.release) n[i] = arg[i] ? pages_of(a, len[i]) : 0;
      else {
        f[i] = arg[i];
        n[i] = pages_of(a, len[i] + arg[i]) - pages_of(a, len[i]);
      }
      rows += f[i];
      pages += n[i];
    }
    if (base == 0) __syncthreads();  // bad is cleared
    if (err) atomicOr(&bad, err);    // (bits of a set: no order)
    int64_t total[2];
    block_scan(rows, pages, total, sm);
    rows += rows0;
    pages += (int)pages0;
#pragma unroll
    for (int i = 0; i < kScanPer; ++i) {
      const int64_t r = base + tid * kScanPer + i;
      if (r < a.R) {  // (sums past 2^31 end in an error below: nothing reads them)
        if (!a.release) a.row_begin[r] = (int32_t)rows;
        if (lds) {
          s_pages[r] = pages, s_rows[r] = (int32_t)rows, s_lengths[r] = len[i];
        } else {
          pages_before[r] = pages;
          lengths[r] = len[i];
        }
      }
      rows += f[i];
      pages += n[i];
    }
    rows0 += total[0];
    pages0 += total[1];
  }
  __syncthreads();
  int status = bad;
  if (count < 0 || count > a.n_pages) status |= LAGA_PLAN_INVALID;
  else if (a.release ? count + pages0 > a.n_pages : pages0 > count) status |= LAGA_PLAN_PAGES;
  if (!a.release && rows0 > a.rows) status |= LAGA_PLAN_ROWS;
  const bool ok = status == 0;
  const int n_pages = ok ? (int)pages0 : 0, n_rows = ok ? (int)rows0 : 0;
  if constexpr (FILL) {  // (apart, so that LDS is read as LDS)
    if (lds) expand(a, Handout{s_pages, s_rows, s_lengths, count, n_pages, n_rows}, tid, kScanThreads);
    else expand(a, Handout{pages_before, a.row_begin, lengths, count, n_pages, n_rows}, tid, kScanThreads);
  }

  // the state after the step (every input has been read)
  auto state = [&](int64_t r, int len, int arg) {
    a.lengths_out[r] = !ok ? len : a.release ? (arg ? 0 : len) : len + arg;
    if (!a.release && !ok) a.row_begin[r] = 0;
  };
  if (a.R <= kScanChunk) {
#pragma unroll
    for (int i = 0; i < kScanPer; ++i)
      if (tid * kScanPer + i < a.R) state(tid * kScanPer + i, len[i], arg[i]);
  } else {
    for (int64_t r = tid; r < a.R; r += kScanThreads) state(r, lengths[r], a.arg[r]);
  }
  if (tid == 0) {
    if (!FILL) a.ws[0] = count, a.ws[1] = n_pages, a.ws[2] = n_rows;
    a.status[0] = status;
    a.free_count_out[0] = !ok ? count : a.release ? count + (int32_t)pages0 : count - (int32_t)pages0;
    if (!a.release) a.row_begin[a.R] = n_rows;
  }
}

__global__ __launch_bounds__(kFillThreads) void plan_fill_kernel(PlanArgs a) {
  __shared__ int32_t s_pages[kSearchLds], s_rows[kSearchLds];
  const int32_t* pages_before = a.ws + kPlanHeader;
  const bool lds = a.R <= kSearchLds;
  if (lds) {
    for (int r = threadIdx.x; r < a.R; r += kFillThreads) {
      s_pages[r] = pages_before[r];
      if (!a.release) s_rows[r] = a.row_begin[r];
    }
    __syncthreads();
  }
  const int32_t* lengths = pages_before + a.R + 1;
  const int first = blockIdx.x * kFillThreads + threadIdx.x, step = gridDim.x * kFillThreads;
  if (lds) expand(a, Handout{s_pages, s_rows, lengths, a.ws[0], a.ws[1], a.ws[2]}, first, step);
  else expand(a, Handout{pages_before, a.row_begin, lengths, a.ws[0], a.ws[1], a.ws[2]}, first, step);
}

// ---------------------------------------------------------------- rows of new tokens
constexpr int kWaves = 4;

// One wave takes TPW tokens: their latent rows are held in registers (CH chunks of 8 elements
// per lane), then its lanes take one pair of the shared key each, of 64 / (d_rope / 2) tokens
// at a time, so that no lane forms more than one angle.
template <typename T, int TPW, int CH>
__global__ __launch_bounds__(64 * kWaves) void append_kernel(AppendArgs a) {
  const int l = threadIdx.x & 63;
  const int64_t t0 = ((int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6)) * TPW;
  if (t0 >= a.T) return;  // wave-uniform; the kernel has no barrier
  const int nch = a.d_c / 8, width = a.d_c + a.d_rope;
  T* cache = (T*)a.cache;
  auto row_of = [&](int slot) {
    return cache + (int64_t)(slot / a.page) * a.page_stride + (int64_t)(slot % a.page) * width;
  };

  float v[TPW][CH][8], ss[TPW];
  int slot[TPW];
#pragma unroll
  for (int i = 0; i < TPW; ++i) {
    slot[i] = t0 + i < a.T ? a.slot[t0 + i] : -1;
    if ((unsigned)slot[i] >= (unsigned)a.n_slots) slot[i] = -1;
    ss[i] = 0.f;
    const T* x = (const T*)a.latent + (t0 + i < a.T ? t0 + i : t0) * a.latent_stride;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int ch = l + 64 * k;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][k][e] = 0.f;
      if (ch < nch) load8(x + 8 * ch, v[i][k]);
    }
  }
#pragma unroll
  for (int i = 0; i < TPW; ++i) {
#pragma unroll
    for (int k = 0; k < CH; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) ss[i] = __builtin_fmaf(v[i][k][e], v[i][k][e], ss[i]);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) ss[i] += __shfl_xor(ss[i], o);
  }
#pragma unroll
  for (int k = 0; k < CH; ++k) {
    const int ch = l + 64 * k;
    if (ch >= nch) continue;
    float g[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = 1.f;
    if (a.gamma) load8((const T*)a.gamma + 8 * ch, g);
#pragma unroll
    for (int i = 0; i < TPW; ++i) {
      if (slot[i] < 0) continue;  // wave-uniform
      const float r = 1.f / sqrtf(ss[i] / (float)a.d_c + a.eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][k][e] = a.gamma ? (v[i][k][e] * r) * g[e] : v[i][k][e] * r;
      store8(row_of(slot[i]) + 8 * ch, v[i][k]);
    }
  }

  const int pairs = a.d_rope / 2, p = l % pairs;  // pairs divides 64
  const double freq = rope_freq(p, a.d_rope, a.log2_base);
  for (int i = l / pairs; i < TPW; i += 64 / pairs) {
    const int64_t t = t0 + i;
    if (t >= a.T) break;
    const int s = a.slot[t];
    if ((unsigned)s >= (unsigned)a.n_slots) continue;
    float cs, sn;
    rope_sincos(a.position_offset + a.position[t], freq, cs, sn);
    const T* x = (const T*)a.kpe + t * a.kpe_stride + 2 * p;
    T* y = row_of(s) + a.d_c + 2 * p;
    const float x0 = to_f32(x[0]), x1 = to_f32(x[1]);
    y[0] = to_elem<T>(x0 * cs - x1 * sn);
    y[1] = to_elem<T>(x0 * sn + x1 * cs);
  }
}

}  // namespace

// One launch, the scanning workgroup expanding its own sums, where it has few rows and pages
// to do; else a second launch over the GPU. Bound by a chain of loads (lengths, sums, stack or table):
// 64 requests 6.2 us in one, 4.3 + 2.9 in two; 500 requests with 15 new tokens each in the mean, 7500 rows,
// 7.5 and 4.5 + 4.3, and a launch's gap in between.
hipError_t launch_plan(const PlanArgs& a, hipStream_t st) {
  const int64_t items = a.release ? (int64_t)a.R * a.width : a.rows;
  if (items <= 8 * kScanThreads) {
    plan_scan_kernel<true><<<1, kScanThreads, 0, st>>>(a);
    return hipGetLastError();
  }
  plan_scan_kernel<false><<<1, kScanThreads, 0, st>>>(a);
  const int64_t wgs = (items + kFillThreads - 1) / kFillThreads;
  plan_fill_kernel<<<(unsigned)(wgs < 4 * kCus ? wgs : 4 * kCus), kFillThreads, 0, st>>>(a);
  return hipGetLastError();
}

template <typename T, int TPW>
static void launch_append_t(const AppendArgs& a, hipStream_t st) {
  const int per = kWaves * TPW;
  const unsigned wgs = (unsigned)(((int64_t)a.T + per - 1) / per);
  if (a.d_c <= 512) append_kernel<T, TPW, 1><<<wgs, 64 * kWaves, 0, st>>>(a);
  else append_kernel<T, TPW, 2><<<wgs, 64 * kWaves, 0, st>>>(a);
}

template <typename T>
hipError_t launch_append(const AppendArgs& a, hipStream_t st) {
  // A wave per token up to 16 waves per CU, then two tokens one after the other, which halves the waves that wait to
  // begin. Us with one, two and four per wave (bf16, d_c = 512, 64 wide band): 64 tokens 3.2, 3.7, 5.2; 2048 3.9, 4.1, 5.5;
  // 4096 5.5, 5.4, 6.7; 8192 9.1, 8.3, 9.5; 16384 14.4, 12.7, 13.0 (37.9 MB read and written: 3.0 TB/s). d_c = 64: 1024 4.1,
  // 4.4, 6.6; 8192 7.1, 5.8, 5.9; d_c = 1024: 2048 5.2, 5.8, 8.3; 16384 21.9, 19.9, 21.1; fp32: 2048 4.4, 4.6, 5.9; 16384 20.4, 19.7, 19.9.
  if (a.T <= 16 * kCus) launch_append_t<T, 1>(a, st);
  else launch_append_t<T, 2>(a, st);
  return hipGetLastError();
}

template hipError_t launch_append<bf16>(const AppendArgs&, hipStream_t);
template hipError_t launch_append<float>(const AppendArgs&, hipStream_t);

}  // namespace laga
