// Attention of new tokens over a paged cache of latents, in the absorbed form: with head h's
// columns [W_k || W_v] of W_kv_b,
//
//   qa = W_k q_nope,  z_j = scale (qa . c_j + q_rope . k_j),  o = sum_j softmax(z)_j c_j,  out = W_v^T o
//
// so that a cached position is one row [c_j || k_j] that every head reads, and no per-head key
// or value exists. Launches: the products qa, the turned q_rope and the layout of the tiles
// (absorb_kernel), the attention split over the cache (split_kernel, or paged_wide.hip's), and the
// join of split rows with the product by W_v (join_vec_kernel, or combine_kernel and join_kernel).
// Bound by the cache's bytes for few heads (2 (2 d_c + d_rope) flop per head for each row of d_c
// + d_rope elements), by the products too for 128.
#include <math.h>

#define LAGA_LDS_DMA_ASM 1
#include "common.hpp"
#include "paged_split.hpp"
#include "rope.hpp"

namespace laga {
namespace {

// ---------------------------------------------------------------- absorb
// qa^T = W_k q_nope^T per head. A workgroup has 128 rows of W_kv_b (their d_nope elements of a head
// are contiguous) and goes through its share of the tokens, 32 at a time; a wave has 32 of the
// rows. Bound by reading W and writing qa: W's rows come in whole by direct copies (fragments
// straight from global memory read each line four times over: 128 heads x 61 tokens 22 us), results
// leave through LDS in rows of 256 bytes. Beside them one workgroup per token turns its
// q_rope, and one lays out the tiles.
constexpr int kAbsorbWaves = 4, kAbsorbRows = 32 * kAbsorbWaves;
static_assert(kAbsorbRows == kQaBlock);

// N elements of qa; bf16 in three parts, each the rounding of what the ones before leave (the sum is
// within 2^-25 of the value: the scores of a row with one key are its lse, and two parts left 2.5e-6 there).
template <typename T, int N>
__device__ __forceinline__ void store_parts(const PagedArgs& a, int64_t at, const float (&y)[N]) {
  typedef __attribute__((__vector_size__(N * sizeof(T)))) T vec;
  vec v, low, low2;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    v[e] = to_elem<T>(y[e]);
    const float rest = y[e] - to_f32(v[e]);
    low[e] = to_elem<T>(rest);
    low2[e] = to_elem<T>(rest - to_f32(low[e]));
  }
  *reinterpret_cast<vec*>((T*)a.qa + at) = v;
  if constexpr (kTwo<T>) {
    *reinterpret_cast<vec*>((T*)a.qa_lo + at) = low;
    *reinterpret_cast<vec*>((T*)a.qa_low2 + at) = low2;
  }
}

// A value of the band in three bf16 parts, each cut off what the ones before leave, so that all have the value's sign
// (and 3 x 8 bits are the whole of it): a cached key may be infinite, and the sum of its products with the parts has
// to be the infinity that its product with the value is. Nor may a part be zero beside one that is not: it is
// 2^-126 then, less than 2^-26 of any value from 2^-100 on.
__device__ __forceinline__ void band_parts(float y, bf16 (&part)[3]) {
  auto cut = [](float x) { return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x) & 0xffff0000u); };
  float p[3];
  p[0] = cut(y);
  p[1] = cut(y - p[0]);
  p[2] = cut((y - p[0]) - p[1]);
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    if (i > 0 && p[i] == 0.f && p[0] != 0.f) p[i] = __builtin_copysignf(0x1p-126f, p[0]);
    part[i] = (bf16)p[i];
  }
}

// Q8 (here and below): qa stays in fp32, four of a head's next to the same four of the next head's, as the split reads them,
// and the largest magnitude of each row of a block is left beside it.
__device__ __forceinline__ f32x4* q8_place(const PagedArgs& a, int t, int h, int c) {
  return (f32x4*)a.qa + ((int64_t)t * ((a.d_c + a.d_rope) / 4) + c / 4) * a.H + h;
}
template <typename T, int DN, bool Q8>
__device__ void absorb_product(const PagedArgs& a, int blk, int cblocks, int tpart, int tparts) {
  constexpr int E = 16 / sizeof(T), CPR = DN / E, PO = kAbsorbRows + 4;  // chunks of a row; pitch of the results
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  T* sw = (T*)smem;
  T* sq = sw + kAbsorbRows * DN;
  float* so = (float*)(sq + 32 * DN);
  const int l = threadIdx.x & 63, n = l & 31, g = l >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = blk / cblocks, c0 = blk % cblocks * kAbsorbRows, nc = min(kAbsorbRows, a.d_c - c0);
  const int W = a.d_c + a.d_rope, dqk = DN + a.d_rope;
  const int64_t ldw = (int64_t)a.H * (DN + a.d_v), ldq = (int64_t)a.H * dqk;
  const T* w = (const T*)a.w + c0 * ldw + (int64_t)h * (DN + a.d_v);
  // chunk c of a row is at c ^ swz (bf16); rows past the end repeat the last one
  auto copy = [&](const T* src, int64_t stride, int rows, int last, T* dst) {
    for (int p0 = wave * 64; p0 < rows * CPR; p0 += 64 * kAbsorbWaves) {
      const int r = (p0 + l) / CPR;
      int c = (p0 + l) % CPR;
      if constexpr (sizeof(T) == 2) c ^= swz<CPR>(r);
      g2lds16(src + min(r, last) * stride + c * E, dst + p0 * E);
    }
  };
  auto frag = [&](const T* tile, int r, int ks) {
    if constexpr (sizeof(T) == 2) return swz_frag<T, CPR>(tile, r, 2 * ks + g);
    else return lds_frag<T>(tile + r * DN + 16 * ks + 8 * g);
  };
  copy(w, ldw, kAbsorbRows, nc - 1, sw);
  for (int t0 = tpart * 32; t0 < a.T; t0 += tparts * 32) {
    const int nt = min(32, a.T - t0);
    copy((const T*)a.q + t0 * ldq + (int64_t)h * dqk, ldq, 32, nt - 1, sq);
    wait_vmem();
    lds_barrier();
    f32x16 acc = {};
#pragma unroll
    for (int ks = 0; ks < DN / 16; ++ks) mma(acc, frag(sw, 32 * wave + n, ks), frag(sq, n, ks));
#pragma unroll
    for (int rr = 0; rr < 4; ++rr)
      *reinterpret_cast<f32x4*>(so + n * PO + 32 * wave + 8 * rr + 4 * g) =
          f32x4{acc[4 * rr], acc[4 * rr + 1], acc[4 * rr + 2], acc[4 * rr + 3]};
    lds_barrier();
    for (int x = threadIdx.x; x < nt * (kAbsorbRows / E); x += 64 * kAbsorbWaves) {
      const int r = x / (kAbsorbRows / E), c = x % (kAbsorbRows / E) * E;
      const int64_t th = (int64_t)(t0 + r) * a.H + h;
      if (!Q8 && c >= nc) continue;
      float y[E];
#pragma unroll
      for (int i = 0; i < E; i += 4) *reinterpret_cast<f32x4*>(y + i) = *reinterpret_cast<const f32x4*>(so + r * PO + c + i);
      if constexpr (Q8) {
        float top = 0.f;  // (rows of W past the end repeat the last one: they change no maximum)
#pragma unroll
        for (int i = 0; i < E; ++i) top = fmaxf(top, fabsf(y[i]));
#pragma unroll
        for (int o = 1; o < kAbsorbRows / E; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));  // (the lanes of a row are all here)
        if (c == 0) a.qa_max[th * qa_blocks(a.d_c) + c0 / kQaBlock] = top;
        if (c < nc)
#pragma unroll
          for (int i = 0; i < E; i += 4) *q8_place(a, t0 + r, h, c0 + c + i) = *reinterpret_cast<f32x4*>(y + i);
      } else {
        store_parts<T, E>(a, th * W + c0 + c, y);
      }
    }
    if (t0 + tparts * 32 < a.T) lds_barrier();  // q and the results are read
  }
}
template <typename T, int DN>
constexpr size_t absorb_lds() {
  return sizeof(T) * (size_t)(kAbsorbRows + 32) * DN + sizeof(float) * 32 * (kAbsorbRows + 4);
}

// q_rope of one token, every head: a thread keeps one pair's angle and has eight heads' pairs under way (one
// after the other, the launch took 11 us for 2 rows of 128 heads, so 7)
constexpr int kBandHeads = 8;
template <typename T, bool Q8>
__device__ void absorb_band(const PagedArgs& a, int t) {
  const int pairs = a.d_rope / 2, i = threadIdx.x % pairs;
  const int W = a.d_c + a.d_rope, dqk = a.d_nope + a.d_rope;
  float cs = 1.f, sn = 0.f;
  if (a.rotate) rope_sincos(a.position_offset + a.position[t], rope_freq(i, a.d_rope, a.log2_base), cs, sn);
  typedef __attribute__((__vector_size__(2 * sizeof(T)))) T pair;
  const int step = 64 * kAbsorbWaves / pairs;
  for (int h0 = threadIdx.x / pairs; h0 < a.H; h0 += kBandHeads * step) {
    pair x[kBandHeads];
#pragma unroll
    for (int u = 0; u < kBandHeads; ++u)
      if (h0 + u * step < a.H)
        x[u] = *reinterpret_cast<const pair*>((const T*)a.q + ((int64_t)t * a.H + h0 + u * step) * dqk + a.d_nope + 2 * i);
#pragma unroll
    for (int u = 0; u < kBandHeads; ++u) {
      if (h0 + u * step >= a.H) break;
      const float x0 = to_f32(x[u][0]), x1 = to_f32(x[u][1]);
      const float y[2] = {x0 * cs - x1 * sn, x0 * sn + x1 * cs};
      const int64_t th = (int64_t)t * a.H + h0 + u * step, at = th * W + a.d_c + 2 * i;
      if constexpr (Q8) {
        float top = fmaxf(fabsf(y[0]), fabsf(y[1]));
        for (int o = 1; o < pairs; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));  // (the lanes of a head are all here)
        const int blocks = qa_blocks(a.d_c);
        if (i == 0) a.qa_max[th * blocks + blocks - 1] = top;
        float2* to = (float2*)q8_place(a, t, h0 + u * step, a.d_c + (2 * i & ~3));
        to[i & 1] = float2{y[0], y[1]};
      } else if constexpr (kTwo<T>) {
        bf16 part[2][3];
#pragma unroll
        for (int e = 0; e < 2; ++e) band_parts(y[e], part[e]);
        *reinterpret_cast<pair*>((T*)a.qa + at) = pair{part[0][0], part[1][0]};
        *reinterpret_cast<pair*>((T*)a.qa_lo + at) = pair{part[0][1], part[1][1]};
        *reinterpret_cast<pair*>((T*)a.qa_low2 + at) = pair{part[0][2], part[1][2]};
      } else {
        *reinterpret_cast<pair*>((T*)a.qa + at) = pair{y[0], y[1]};
      }
    }
  }
}

// Units before each row, units per worker, and each worker's first share.
constexpr int kLayoutLds = 2048;  // rows whose sums and states are kept in LDS
__device__ void lay_out_tiles(const PagedArgs& a) {
  constexpr int NT = 64 * kAbsorbWaves;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  int32_t *s_before = (int32_t*)smem, *s_request = s_before + kLayoutLds, *s_visible = s_request + kLayoutLds;
  int32_t* sm = s_visible + kLayoutLds;
  const int tid = threadIdx.x, l = tid & 63, wave = tid >> 6;
  const bool lds = a.T <= kLayoutLds;
  int32_t* before = a.sched + kSchedHeader;
  // all tiles, the rows that have any, and whether one has the request of the row before it
  RowState mine = {0, 0, false};
  int tiles = 0, rows = 0, again = 0;
  for (int t = tid; t < a.T; t += NT) {
    const RowState rs = row_state(a, t);
    if (t < NT) mine = rs;
    tiles += tiles_of(rs.visible);
    rows += rs.visible > 0;
    if (a.row_request && t > 0 && rs.visible > 0) {
      const RowState last = row_state(a, t - 1);
      again |= last.visible > 0 && last.request == rs.request;
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    tiles += __shfl_xor(tiles, o);
    rows += __shfl_xor(rows, o);
  }
  if (l == 0) sm[wave] = tiles, sm[kAbsorbWaves + wave] = rows;
  again = __syncthreads_or(again);
  tiles = rows = 0;
  for (int w = 0; w < kAbsorbWaves; ++w) tiles += sm[w], rows += sm[kAbsorbWaves + w];
  Shares sh = shares_of(tiles, rows, a.workers, a.groups);
  if (a.row_cost > 0) {
    sh.cost = a.row_cost;
    sh.total = tiles + rows * sh.cost;
    sh.per = units_per_worker(sh.total, sh.workers);
  }
  __syncthreads();
  int sum = 0;
  for (int base = 0; base < a.T; base += NT) {
    const int t = base + tid;
    RowState rs = {0, 0, false};
    if (t < a.T) rs = base == 0 ? mine : row_state(a, t);
    const int n = units_of(rs.visible, sh.cost);
    int inc = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int up = __shfl_up(inc, o);
      if (l >= o) inc += up;
    }
    if (l == 63) sm[wave] = inc;
    __syncthreads();
    int b = sum;
    for (int w = 0; w < kAbsorbWaves; ++w) {
      if (w < wave) b += sm[w];
      sum += sm[w];
    }
    __syncthreads();
    if (t < a.T) {
      before[t] = b + inc - n;
      if (lds) {
        s_before[t] = b + inc - n;
        s_request[t] = rs.request;
        s_visible[t] = rs.visible;
      }
    }
  }
  if (tid == 0) {
    before[a.T] = sum;
    a.sched[0] = sh.per;
    a.sched[1] = sum;
    a.sched[2] = sh.groups;
    a.sched[3] = sh.cost;
    a.sched[4] = again != 0;
  }
  __syncthreads();
  const int32_t* sums = lds ? s_before : before;
  for (int w = tid; w < sh.workers; w += NT) {
    const int64_t start = (int64_t)w * sh.per;
    if (start >= sum) break;
    int lo = 0, hi = a.T;  // last row whose units begin at or before start
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (sums[mid] <= start) lo = mid; else hi = mid;
    }
    const int end = lo + 1 < a.T ? sums[lo + 1] : sum;
    const RowState rs = lds ? RowState{s_request[lo], s_visible[lo], false} : row_state(a, lo);
    int32_t* out = a.sched + sched_shares(a.T) + (int64_t)w * kShareInts;
    typedef __attribute__((__vector_size__(4 * sizeof(int)))) int i32x4;
    *reinterpret_cast<i32x4*>(out) = i32x4{lo, sums[lo] + sh.cost, end, rs.request};
    out[4] = rs.visible;
  }
}
constexpr size_t layout_lds() { return sizeof(int32_t) * (3 * kLayoutLds + 2 * kAbsorbWaves); }

template <typename T, int DN, bool Q8>
__global__ __launch_bounds__(64 * kAbsorbWaves) void absorb_kernel(PagedArgs a, int cblocks, int tparts) {
  // the few long jobs first
  const int others = a.T + 1, id = blockIdx.x;
  if (id == 0) lay_out_tiles(a);
  else if (id < others) absorb_band<T, Q8>(a, id - 1);
  else absorb_product<T, DN, Q8>(a, (id - others) / tparts, cblocks, (id - others) % tparts, tparts);
}

// ---------------------------------------------------------------- split attention
template <typename T, int ND>
__global__ __launch_bounds__(256, sizeof(T) == 2 && ND <= 2 ? 2 : 1) void split_kernel(PagedArgs a, int head_blocks) {
  __shared__ __attribute__((aligned(16))) unsigned char smem[SplitCfg<T, ND>::LDS];
  // the head blocks of a worker follow each other on one XCD: its L2 serves all but the first
  const int id = blockIdx.x, hb = id / 8 % head_blocks, w = id / (8 * head_blocks) * 8 + id % 8;
  const int h0 = hb * a.heads_per_wg;
  split_shares<T, ND>(a, smem, w, h0, min(a.heads_per_wg, a.H - h0), a.sched[0], a.sched[1]);
}

// ---------------------------------------------------------------- join
// The running softmax of some partials of a row: this thread's four columns of sum f o, with f
// = exp2(m - max m), and the sum of f l.
struct Joined {
  float m, l;
  f32x4 o;
};
__device__ __forceinline__ void join_in(Joined& x, float m, float l, const f32x4& o) {
  const float m_new = fmaxf(x.m, m), m_use = m_new == -INFINITY ? 0.f : m_new;
  const float f = fast_exp2(m - m_use), old = x.m == -INFINITY ? 0.f : fast_exp2(x.m - m_use);
  x.m = m_new;
  x.l = __builtin_fmaf(x.l, old, f * l);
#pragma unroll
  for (int e = 0; e < 4; ++e) x.o[e] = __builtin_fmaf(f, o[e], x.o[e] * old);
}
// The workers [w0, w1] that share row t; split false: one worker took the row whole, or none did
// (seen false), or the row is bad (fill: what its results are then).
struct RowParts {
  int first, w0, w1;
  bool seen, split;
  float fill;
};
__device__ __forceinline__ RowParts parts_of(const PagedArgs& a, int t) {
  const int32_t* before = a.sched + kSchedHeader;
  const int per = a.sched[0], first = before[t] + a.sched[3], end = before[t + 1];
  if (before[t] == end) return {0, 0, -1, false, false, row_state(a, t).bad ? NAN : 0.f};
  const int w0 = first / per, w1 = (end - 1) / per;
  return {first, w0, w1, true, w0 != w1, 0.f};
}
// bf16: the scores lack the third part of q W_k^T. lse's share of it to first order is scale sum_c dqa_c o_c with the
// row's normalised sum o; out's is below 2^-16 of a probability.
// Partials of a row's head, dealt to `groups` threads of the same four columns (c), then joined in order
// through LDS (room: 24 bytes per thread). The result is complete in the threads of group 0.
__device__ __forceinline__ Joined join_parts(const PagedArgs& a, const RowParts& r, int h, int c, int group, int groups,
                                             int quads, bool mine, unsigned char* lds) {
  Joined x = {-INFINITY, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
  const int per = a.sched[0];
  if (mine)
#pragma unroll 8
    for (int w = r.w0 + group; w <= r.w1; w += groups) {
      const int64_t p = (int64_t)partial_place(w, per, r.first) * a.H + h;
      join_in(x, a.part_ml[2 * p], a.part_ml[2 * p + 1], *reinterpret_cast<const f32x4*>(a.part_o + p * a.d_c + c));
    }
  if (groups == 1) return x;
  f32x4* so = (f32x4*)lds;
  float2* sm = (float2*)(so + blockDim.x);
  so[threadIdx.x] = x.o;
  sm[threadIdx.x] = float2{x.m, x.l};
  __syncthreads();
  if (group == 0 && mine)
    for (int u = 1; u < groups; ++u) join_in(x, sm[u * quads + threadIdx.x].x, sm[u * quads + threadIdx.x].y, so[u * quads + threadIdx.x]);
  return x;
}

// Rows that several workers share, put together in obar: a workgroup per row and some heads. Bound by
// reading the partials (128 heads x 61 rows 17 us; within the product's own kernel, where a lane had several
// loads of 16 bytes under way at most, 47 us for both against 19 + 17).
constexpr int kCombineThreads = 256;
template <int HEADS>
__global__ __launch_bounds__(kCombineThreads) void combine_kernel(PagedArgs a) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[24 * kCombineThreads];
  const int hblocks = (a.H + HEADS - 1) / HEADS, t = blockIdx.x / hblocks, h0 = blockIdx.x % hblocks * HEADS;
  const RowParts r = parts_of(a, t);
  if (!r.split) return;
  const int quads = a.d_c / 4, groups = kCombineThreads / quads, group = threadIdx.x / quads;
  const int c = threadIdx.x % quads * 4;
  for (int h = h0; h < min(a.H, h0 + HEADS); ++h) {
    const Joined x = join_parts(a, r, h, c, group, groups, quads, group < groups, lds);
    if (group == 0) {
      const int64_t th = (int64_t)t * a.H + h;
      const float inv = 1.f / x.l;
      *reinterpret_cast<f32x4*>(a.obar + th * a.d_c + c) = f32x4{x.o[0] * inv, x.o[1] * inv, x.o[2] * inv, x.o[3] * inv};
      if (c == 0 && a.lse) a.lse[th] = (x.m + fast_log2(x.l)) * kLn2;
    }
    if (HEADS > 1) __syncthreads();  // lds is read
  }
}

constexpr int kJoinRed = 16384;  // LDS in which the waves' sums meet
// out^T = W_v^T o^T, 32 rows of one head at a time, o normalised in obar. The four waves take a quarter
// of the contraction each, o straight from global memory as operands, W_v's rows by direct copies
// once. A workgroup takes every tparts-th block of rows, and reads the next one's o beside this one's
// products: with one block per workgroup, each waited for W_v and o (300 rows, 128 heads: 72 us, so 46). Bound by
// the latency of those two reads with few rows, by reading o with many.
template <typename T, int DV, int NB, int NST, bool FIX>  // NB 32-column blocks of out; NST steps of 16 per wave; FIX: lse lacks qa_low2's share
__global__ __launch_bounds__(256) void join_kernel(PagedArgs a, int tparts) {
  constexpr int E = 16 / sizeof(T), CPR = 32 * NB / E;  // 16-byte chunks of a staged row
  typedef typename FragOf<T>::half quad;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  __shared__ float s_dot[2][4][32];
  f32x4* red = (f32x4*)smem;
  T* sw = (T*)(smem + kJoinRed);
  const int l = threadIdx.x & 63, n = l & 31, g = l >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  constexpr int VB = DV / (32 * NB);
  const int vb = blockIdx.x % VB, h = blockIdx.x / VB / tparts;
  const int dc = a.d_c, nch = dc * CPR, step = 32 * tparts;
  const int64_t ldw = (int64_t)a.H * (a.d_nope + DV);
  const T* wv = (const T*)a.w + (int64_t)h * (a.d_nope + DV) + a.d_nope + 32 * NB * vb;
  const bool fix = FIX && a.lse && vb == 0;
  const int32_t* before = a.sched + kSchedHeader;
  // step i of this wave: columns 16 (NST wave + i) + {4 g .. + 3, 8 + 4 g .. + 3}
  const int c0 = 16 * NST * wave + 4 * g;
  struct Row {
    bool seen;
    float fill;
  };
  auto row = [&](int t) {
    Row r = {false, 0.f};
    if (t < a.T) {
      r.seen = before[t] != before[t + 1];
      if (!r.seen && row_state(a, t).bad) r.fill = NAN;
    }
    return r;
  };
  f32x4 x[NST][2];
  quad y[FIX ? NST : 1][2];
  const T* lacks = (const T*)a.qa_low2;
  auto load = [&](int i, int t, const Row& r) {
    x[i][0] = x[i][1] = f32x4{r.fill, r.fill, r.fill, r.fill};
    if (r.seen && 16 * (NST * wave + i) < dc) {
      const int64_t th = (int64_t)t * a.H + h;
      const float* o = a.obar + th * dc + c0 + 16 * i;
      x[i][0] = *reinterpret_cast<const f32x4*>(o);
      x[i][1] = *reinterpret_cast<const f32x4*>(o + 8);
      if constexpr (FIX)
        if (fix) {
          const T* q = lacks + th * (dc + a.d_rope) + c0 + 16 * i;
          y[i][0] = *reinterpret_cast<const quad*>(q);
          y[i][1] = *reinterpret_cast<const quad*>(q + 8);
        }
    }
  };
  int t = blockIdx.x / VB % tparts * 32 + n;
  Row now = row(t), next = row(t + step);
#pragma unroll
  for (int i = 0; i < NST; ++i) load(i, t, now);
  for (int p0 = wave * 64; p0 < nch; p0 += 256) {
    const int r = (p0 + l) / CPR;
    int c = (p0 + l) % CPR;
    if constexpr (sizeof(T) == 2) c ^= swz<CPR>(r);
    g2lds16(wv + r * ldw + c * E, sw + p0 * E);
  }
  wait_vmem();
  lds_barrier();
  for (int turn = 0;; turn ^= 1) {
    const int64_t th = (int64_t)t * a.H + h;
    const bool more = t - n + step < a.T;
    const Row third = row(t + 2 * step);
    float lse = now.fill == 0.f ? -INFINITY : NAN;
    if (fix) {
      if (now.seen) lse = a.lse[th];
      float dot = 0.f;
      if constexpr (FIX)
        if (now.seen)
#pragma unroll
          for (int i = 0; i < NST; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (16 * (NST * wave + i) < dc) dot = __builtin_fmaf(x[i][e / 4][e % 4], to_f32(y[i][e / 4][e % 4]), dot);
      dot = wave_xor32_sum(dot);
      if (g == 0) s_dot[turn][wave][n] = dot;
    }
    f32x16 acc[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[b] = f32x16{};
#pragma unroll
    for (int i = 0; i < NST; ++i) {
      const int ks = NST * wave + i;
      if (16 * ks >= dc) continue;  // wave-uniform
      frag_t<T> hi, lo;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        hi[e] = to_elem<T>(x[i][e / 4][e % 4]);
        lo[e] = to_elem<T>(x[i][e / 4][e % 4] - to_f32(hi[e]));
      }
      if (more) load(i, t + step, next);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int ra = 16 * ks + 4 * g;
        frag_t<T> wf;
        if constexpr (sizeof(T) == 2) wf = swz_tr_frag<CPR>((const bf16*)sw, ra, ra + 8, 32 * b);
        else wf = TrRead<float>::get((const float*)sw, 32 * NB, ra, ra + 8, 32 * b);
        mma(acc[b], wf, hi);
        if constexpr (kTwo<T>) mma(acc[b], wf, lo);
      }
    }
    // the waves' sums, a block of columns at a time; each wave adds up a quarter
    T* o = (T*)a.out + th * DV + 32 * NB * vb + 4 * g;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      lds_barrier();  // the block before is read
#pragma unroll
      for (int rr = 0; rr < 4; ++rr)
        red[(wave * 4 + rr) * 64 + l] = f32x4{acc[b][4 * rr], acc[b][4 * rr + 1], acc[b][4 * rr + 2], acc[b][4 * rr + 3]};
      lds_barrier();
      f32x4 y = red[wave * 64 + l];
#pragma unroll
      for (int w = 1; w < 4; ++w) y += red[(w * 4 + wave) * 64 + l];
      quad z;
#pragma unroll
      for (int e = 0; e < 4; ++e) z[e] = to_elem<T>(y[e]);
      if (t < a.T) *reinterpret_cast<quad*>(o + 32 * b + 8 * wave) = z;
    }
    if (t < a.T && a.lse && vb == 0 && wave == 0 && g == 0 && (fix || !now.seen)) {
      const float(*d)[32] = s_dot[turn];
      if (fix && now.seen) lse += (((d[0][n] + d[1][n]) + d[2][n]) + d[3][n]) * a.scale_log2 * kLn2;
      a.lse[th] = lse;
    }
    if (!more) return;
    t += step;
    now = next;
    next = third;
  }
}

template <typename T, int DV, bool FIX, int NB>
void launch_join_product(const PagedArgs& a, hipStream_t st) {
  const size_t lds = kJoinRed + (size_t)a.d_c * 32 * NB * sizeof(T);
  const int64_t blocks = (int64_t)a.H * (DV / (32 * NB));
  const int tb = (a.T + 31) / 32, want = (int)((kCus * (160 * 1024 / lds) + blocks - 1) / blocks);  // what runs at once
  const int tparts = tb < want ? tb : want;
  const unsigned wgs = (unsigned)(blocks * tparts);
  if (a.d_c <= 128) join_kernel<T, DV, NB, 2, FIX><<<wgs, 256, lds, st>>>(a, tparts);
  else if (a.d_c <= 256) join_kernel<T, DV, NB, 4, FIX><<<wgs, 256, lds, st>>>(a, tparts);
  else if (a.d_c <= 512) join_kernel<T, DV, NB, 8, FIX><<<wgs, 256, lds, st>>>(a, tparts);
  else if constexpr (NB == 1 || 64 * NB == DV) join_kernel<T, DV, NB, 16, FIX><<<wgs, 256, lds, st>>>(a, tparts);
}

// The same for one row and head per workgroup, partials and all, in fp32: where there are no more of
// them than CUs. W_v's rows are on their way to registers (16 bytes of a row per thread, up to
// kVecRows rows) before the partials are known. 256 threads for small heads, else 1024.
constexpr int kVecRows = 16;
template <typename T, int DV, int NT, bool FIX>
__global__ __launch_bounds__(NT) void join_vec_kernel(PagedArgs a) {
  constexpr int E = 16 / sizeof(T), CPR = DV / E, SLICES = NT / CPR;  // columns of a thread; threads of a row
  typedef __attribute__((__vector_size__(16))) T chunk_t;
  __shared__ __attribute__((aligned(16))) unsigned char lds[24 * NT];
  __shared__ float s_o[1024], s_out[NT / 64][DV];
  const int tid = threadIdx.x, t = blockIdx.x / a.H, h = blockIdx.x % a.H, dc = a.d_c;
  const int64_t th = (int64_t)t * a.H + h, ldw = (int64_t)a.H * (a.d_nope + DV);
  const int v = tid % CPR * E, slice = tid / CPR;  // rows slice, slice + SLICES, ...
  const T* w = (const T*)a.w + (int64_t)h * (a.d_nope + DV) + a.d_nope + v;
  chunk_t wr[kVecRows];
#pragma unroll
  for (int i = 0; i < kVecRows; ++i)
    if (slice + i * SLICES < dc) wr[i] = *reinterpret_cast<const chunk_t*>(w + (slice + i * SLICES) * ldw);
  const RowParts r = parts_of(a, t);
  // what lse lacks, in the first wave
  float lack[2][8] = {};
  if (FIX && a.lse && tid < 64 && r.seen) {
    const T* q = (const T*)a.qa_low2 + th * (dc + a.d_rope);
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (8 * tid + 512 * k < dc) load8(q + 8 * tid + 512 * k, lack[k]);
  }
  const int quads = dc / 4, groups = NT / quads, group = tid / quads, c = tid % quads * 4;
  float lse = -INFINITY;
  if (r.split) {
    const Joined x = join_parts(a, r, h, c, group, groups, quads, group < groups, lds);
    if (group == 0) {
      const float inv = 1.f / x.l;
#pragma unroll
      for (int e = 0; e < 4; ++e) s_o[c + e] = x.o[e] * inv;
      lse = (x.m + fast_log2(x.l)) * kLn2;
    }
  } else if (group == 0) {
    f32x4 x = {r.fill, r.fill, r.fill, r.fill};
    if (r.seen) {
      x = *reinterpret_cast<const f32x4*>(a.obar + th * dc + c);
      if (a.lse) lse = a.lse[th];
    } else if (r.fill != 0.f) {
      lse = NAN;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) s_o[c + e] = x[e];
  }
  __syncthreads();
  if (a.lse && tid < 64) {
    float dot = 0.f;
    if (FIX && r.seen) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
        if (8 * tid + 512 * k < dc)
#pragma unroll
          for (int e = 0; e < 8; ++e) dot = __builtin_fmaf(s_o[8 * tid + 512 * k + e], lack[k][e], dot);
#pragma unroll
      for (int o = 32; o >= 1; o >>= 1) dot += __shfl_xor(dot, o);
    }
    if (tid == 0) a.lse[th] = lse + dot * a.scale_log2 * kLn2;
  }
  float y[E];
#pragma unroll
  for (int e = 0; e < E; ++e) y[e] = 0.f;
#pragma unroll
  for (int i = 0; i < kVecRows; ++i)
    if (slice + i * SLICES < dc)
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = __builtin_fmaf(s_o[slice + i * SLICES], to_f32(wr[i][e]), y[e]);
  for (int i = slice + kVecRows * SLICES; i < dc; i += SLICES) {
    const chunk_t x = *reinterpret_cast<const chunk_t*>(w + i * ldw);
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] = __builtin_fmaf(s_o[i], to_f32(x[e]), y[e]);
  }
  // the slices of a wave, then the waves, in order
#pragma unroll
  for (int o = CPR; o < 64; o <<= 1)
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] += __shfl_xor(y[e], o);
  if ((tid & 63) < CPR)
#pragma unroll
    for (int e = 0; e < E; ++e) s_out[tid / 64][v + e] = y[e];
  __syncthreads();
  if (tid < DV) {
    float out = 0.f;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) out += s_out[i][tid];
    ((T*)a.out)[th * DV + tid] = to_elem<T>(out);
  }
}

template <typename T, int DV, bool FIX>
void launch_join(const PagedArgs& a, hipStream_t st) {
  const int64_t pairs = (int64_t)a.T * a.H;
  // both in one launch where no workgroup would wait for another: 16 heads of one row 7.6 us (4.7 + 6.7 in two), 2
  // rows of 128 heads 23.6 (18.4 + 10.4). Small heads with 256 threads: 5.1 us, 8.9 with 1024 (8 rows, 4
  // heads, d_c = 64, fp32).
  if (pairs <= kCus) {
    if (a.d_c * DV <= 128 * 64) join_vec_kernel<T, DV, 256, FIX><<<(unsigned)pairs, 256, 0, st>>>(a);
    else join_vec_kernel<T, DV, 1024, FIX><<<(unsigned)pairs, 1024, 0, st>>>(a);
    return;
  }
  // one head per workgroup; eight where most rows cannot be shared, being more than the workers (300 rows, 128
  // heads: 24 us and 15; 61 rows 20 and 23)
  if (a.T > a.workers) combine_kernel<8><<<(unsigned)((int64_t)a.T * ((a.H + 7) / 8)), kCombineThreads, 0, st>>>(a);
  else combine_kernel<1><<<(unsigned)pairs, kCombineThreads, 0, st>>>(a);
  // all of out's columns in one workgroup, or half of them with d_c above 512 (o is then read once or twice: W_v's
  // rows of a head have to fit in LDS), where heads and rows alone fill half of the GPU (61 rows,
  // 128 heads: 16 us, 32 with a quarter per workgroup; 416 rows, d_c = 1024: 284 us with a quarter, so 163)
  constexpr int NB = DV / 32;
  if constexpr (sizeof(T) == 2 && NB > 1)
    if ((int64_t)a.H * ((a.T + 31) / 32) >= kCus / 2) {
      if (a.d_c <= 512) return launch_join_product<T, DV, FIX, NB>(a, st);
      return launch_join_product<T, DV, FIX, NB / 2>(a, st);
    }
  launch_join_product<T, DV, FIX, 1>(a, st);
}

template <typename T, int DN, bool Q8>
hipError_t launch_paged_t(const PagedArgs& a, hipStream_t st) {
  const int cblocks = (a.d_c + kAbsorbRows - 1) / kAbsorbRows;
  const int64_t blocks = (int64_t)a.H * cblocks;
  const int ttiles = (a.T + 31) / 32;
  const int want = (int)((4 * kCus + blocks - 1) / blocks), tparts = ttiles < want ? ttiles : want;
  absorb_kernel<T, DN, Q8><<<(unsigned)(a.T + 1 + blocks * tparts), 64 * kAbsorbWaves, max(absorb_lds<T, DN>(), layout_lds()), st>>>(
      a, cblocks, tparts);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int hb = (a.H + a.heads_per_wg - 1) / a.heads_per_wg;
  const unsigned wgs = (unsigned)(hb * a.workers);
  if constexpr (Q8) launch_paged_split_q8(a, hb, st);
  else if (a.wide) launch_paged_wide(a, hb, st);
  else if (a.d_c <= 128) split_kernel<T, 1><<<wgs, 256, 0, st>>>(a, hb);
  else if (a.d_c <= 256) split_kernel<T, 2><<<wgs, 256, 0, st>>>(a, hb);
  else if (a.d_c <= 512) split_kernel<T, 4><<<wgs, 256, 0, st>>>(a, hb);
  else split_kernel<T, 8><<<wgs, 256, 0, st>>>(a, hb);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  launch_join<T, DN, kTwo<T> && !Q8>(a, st);
  return hipGetLastError();
}

}  // namespace

template <typename T>
hipError_t launch_paged_attn(const PagedArgs& a, hipStream_t st) {
  if (a.d_nope == 128) return launch_paged_t<T, 128, false>(a, st);
  if (a.d_nope == 64) return launch_paged_t<T, 64, false>(a, st);
  return launch_paged_t<T, 32, false>(a, st);
}
template <typename T>
hipError_t launch_paged_attn_q8(const PagedArgs& a, hipStream_t st) {
  if (a.d_nope == 128) return launch_paged_t<T, 128, true>(a, st);
  if (a.d_nope == 64) return launch_paged_t<T, 64, true>(a, st);
  return launch_paged_t<T, 32, true>(a, st);
}

template hipError_t launch_paged_attn<bf16>(const PagedArgs&, hipStream_t);
template hipError_t launch_paged_attn<float>(const PagedArgs&, hipStream_t);
template hipError_t launch_paged_attn_q8<bf16>(const PagedArgs&, hipStream_t);
template hipError_t launch_paged_attn_q8<float>(const PagedArgs&, hipStream_t);

}  // namespace laga
