// Attention of new tokens over a paged cache of latents, in the absorbed form: with head h's
// columns [W_k || W_v] of W_kv_b,
//
//   qa = W_k q_nope,  z_j = scale (qa . c_j + q_rope . k_j),  o = sum_j softmax(z)_j c_j,  out = W_v^T o
//
// so that a cached position is one row [c_j || k_j] that every head reads, and no per-head key
// or value exists. Three launches: the products qa and the turned q_rope (absorb_kernel), the
// attention split over the cache (split_kernel), and the join of split rows with the product
// by W_v (join_kernel). Bound by the cache's bytes for few heads (2 (2 d_c + d_rope) flop per
// head for each row of d_c + d_rope elements).
#include <math.h>
#include <stdlib.h>

#define LAGA_LDS_DMA_ASM 1
#include "common.hpp"
#include "paged_dev.hpp"
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

template <typename T, int DN>
__device__ void absorb_product(const PagedArgs& a, int blk, int cblocks, int tpart, int tparts) {
  constexpr int E = 16 / sizeof(T), CPR = DN / E, PO = kAbsorbRows + E;  // chunks of a row; pitch of the results
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  T* sw = (T*)smem;
  T* sq = sw + kAbsorbRows * DN;
  T* so = sq + 32 * DN;
  T* sl = so + 32 * PO;  // bf16: low halves
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
    for (int rr = 0; rr < 4; ++rr) {
      typename FragOf<T>::half v, low;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = to_elem<T>(acc[4 * rr + e]);
        low[e] = to_elem<T>(acc[4 * rr + e] - to_f32(v[e]));
      }
      const int at = n * PO + 32 * wave + 8 * rr + 4 * g;
      *reinterpret_cast<typename FragOf<T>::half*>(so + at) = v;
      if constexpr (kTwo<T>) *reinterpret_cast<typename FragOf<T>::half*>(sl + at) = low;
    }
    lds_barrier();
    for (int x = threadIdx.x; x < nt * (kAbsorbRows / E); x += 64 * kAbsorbWaves) {
      const int r = x / (kAbsorbRows / E), c = x % (kAbsorbRows / E) * E;
      if (c >= nc) continue;
      const int64_t at = ((int64_t)(t0 + r) * a.H + h) * W + c0 + c;
      *reinterpret_cast<chunk16*>((T*)a.qa + at) = *reinterpret_cast<const chunk16*>(so + r * PO + c);
      if constexpr (kTwo<T>)
        *reinterpret_cast<chunk16*>((T*)a.qa_lo + at) = *reinterpret_cast<const chunk16*>(sl + r * PO + c);
    }
    if (t0 + tparts * 32 < a.T) lds_barrier();  // q and the results are read
  }
}
template <typename T, int DN>
constexpr size_t absorb_lds() {
  return sizeof(T) * ((size_t)(kAbsorbRows + 32) * DN + (kTwo<T> ? 2 : 1) * 32 * (kAbsorbRows + 16 / sizeof(T)));
}

// q_rope of one token, every head: a thread keeps one pair's angle
template <typename T>
__device__ void absorb_band(const PagedArgs& a, int t) {
  const int pairs = a.d_rope / 2, i = threadIdx.x % pairs;
  const int W = a.d_c + a.d_rope, dqk = a.d_nope + a.d_rope;
  float cs = 1.f, sn = 0.f;
  if (a.rotate) rope_sincos(a.position_offset + a.position[t], rope_freq(i, a.d_rope, a.log2_base), cs, sn);
  for (int h = threadIdx.x / pairs; h < a.H; h += 64 * kAbsorbWaves / pairs) {
    const T* x = (const T*)a.q + ((int64_t)t * a.H + h) * dqk + a.d_nope + 2 * i;
    const int64_t at = ((int64_t)t * a.H + h) * W + a.d_c + 2 * i;
    const float x0 = to_f32(x[0]), x1 = to_f32(x[1]);
    const float y[2] = {x0 * cs - x1 * sn, x0 * sn + x1 * cs};
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const T v = to_elem<T>(y[e]);
      ((T*)a.qa)[at + e] = v;
      if constexpr (kTwo<T>) ((T*)a.qa_lo)[at + e] = to_elem<T>(y[e] - to_f32(v));
    }
  }
}

// Tiles before each row, tiles per worker, and the row in which each worker's share begins.
__device__ void lay_out_tiles(const PagedArgs& a) {
  constexpr int NT = 64 * kAbsorbWaves;
  __shared__ int sm[kAbsorbWaves];
  const int tid = threadIdx.x, l = tid & 63, wave = tid >> 6;
  int32_t* before = a.sched + kSchedHeader;
  int32_t* first_row = before + a.T + 1;
  int sum = 0;
  for (int base = 0; base < a.T; base += NT) {
    const int t = base + tid;
    int n = 0;
    if (t < a.T) n = tiles_of(row_state(a, t).visible);
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
    if (t < a.T) before[t] = b + inc - n;
  }
  const int per = tiles_per_worker(sum, a.workers, a.min_per);
  if (tid == 0) {
    before[a.T] = sum;
    a.sched[0] = per;
    a.sched[1] = sum;
  }
  __syncthreads();
  for (int w = tid; w < a.workers; w += NT) {
    const int64_t start = (int64_t)w * per;
    int lo = 0;
    if (start < sum) {
      int hi = a.T;  // last row whose tiles begin at or before start
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (before[mid] <= start) lo = mid; else hi = mid;
      }
    }
    first_row[w] = lo;
  }
}

template <typename T, int DN>
__global__ __launch_bounds__(64 * kAbsorbWaves) void absorb_kernel(PagedArgs a, int cblocks, int tparts) {
  // the few long jobs first
  const int others = a.T + 1, id = blockIdx.x;
  if (id == 0) lay_out_tiles(a);
  else if (id < others) absorb_band<T>(a, id - 1);
  else absorb_product<T, DN>(a, (id - others) / tparts, cblocks, (id - others) % tparts, tparts);
}

// ---------------------------------------------------------------- split attention
// One workgroup of four waves takes 32 heads of a worker's tiles of 32 keys:
//   S^T = K Q^T: the contraction over d_c + d_rope is dealt to the four waves (K fragments
//     from LDS, the wave's part of Q in registers), whose partial S^T meet in LDS, so that every
//     wave holds all of S^T and runs the same softmax, a lane per head;
//   O^T += C^T P^T: the columns of c are dealt to the waves in blocks of 32, P^T straight from
//     the S^T accumulators, C^T by transposing reads of the same LDS tile.
// So a wave reads each byte of the tile once per product and holds a quarter of Q and O.
// Tiles arrive by direct copies in a ring of NS stages. A key past the row's end, or whose page
// lies outside the pool, is copied from a row of zeros: whatever the cache holds there is never
// read; the first has probability zero, the second makes the row NaN.

// LDS rows of P 16-byte chunks: [c || k || padding]. bf16: chunk c of row r at c ^ swz<24>(r),
// conflict-free for both kinds of read at P % 16 == 8 (rows start half-way round the banks in
// turn, as 24-chunk rows do); fp32: an odd pitch.
template <typename T, int ND>
struct SplitCfg {
  static constexpr int E = 16 / sizeof(T);
  static constexpr int P = (128 * ND + 64) / E + (sizeof(T) == 4 ? 1 : 0);
  static constexpr int NI = (kTileKeys * P + 63) / 64;  // copies of 64 chunks per tile
  static constexpr int PER = NI / 4;                     // of each wave, at least
  static constexpr int TILE = NI * 64 * E;               // elements
  static constexpr int kMost = sizeof(T) == 2 && ND <= 2 ? 2 : 4;  // two stages where that lets more workgroups on a CU
  static constexpr int kRing = 140 * 1024 / (NI * 1024);
  static constexpr int NS = kRing < 1 ? 1 : kRing > kMost ? kMost : kRing;
  static constexpr int KS = 2 * ND + 1;                  // contraction steps of 16 per wave
};
constexpr int kWindow = 512;  // page ids of a row held in LDS

template <typename T, int ND>
__global__ __launch_bounds__(256, sizeof(T) == 2 && ND <= 2 ? 2 : 1) void split_kernel(PagedArgs a, int head_blocks) {
  using C = SplitCfg<T, ND>;
  constexpr int NS = C::NS, P = C::P, E = C::E;
  __shared__ __attribute__((aligned(16))) T ring[NS * C::TILE];
  __shared__ f32x4 s_part[4 * 4 * 64];
  __shared__ int32_t s_page[kWindow];
  __shared__ uint32_t s_bad[NS];

  const int l = threadIdx.x & 63, n = l & 31, g = l >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // the head blocks of a worker follow each other on one XCD: its L2 serves all but the first
  const int id = blockIdx.x, hb = id / 8 % head_blocks, w = id / (8 * head_blocks) * 8 + id % 8;
  const int h0 = hb * a.heads_per_wg, nh = min(a.heads_per_wg, a.H - h0);
  const int W = a.d_c + a.d_rope;
  const int per = a.sched[0], total = a.sched[1];
  const int64_t start = (int64_t)w * per;
  if (start >= total) return;
  const int end = (int)min((int64_t)total, start + per);
  const int32_t* before = a.sched + kSchedHeader;
  int t = before[a.T + 1 + w];

  for (int at = (int)start; at < end; ++t) {
    const int row_first = before[t], row_end = before[t + 1];
    if (row_end <= at) continue;
    const int it0 = at - row_first, it1 = min(end, row_end) - row_first;
    at = min(end, row_end);
    const RowState rs = row_state(a, t);
    const int32_t* pages = a.table + (int64_t)rs.request * a.width;

    // this wave's part of the queries: step i covers elements 16 (wave + 4 i) ..
    frag_t<T> qf[C::KS], ql[kTwo<T> ? C::KS : 1];
    {
      const int64_t q = ((int64_t)t * a.H + h0 + min(n, nh - 1)) * W + 8 * g;
#pragma unroll
      for (int i = 0; i < C::KS; ++i) {
        const int c = 16 * (wave + 4 * i);
        qf[i] = frag_t<T>{};
        if (c < W) qf[i] = *reinterpret_cast<const frag_t<T>*>((const T*)a.qa + q + c);
        if constexpr (kTwo<T>) {
          ql[i] = frag_t<T>{};
          if (c < W) ql[i] = *reinterpret_cast<const frag_t<T>*>((const T*)a.qa_lo + q + c);
        }
      }
    }
    f32x16 oacc[ND];
#pragma unroll
    for (int i = 0; i < ND; ++i) oacc[i] = f32x16{};
    float m = -INFINITY, lsum = 0.f;

    int win = -1;  // first page of the window
    auto page_of = [&](int key) { return (int)((uint64_t)(uint32_t)key * a.page_magic >> a.page_shift); };
    // copies of tile `it` into stage st, after a barrier that freed it
    auto fetch = [&](int it, int st) {
      const int k0 = it * kTileKeys, last = page_of(min(k0 + kTileKeys, rs.visible) - 1);
      if (win < 0 || last >= win + kWindow) {  // the same for every thread
        lds_barrier();
        win = page_of(k0);
        const int have = page_of(rs.visible - 1) + 1;
        for (int i = threadIdx.x; i < kWindow; i += 256) s_page[i] = win + i < have ? pages[win + i] : -1;
        lds_barrier();
      }
      const int key = k0 + n;
      const bool live = key < rs.visible;
      const int pg = live ? page_of(key) : win, off = live ? key - pg * a.page : 0;
      const int pid = s_page[pg - win];
      const bool ok = live && (unsigned)pid < (unsigned)a.n_pages;
      const T* src = ok ? (const T*)a.cache + (int64_t)pid * a.page_stride + (int64_t)off * W : (const T*)kZeroRow;
      const uint32_t bad = (uint32_t)__ballot(live && !ok);
      if (threadIdx.x == 0) s_bad[st] = bad;
      const uint32_t lo = (uint32_t)(uintptr_t)src, hi = (uint32_t)((uintptr_t)src >> 32);
#pragma unroll
      for (int jj = 0; jj < (C::NI + 3) / 4; ++jj) {
        const int j = wave + 4 * jj;
        if (C::NI % 4 == 0 || j < C::NI) {
          const int p = j * 64 + l;
          int row = p / P, c = p - row * P;
          if (C::NI * 64 > kTileKeys * P && row >= kTileKeys) row = 0, c = 0;
          if constexpr (sizeof(T) == 2) c ^= swz<24>(row);
          const uintptr_t base = (uintptr_t)(uint32_t)__shfl((int)lo, row) |
                                 ((uintptr_t)(uint32_t)__shfl((int)hi, row) << 32);
          const unsigned char* from = c * E < W ? (const unsigned char*)base : kZeroRow;
          g2lds16(from + c * 16, ring + st * C::TILE + j * 64 * E);
        }
      }
    };

    lds_barrier();  // the tiles and pages of the row before are read
#pragma unroll
    for (int i = 0; i < NS - 1; ++i)
      if (it0 + i < it1) fetch(it0 + i, i);
    int st = 0;
    for (int it = it0; it < it1; ++it) {
      if constexpr (NS == 1) {
        lds_barrier();  // the tile before is read
        fetch(it, 0);
        wait_vmem();
      } else {
        // tile `it` has landed: only the tiles issued after it may be in flight
        if (it + 1 < it1 && NS >= 3) {
          if (it + 2 < it1 && NS >= 4) wait_vmem_le<2 * C::PER>();
          else wait_vmem_le<C::PER>();
        } else {
          wait_vmem();
        }
      }
      lds_barrier();  // ... every wave's copies, and the stage before is read
      if constexpr (NS > 1)
        if (it + NS - 1 < it1) fetch(it + NS - 1, st == 0 ? NS - 1 : st - 1);
      const T* tile = ring + st * C::TILE;

      f32x16 s = {};
#pragma unroll
      for (int i = 0; i < C::KS; ++i) {
        const int ks = wave + 4 * i;
        frag_t<T> k;
        if constexpr (sizeof(T) == 2) k = *reinterpret_cast<const frag_t<T>*>(tile + n * P * E + (((2 * ks + g) ^ swz<24>(n)) * E));
        else k = *reinterpret_cast<const frag_t<T>*>(tile + n * P * E + 16 * ks + 8 * g);
        mma(s, k, qf[i]);
        if constexpr (kTwo<T>) mma(s, k, ql[i]);
      }
#pragma unroll
      for (int rr = 0; rr < 4; ++rr)
        s_part[(wave * 4 + rr) * 64 + l] = f32x4{s[4 * rr], s[4 * rr + 1], s[4 * rr + 2], s[4 * rr + 3]};
      lds_barrier();
#pragma unroll
      for (int rr = 0; rr < 4; ++rr) {
        f32x4 v = s_part[rr * 64 + l];
#pragma unroll
        for (int u = 1; u < 4; ++u) v += s_part[(u * 4 + rr) * 64 + l];
#pragma unroll
        for (int e = 0; e < 4; ++e) s[4 * rr + e] = v[e];
      }
      const int lim = rs.visible - it * kTileKeys - 4 * g;
      const uint32_t bad = s_bad[st];
      if (lim + 4 * g < kTileKeys || bad) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int k = (r >> 2) * 8 + (r & 3);
          s[r] = k < lim ? (bad >> (k + 4 * g) & 1 ? NAN : s[r]) : -INFINITY;
        }
      }
      // online softmax in base 2, the maximum raised only past a margin (kRescaleLog2)
      float mraw = -INFINITY;
#pragma unroll
      for (int r = 0; r < 16; ++r) mraw = fmaxf(mraw, s[r]);
      const float m_new = fmaxf(m, wave_xor32_max(mraw) * a.scale_log2);
      const bool bump = m_new > m + kRescaleLog2;
      const float alpha = bump ? fast_exp2(m - m_new) : 1.f;
      m = bump ? m_new : m;
      const float m_use = m == -INFINITY ? 0.f : m;
      float ps = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[r] = fast_exp2(__builtin_fmaf(s[r], a.scale_log2, -m_use));
        ps += s[r];
      }
      lsum = lsum * alpha + ps;
      if (__ballot(bump)) {
#pragma unroll
        for (int i = 0; i < ND; ++i) oacc[i] *= alpha;
      }
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        const frag_t<T> pf = acc_to_frag<T>(s, kk);
        frag_t<T> pl;
        if constexpr (kTwo<T>) {
          f32x16 low;
#pragma unroll
          for (int e = 0; e < 8; ++e) low[8 * kk + e] = s[8 * kk + e] - to_f32(pf[e]);
          pl = acc_to_frag<T>(low, kk);
        }
        const int ra = 16 * kk + 4 * g;
#pragma unroll
        for (int i = 0; i < ND; ++i) {
          const int c0 = 32 * (wave + 4 * i);
          frag_t<T> cf;
          if constexpr (sizeof(T) == 2) {
            const int sl = l & 15, col = c0 + 16 * ((l >> 4) & 1) + 4 * (sl & 3);
            const int r0 = ra + (sl >> 2), r1 = r0 + 8;
            typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
            const bf16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
                (lds_bf16x4*)(tile + r0 * P * E + (((col / E) ^ swz<24>(r0)) * E) + col % E));
            const bf16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
                (lds_bf16x4*)(tile + r1 * P * E + (((col / E) ^ swz<24>(r1)) * E) + col % E));
            cf = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
          } else {
            cf = TrRead<float>::get((const float*)tile, P * E, ra, ra + 8, c0);
          }
          mma(oacc[i], cf, pf);
          if constexpr (kTwo<T>) mma(oacc[i], cf, pl);
        }
      }
      st = st + 1 == NS ? 0 : st + 1;
    }

    // lane: head n, columns 32 (wave + 4 i) + 8 (r / 4) + 4 g + r % 4
    const float ltot = wave_xor32_sum(lsum);
    const bool whole = it0 == 0 && it1 == row_end - row_first;
    const int h = h0 + n;
    if (n >= nh) {
      // a lane of padding
    } else if (whole) {
      const float inv = 1.f / ltot;
      float* o = a.obar + ((int64_t)t * a.H + h) * a.d_c + 4 * g;
#pragma unroll
      for (int i = 0; i < ND; ++i)
        if (32 * (wave + 4 * i) < a.d_c)
#pragma unroll
          for (int rr = 0; rr < 4; ++rr)
            *reinterpret_cast<f32x4*>(o + 32 * (wave + 4 * i) + 8 * rr) =
                f32x4{oacc[i][4 * rr] * inv, oacc[i][4 * rr + 1] * inv, oacc[i][4 * rr + 2] * inv,
                      oacc[i][4 * rr + 3] * inv};
      if (wave == 0 && g == 0 && a.lse) a.lse[(int64_t)t * a.H + h] = (m + fast_log2(ltot)) * kLn2;
    } else {
      const int64_t place = (int64_t)partial_place(w, per, row_first) * a.H + h;
      float* o = a.part_o + place * a.d_c + 4 * g;
#pragma unroll
      for (int i = 0; i < ND; ++i)
        if (32 * (wave + 4 * i) < a.d_c)
#pragma unroll
          for (int rr = 0; rr < 4; ++rr)
            *reinterpret_cast<f32x4*>(o + 32 * (wave + 4 * i) + 8 * rr) =
                f32x4{oacc[i][4 * rr], oacc[i][4 * rr + 1], oacc[i][4 * rr + 2], oacc[i][4 * rr + 3]};
      if (wave == 0 && g == 0) {
        a.part_ml[2 * place] = m;
        a.part_ml[2 * place + 1] = ltot;
      }
    }
  }
}

// ---------------------------------------------------------------- join
// out^T = W_v^T o^T for some rows of one head. The four waves take a quarter of the contraction
// each; a lane's column of o^T is one row's partials j, j + SUB, ... (SUB lanes share a row,
// rows of the 32 columns: 32 / SUB), weighted by exp2(m - max m) / sum and added up in registers; as the
// product is linear, the SUB columns are added after it. So one row split over all workers has
// its partials read by 32 lanes at once, and a batch of whole rows keeps 32 rows per product.
// W_v's rows arrive by direct copies meanwhile. Bound by the latency of those two reads.
template <typename T, int DV, int NB, int NST>  // NB 32-column blocks of out; NST steps of 16 per wave
__global__ __launch_bounds__(256) void join_kernel(PagedArgs a, int sub_log2, int tblocks, int joined) {
  constexpr int E = 16 / sizeof(T), CPR = 32 * NB / E;  // 16-byte chunks of a staged row
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  __shared__ float s_dot[4][32];
  T* sw = (T*)smem;
  const int l = threadIdx.x & 63, n = l & 31, g = l >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int sub = 1 << sub_log2, j = n & (sub - 1);
  constexpr int VB = DV / (32 * NB);
  const int vb = blockIdx.x % VB, h = blockIdx.x / VB / tblocks;
  const int t0 = blockIdx.x / VB % tblocks * (32 >> sub_log2), t = t0 + (n >> sub_log2);
  const int dc = a.d_c, nch = dc * CPR;
  const int64_t ldw = (int64_t)a.H * (a.d_nope + DV);
  const T* wv = (const T*)a.w + (int64_t)h * (a.d_nope + DV) + a.d_nope + 32 * NB * vb;
  for (int p0 = wave * 64; p0 < nch; p0 += 256) {
    const int r = (p0 + l) / CPR;
    int c = (p0 + l) % CPR;
    if constexpr (sizeof(T) == 2) c ^= swz<CPR>(r);
    g2lds16(wv + r * ldw + c * E, sw + p0 * E);
  }

  // this lane's share of its row's partials
  const int32_t* before = a.sched + kSchedHeader;
  const int per = a.sched[0];
  int first = 0, last = 0, w0 = 0;  // its partials: workers first, first + sub, .. < last
  bool whole = false;
  float fill = 0.f;
  float lse = -INFINITY;
  if (t < a.T) {
    first = before[t];
    last = before[t + 1];
    if (first == last) {
      if (row_state(a, t).bad) fill = lse = NAN;
      last = 0;
      w0 = 0;
    } else {
      w0 = first / per;
      last = (last - 1) / per + 1;
      if (joined) last = w0 + 1;
      whole = last == w0 + 1;
    }
  }
  const int row_first = first;
  if (whole && a.lse) lse = a.lse[(int64_t)t * a.H + h];

  // step i of this wave: columns 16 (NST wave + i) + {4 g .. + 3, 8 + 4 g .. + 3}
  float v[NST][8];
#pragma unroll
  for (int i = 0; i < NST; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] = j == 0 ? fill : 0.f;
  const int c0 = 16 * NST * wave + 4 * g;
  // this lane's partials under their own running maximum: nothing waits for another lane's
  float mx = -INFINITY, sum = 0.f;
  for (int w = w0 + j; w < last; w += sub) {
    const int64_t p = (int64_t)partial_place(w, per, row_first) * a.H + h;
    const float* o = whole ? a.obar + ((int64_t)t * a.H + h) * dc : a.part_o + p * dc;
    f32x4 x[NST], y[NST];
#pragma unroll
    for (int i = 0; i < NST; ++i) {
      if (16 * (NST * wave + i) >= dc) continue;  // wave-uniform
      x[i] = *reinterpret_cast<const f32x4*>(o + c0 + 16 * i);
      y[i] = *reinterpret_cast<const f32x4*>(o + c0 + 16 * i + 8);
    }
    float f = 1.f, old = 1.f;
    if (!whole) {
      const float m = a.part_ml[2 * p], l = a.part_ml[2 * p + 1], m_new = fmaxf(mx, m);
      const float m_use = m_new == -INFINITY ? 0.f : m_new;
      f = fast_exp2(m - m_use);
      old = mx == -INFINITY ? 0.f : fast_exp2(mx - m_use);
      mx = m_new;
      sum = __builtin_fmaf(sum, old, f * l);
    }
#pragma unroll
    for (int i = 0; i < NST; ++i) {
      if (16 * (NST * wave + i) >= dc) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[i][e] = __builtin_fmaf(f, x[i][e], v[i][e] * old);
        v[i][4 + e] = __builtin_fmaf(f, y[i][e], v[i][4 + e] * old);
      }
    }
  }
  // and brought to the row's
  if (last > 0 && !whole) {  // (the same for the lanes of a row)
    float all = mx;
    for (int o = sub >> 1; o > 0; o >>= 1) all = fmaxf(all, __shfl_xor(all, o));
    const float m_use = all == -INFINITY ? 0.f : all;
    float f = mx == -INFINITY ? 0.f : fast_exp2(mx - m_use);
    sum *= f;
    for (int o = sub >> 1; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    lse = (all + fast_log2(sum)) * kLn2;
    f /= sum;
#pragma unroll
    for (int i = 0; i < NST; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] *= f;
  }
  if (a.lse && a.lse_fix && vb == 0) {
    float dot = 0.f;
    if (t < a.T) {
      const T* q = (const T*)a.qa_lo + ((int64_t)t * a.H + h) * (dc + a.d_rope) + c0;
#pragma unroll
      for (int i = 0; i < NST; ++i) {
        if (16 * (NST * wave + i) >= dc) continue;
        typedef typename FragOf<T>::half half4;
        const half4 x = *reinterpret_cast<const half4*>(q + 16 * i), y = *reinterpret_cast<const half4*>(q + 16 * i + 8);
#pragma unroll
        for (int e = 0; e < 4; ++e) dot += v[i][e] * to_f32(x[e]) + v[i][4 + e] * to_f32(y[e]);
      }
    }
    dot = wave_xor32_sum(dot);
    for (int o = sub >> 1; o > 0; o >>= 1) dot += __shfl_xor(dot, o);
    if (g == 0) s_dot[wave][n] = dot;
  }

  wait_vmem();
  lds_barrier();
  f32x16 acc[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) acc[b] = f32x16{};
#pragma unroll
  for (int i = 0; i < NST; ++i) {
    const int ks = NST * wave + i;
    if (16 * ks >= dc) continue;
    frag_t<T> hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      hi[e] = to_elem<T>(v[i][e]);
      lo[e] = to_elem<T>(v[i][e] - to_f32(hi[e]));
    }
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
  for (int o = sub >> 1; o > 0; o >>= 1)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[b][r] += __shfl_xor(acc[b][r], o);
  lds_barrier();  // W_v is read
  f32x4* red = (f32x4*)smem;
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int rr = 0; rr < 4; ++rr)
      red[((wave * NB + b) * 4 + rr) * 64 + l] = f32x4{acc[b][4 * rr], acc[b][4 * rr + 1], acc[b][4 * rr + 2], acc[b][4 * rr + 3]};
  lds_barrier();
  if (a.lse && vb == 0 && wave == 0 && g == 0 && j == 0 && t < a.T) {
    if (a.lse_fix)
      lse += (((s_dot[0][n] + s_dot[1][n]) + s_dot[2][n]) + s_dot[3][n]) * a.scale_log2 * kLn2;
    if (a.lse_fix || !whole) a.lse[(int64_t)t * a.H + h] = lse;
  }
  // 4 NB groups of four columns per lane, dealt to the waves
  if (t >= a.T || j != 0) return;
  T* o = (T*)a.out + ((int64_t)t * a.H + h) * DV + 32 * NB * vb + 4 * g;
#pragma unroll
  for (int x = 0; x < NB; ++x) {
    const int i = wave + 4 * x, b = i / 4, rr = i % 4;
    f32x4 y = red[(b * 4 + rr) * 64 + l];
#pragma unroll
    for (int u = 1; u < 4; ++u) y += red[((u * NB + b) * 4 + rr) * 64 + l];
    typename FragOf<T>::half z;
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = to_elem<T>(y[e]);
    *reinterpret_cast<typename FragOf<T>::half*>(o + 32 * b + 8 * rr) = z;
  }
}

// Rows that several workers share, put together in obar: a thread per four columns of a row's
// head adds its partials up in order.
__global__ __launch_bounds__(256) void combine_kernel(PagedArgs a) {
  const int quads = a.d_c / 4;
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x, th = x / quads;
  const int c = (int)(x % quads) * 4;
  const int t = (int)(th / a.H), h = (int)(th % a.H);
  if (t >= a.T) return;
  const int32_t* before = a.sched + kSchedHeader;
  const int per = a.sched[0], first = before[t], end = before[t + 1];
  if (first == end) return;
  const int w0 = first / per, w1 = (end - 1) / per;
  if (w0 == w1) return;
  float mx = -INFINITY, sum = 0.f;
  f32x4 v = {};
#pragma unroll 8
  for (int w = w0; w <= w1; ++w) {
    const int64_t p = (int64_t)partial_place(w, per, first) * a.H + h;
    const f32x4 o = *reinterpret_cast<const f32x4*>(a.part_o + p * a.d_c + c);
    const float m = a.part_ml[2 * p], l = a.part_ml[2 * p + 1], m_new = fmaxf(mx, m);
    const float m_use = m_new == -INFINITY ? 0.f : m_new;
    const float f = fast_exp2(m - m_use), old = mx == -INFINITY ? 0.f : fast_exp2(mx - m_use);
    mx = m_new;
    sum = __builtin_fmaf(sum, old, f * l);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(f, o[e], v[e] * old);
  }
  const float inv = 1.f / sum;
  *reinterpret_cast<f32x4*>(a.obar + th * a.d_c + c) = f32x4{v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
  if (c == 0 && a.lse) a.lse[th] = (mx + fast_log2(sum)) * kLn2;
}

// Lanes per row: as many as leave 32 / SUB >= T rows, and more while the launch is small and a
// row may have that many partials.
template <typename T, int DV, int NB>
hipError_t launch_join(const PagedArgs& a, bool joined, hipStream_t st) {
  int sl = 0;
  while (!joined && sl < 5 && (a.T << sl) <= 16) ++sl;
  auto blocks = [&] { return (int)(((int64_t)a.T + (32 >> sl) - 1) / (32 >> sl)); };
  while (!joined && sl < 5 && (int64_t)a.H * (DV / (32 * NB)) * blocks() < 2 * kCus && ((int64_t)a.T << sl) < a.workers) ++sl;
  const unsigned wgs = (unsigned)((int64_t)a.H * (DV / (32 * NB)) * blocks());
  const size_t w = (size_t)a.d_c * 32 * NB * sizeof(T), red = (size_t)NB * 16384, lds = w > red ? w : red;
  const int tb = blocks();
  if (a.d_c <= 128) join_kernel<T, DV, NB, 2><<<wgs, 256, lds, st>>>(a, sl, tb, joined);
  else if (a.d_c <= 256) join_kernel<T, DV, NB, 4><<<wgs, 256, lds, st>>>(a, sl, tb, joined);
  else if (a.d_c <= 512) join_kernel<T, DV, NB, 8><<<wgs, 256, lds, st>>>(a, sl, tb, joined);
  else join_kernel<T, DV, NB, 16><<<wgs, 256, lds, st>>>(a, sl, tb, joined);
  return hipGetLastError();
}

template <typename T, int DN>
hipError_t launch_paged_t(const PagedArgs& a, hipStream_t st) {
  const int cblocks = (a.d_c + kAbsorbRows - 1) / kAbsorbRows;
  const int64_t blocks = (int64_t)a.H * cblocks;
  const int ttiles = (a.T + 31) / 32;
  const int want = (int)((4 * kCus + blocks - 1) / blocks), tparts = ttiles < want ? ttiles : want;
  absorb_kernel<T, DN><<<(unsigned)(a.T + 1 + blocks * tparts), 64 * kAbsorbWaves, absorb_lds<T, DN>(), st>>>(
      a, cblocks, tparts);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int hb = (a.H + a.heads_per_wg - 1) / a.heads_per_wg;
  const unsigned wgs = (unsigned)(hb * a.workers);
  if (a.lse_fix) launch_paged_wide(a, hb, st);
  else if (a.d_c <= 128) split_kernel<T, 1><<<wgs, 256, 0, st>>>(a, hb);
  else if (a.d_c <= 256) split_kernel<T, 2><<<wgs, 256, 0, st>>>(a, hb);
  else if (a.d_c <= 512) split_kernel<T, 4><<<wgs, 256, 0, st>>>(a, hb);
  else split_kernel<T, 8><<<wgs, 256, 0, st>>>(a, hb);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  // all of out's columns in one workgroup where W_v's rows of a head fit in LDS beside another workgroup's
  // (o is then read once), and by 32 where the launch would be small
  constexpr int NB = DN / 32;
  const bool joined = getenv("JOINED") != nullptr;
  if (joined) combine_kernel<<<(unsigned)(((int64_t)a.T * a.H * a.d_c / 4 + 255) / 256), 256, 0, st>>>(a);
  if (sizeof(T) == 2 && NB > 1 && a.d_c <= 512 && (int64_t)a.H * ((a.T + 31) / 32) >= kCus / 2)
    return launch_join<T, DN, NB>(a, joined, st);
  return launch_join<T, DN, 1>(a, joined, st);
}

}  // namespace

template <typename T>
hipError_t launch_paged_attn(const PagedArgs& a, hipStream_t st) {
  if (a.d_nope == 128) return launch_paged_t<T, 128>(a, st);
  if (a.d_nope == 64) return launch_paged_t<T, 64>(a, st);
  return launch_paged_t<T, 32>(a, st);
}

template hipError_t launch_paged_attn<bf16>(const PagedArgs&, hipStream_t);
template hipError_t launch_paged_attn<float>(const PagedArgs&, hipStream_t);

}  // namespace laga
