// Split attention over the paged cache: the general form (any width and type), which the wide kernel
// takes too where there are few tiles.
#pragma once
#include "paged_dev.hpp"

namespace laga {

// Attention over a worker's share of the tiles for 32 heads, by a workgroup of four waves, tiles of 32
// keys:
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
constexpr int kWindow = 512;  // page ids of a row held in LDS
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
  static constexpr int LDS = NS * TILE * (int)sizeof(T) + 4 * 4 * 64 * 16 + 4 * kWindow + 16;
};

// Worker w's share for heads h0 .. h0 + nh (nh <= 32); smem: SplitCfg::LDS bytes.
template <typename T, int ND>
__device__ __forceinline__ void split_shares(const PagedArgs& a, unsigned char* smem, int w, int h0, int nh, int per, int total) {
  using C = SplitCfg<T, ND>;
  constexpr int NS = C::NS, P = C::P, E = C::E;
  T* ring = (T*)smem;
  f32x4* s_part = (f32x4*)(smem + NS * C::TILE * sizeof(T));
  int32_t* s_page = (int32_t*)(s_part + 4 * 4 * 64);
  uint32_t* s_bad = (uint32_t*)(s_page + kWindow);

  const int l = threadIdx.x & 63, n = l & 31, g = l >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int W = a.d_c + a.d_rope;
  const int64_t start = (int64_t)w * per;
  if (start >= total) return;
  const int end = (int)min((int64_t)total, start + per);
  Share share = first_share(a, w);
  if (share.first >= end) return;  // (units of no tile)

  // copy j's lane: chunk c of the tile's row; and its place in a tile whose rows follow each other
  constexpr int NJ = (C::NI + 3) / 4;
  constexpr uint32_t kNoPlace = ~0u;
  auto chunk_of = [&](int j, int lane, int& row, int& c) {
    const int p = j * 64 + lane;
    row = p / P;
    c = p - row * P;
    if (C::NI * 64 > kTileKeys * P && row >= kTileKeys) row = 0, c = 0;
    if constexpr (sizeof(T) == 2) c ^= swz<24>(row);
  };
  auto place_of = [&](int jj, int lane) {
    int row, c;
    chunk_of(wave + 4 * jj, lane, row, c);
    return c * E < W ? (uint32_t)(row * W * (int)sizeof(T) + c * 16) : kNoPlace;
  };
  // (d_c above 512: formed anew for each copy, for want of registers to keep them in)
  uint32_t place[ND > 4 ? 1 : NJ];
  if constexpr (ND <= 4)
#pragma unroll
    for (int jj = 0; jj < NJ; ++jj) place[jj] = place_of(jj, l);

  for (int at = max((int)start, share.first);;) {
    const int t = share.t, row_first = share.first, row_end = share.end;
    const int it0 = at - row_first, it1 = min(end, row_end) - row_first;
    at = min(end, row_end);
    const RowState rs = {share.request, share.visible, false};
    const int32_t* pages = a.table + (int64_t)rs.request * a.width;

    // this wave's part of the queries: step i covers elements 16 (wave + 4 i) ..
    // (bf16: and the second parts, and the third of the band's one step)
    frag_t<T> qf[C::KS], ql[kTwo<T> ? C::KS : 1], q3 = frag_t<T>{};
    const int band = (wave - a.d_c / 16 & 3) + a.d_c / 16;
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
      if (kTwo<T> && 16 * band < W) q3 = *reinterpret_cast<const frag_t<T>*>((const T*)a.qa_low2 + q + 16 * band);
    }
    f32x16 oacc[ND];
#pragma unroll
    for (int i = 0; i < ND; ++i) oacc[i] = f32x16{};
    float m = -INFINITY, lsum = 0.f;

    int win = -1;  // first page of the window
    auto page_of = [&](int key) { return (int)((uint64_t)(uint32_t)key * a.page_magic >> a.page_shift); };
    // copies of tile `it` into stage st, after a barrier that freed it; of a tile in one page the
    // copies are only made ready, and issued in kSlots parts (at_once: here)
    const char* flat = nullptr;
    T* flat_to = nullptr;
    constexpr int kSlots = 8, kPerSlot = (NJ + kSlots - 1) / kSlots;
    auto some = [&](int slot) {
      if (!flat) return;
#pragma unroll
      for (int i = 0; i < kPerSlot; ++i) {
        const int jj = slot * kPerSlot + i, j = wave + 4 * jj;
        if (jj < NJ && (C::NI % 4 == 0 || j < C::NI)) {
          const uint32_t at = ND > 4 ? place_of(jj, fresh_lane()) : place[jj < NJ && ND <= 4 ? jj : 0];
          g2lds16(at == kNoPlace ? (const char*)kZeroRow : flat + at, flat_to + j * 64 * E);
        }
      }
    };
    auto fetch = [&](int it, int st, bool at_once) {
      const int k0 = it * kTileKeys, p0 = page_of(k0), o0 = k0 - p0 * a.page;
      if (win < 0 || page_of(min(k0 + kTileKeys, rs.visible) - 1) >= win + kWindow) {  // the same for every thread
        lds_barrier();
        win = p0;
        const int have = page_of(rs.visible - 1) + 1;
        for (int i = threadIdx.x; i < kWindow; i += 256) s_page[i] = win + i < have ? pages[win + i] : -1;
        lds_barrier();
      }
      // a tile that lies in one page: rows follow each other, places relative to the tile's are known
      const int pid0 = uniform(s_page[p0 - win]);
      if (k0 + kTileKeys <= rs.visible && o0 + kTileKeys <= a.page && (unsigned)pid0 < (unsigned)a.n_pages) {
        if (threadIdx.x == 0) s_bad[st] = 0;
        flat = (const char*)((const T*)a.cache + (int64_t)pid0 * a.page_stride + (int64_t)o0 * W);
        flat_to = ring + st * C::TILE;
        if (at_once)
#pragma unroll
          for (int i = 0; i < kSlots; ++i) some(i);
        return;
      }
      flat = nullptr;
      const int key = k0 + n;
      const bool live = key < rs.visible;
      const int pg = live ? page_of(key) : win, off = live ? key - pg * a.page : 0;
      const int pid = s_page[pg - win];
      const bool ok = live && (unsigned)pid < (unsigned)a.n_pages;
      const T* src = ok ? (const T*)a.cache + (int64_t)pid * a.page_stride + (int64_t)off * W : (const T*)kZeroRow;
      const uint32_t bad = (uint32_t)__ballot(live && !ok);
      if (threadIdx.x == 0) s_bad[st] = bad;
      const int lane = ND > 4 ? fresh_lane() : l;
      const uint32_t lo = (uint32_t)(uintptr_t)src, hi = (uint32_t)((uintptr_t)src >> 32);
#pragma unroll
      for (int jj = 0; jj < NJ; ++jj) {
        const int j = wave + 4 * jj;
        if (C::NI % 4 == 0 || j < C::NI) {
          int row, c;
          chunk_of(j, lane, row, c);
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
      if (it0 + i < it1) fetch(it0 + i, i, true);
    int st = 0;
    for (int it = it0; it < it1; ++it) {
      if constexpr (NS == 1) {
        lds_barrier();  // the tile before is read
        fetch(it, 0, true);
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
      {
        flat = nullptr;
        if (it + NS - 1 < it1) fetch(it + NS - 1, st == 0 ? NS - 1 : st - 1, false);
      }
      const T* tile = ring + st * C::TILE;
      // d_c above 512: addresses are formed anew in each tile, for want of registers to keep them in (64 requests
      // x 4000 keys, 16 heads, d_c = 1024: 94 us, 235 with them and what they spilled)
      const int tl = ND > 4 ? fresh_lane() : l, tn = tl & 31, tg = tl >> 5;

      f32x16 s = {};
      constexpr int KB = C::KS < 9 ? C::KS : C::KS > 9 ? 4 : 9;  // K fragments in flight
      frag_t<T> k[KB];
      auto k_frag = [&](int ks) {
        if constexpr (sizeof(T) == 2) return *reinterpret_cast<const frag_t<T>*>(tile + tn * P * E + (((2 * ks + tg) ^ swz<24>(tn)) * E));
        else return *reinterpret_cast<const frag_t<T>*>(tile + tn * P * E + 16 * ks + 8 * tg);
      };
#pragma unroll
      for (int i = 0; i < KB; ++i) k[i] = k_frag(wave + 4 * i);
      frag_t<T> kb;
      if constexpr (kTwo<T>) kb = k_frag(band);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < C::KS; ++i) {
        mma(s, k[i % KB], qf[i]);
        if constexpr (kTwo<T>) mma(s, k[i % KB], ql[i]);
        if (i + KB < C::KS) k[i % KB] = k_frag(wave + 4 * (i + KB));
        if (NS > 1 && i == C::KS / 3) some(0);
        if (NS > 1 && i == 2 * C::KS / 3) some(1);
      }
      if constexpr (kTwo<T>) mma(s, kb, q3);
      if (NS > 1) some(2);
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
      if (NS > 1) some(3);
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
      if (NS > 1) some(4);
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
      if (NS > 1) some(5);
      if (__ballot(bump)) {
#pragma unroll
        for (int i = 0; i < ND; ++i) oacc[i] *= alpha;
      }
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        if (NS > 1) some(6 + kk);
        const frag_t<T> pf = acc_to_frag<T>(s, kk);
        frag_t<T> pl;
        if constexpr (kTwo<T>) {
          f32x16 low;
#pragma unroll
          for (int e = 0; e < 8; ++e) low[8 * kk + e] = s[8 * kk + e] - to_f32(pf[e]);
          pl = acc_to_frag<T>(low, kk);
        }
        const int ra = 16 * kk + 4 * tg;
#pragma unroll
        for (int i = 0; i < ND; ++i) {
          const int c0 = 32 * (wave + 4 * i);
          frag_t<T> cf;
          if constexpr (sizeof(T) == 2) {
            const int sl = tl & 15, col = c0 + 16 * ((tl >> 4) & 1) + 4 * (sl & 3);
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
    if (at >= end) return;
    share = next_share(a, t, at);
    at = share.first;
    if (at >= end) return;
  }
}

}  // namespace laga
