// Split attention over the paged cache for bf16 with d_c = 512 and d_rope = 64: up to 64 heads share a tile that is
// read from memory once, and a tile's scores are formed beside the softmax of the tile before.
// (paged_split.hpp has the form for any width.)
#define LAGA_LDS_DMA_ASM 1
#include "paged_split.hpp"

namespace laga {
namespace {

// A workgroup's four waves are HG groups of 32 heads x NP = 4 / HG parts. The waves of a group divide both
// products among them, and each holds its part of Q, three bf16 parts of each value, and of O, in registers:
//   S^T = K Q^T: every NP-th step of the contraction over 512 + 64; the partial sums meet in LDS,
//     and each wave has all of S^T for the softmax, a lane per head;
//   O^T += C^T P^T: every NP-th block of 32 columns.
// Tiles of 32 keys arrive by direct copies in a ring of three. A step forms tile i + 1's scores beside tile i's
// softmax and the copies of tile i + 2, then multiplies by tile i; its one barrier, before the last of these
// products, orders copies, partial scores and the reads of both. A lone wave per SIMD hides about six
// instructions behind a product, so what goes beside which is laid out by hand.
constexpr int kDc = 512, kDr = 64, kRow = kDc + kDr;
constexpr int kMain = kTileKeys * kDc, kBand = kTileKeys * kDr, kTile = kMain + kBand;  // elements
constexpr int kStages = 3;
constexpr int kPages = 128;  // page ids of a row that a wave keeps in LDS
// The softmax's reference is the maximum of the share's first tile and stays, so that no sum is ever rescaled
// (O would have to leave the accumulation registers for it): bf16 and fp32 hold 2^kHead as
// they hold 1, and probabilities, sums and their parts keep their precision. Where a later tile's sum passes it, or
// the first tile has no maximum, the row's share is swept again, for its maximum and then with it.
constexpr float kHead = 64.f;

// A product of the chain S^T. Written out, because the parts of Q are to stay where they are, the first in ordinary
// registers and the others in accumulation registers; scores_done waits until the chain's last is written.
__device__ __forceinline__ void score_step(f32x16& s, const bf16x8& k, const bf16x8& q, bool first) {
  if (first) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(k), "v"(q));
  else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(k), "v"(q));
}
__device__ __forceinline__ void score_step_low(f32x16& s, const bf16x8& k, const bf16x8& q) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(k), "a"(q));
}
__device__ __forceinline__ void scores_done(f32x16& s) { asm volatile("s_nop 15\n\ts_nop 3" : "+v"(s)); }

// A direct copy of 1 KB to LDS byte address to + at. (A base that a vector instruction wrote may be read five wait
// states after it: four are here, and between the two the caller has a written-out instruction, too.)
template <bool NT>
__device__ __forceinline__ void copy_row(const void* base, uint32_t off, uint32_t to, int at) {
  if constexpr (NT)
    asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 2\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(off), "s"(base), "s"(to), "i"(at)
                 : "memory", "m0", "scc");
  else
    asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 2\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(to), "i"(at)
                 : "memory", "m0", "scc");
}
template <bool NT>
__device__ __forceinline__ void copy_lanes(const void* g, uint32_t to, int at) {
  if constexpr (NT)
    asm volatile("s_add_u32 m0, %1, %2\n\ts_nop 1\n\tglobal_load_lds_dwordx4 %0, off nt" ::"v"(g), "s"(to), "i"(at)
                 : "memory", "m0", "scc");
  else
    asm volatile("s_add_u32 m0, %1, %2\n\ts_nop 1\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(g), "s"(to), "i"(at)
                 : "memory", "m0", "scc");
}

// Computed here, not where it is read.
template <typename V>
__device__ __forceinline__ V here(V x) {
  asm volatile("" : "+v"(x));
  return x;
}

typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}
template <typename V>
__device__ __forceinline__ V lds_at(uint32_t address) {
  return *(__attribute__((address_space(3))) const V*)(uintptr_t)address;
}

// The share of worker w, for heads h0 .. h0 + 64 (HG = 2) or 32, below hb1. NT: see wide_kernel.
constexpr int kSums = 2 * 4 * 4 * 64;  // partial scores of two tiles, in f32x4
constexpr int kLds = kStages * kTile * 2 + kSums * 16;
template <int HG, bool NT>
__device__ __forceinline__ void wide_shares(const PagedArgs& a, unsigned char* smem, int32_t (*s_page)[kPages], int* s_high, int w,
                                            int hb0, int hb1, int per, int total) {
  static_assert(HG == 1 || HG == 2);
  constexpr int NP = 4 / HG;
  constexpr int KS = kRow / 16 / NP, KC = kDc / 16 / NP;  // steps of a wave; of them over the latent
  constexpr int NB = kDc / 32 / NP;                       // blocks of columns of a wave
  f32x4* sums = (f32x4*)(smem + kStages * kTile * 2);

  const int l = threadIdx.x & 63, n = l & 31, g = l >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hg = wave % HG, part = wave / HG;
  const int h0 = hb0 + 32 * hg, nh = min(32, hb1 - h0);  // nh <= 0: this wave's results are not stored
  const int64_t start = (int64_t)w * per;
  if (start >= total) return;
  const int end = (int)min((int64_t)total, start + per);
  int32_t* win_ids = s_page[wave];

  // Chunk c of a tile's row r is at c ^ swz<16>(r) (c part; c ^ swz<8>(r) in the band). Of a tile at LDS address x, this
  // lane reads the fragment of this wave's step i in row n at x + (k ^ 32 (NP i % 8)) + 256 (NP i / 8), of
  // the band's step i at x + (b ^ 32 NP i), and for the transposing reads of its column block i, rows vr
  // and vr + 8, at x + (v ^ 64 (NP i % 4)) + 256 (NP i / 4) and likewise v8. (x is a multiple of 256.)
  const uint32_t ring = lds_address(smem);
  uint32_t at_k, at_b, at_v, at_v8, at_copy, at_band;
  {
    const int sl = l & 15, vr = 4 * g + (sl >> 2), vc = 2 * ((l >> 4) & 1) + ((sl & 3) >> 1);
    at_k = 2 * n * kDc + (((g + 2 * part) ^ swz<16>(n)) * 16);
    at_b = 2 * (kMain + n * kDr) + (((g + 2 * part) ^ swz<8>(n)) * 16);
    at_v = 2 * vr * kDc + (((vc + 4 * part) ^ swz<16>(vr)) * 16) + 8 * (sl & 1);
    at_v8 = 2 * (vr + 8) * kDc + (((vc + 4 * part) ^ swz<16>(vr + 8)) * 16) + 8 * (sl & 1);
    at_copy = (l ^ swz<16>(wave)) * 16;
    at_band = 2 * kDc + ((l & 7) ^ swz<8>(8 * wave + (l >> 3))) * 16;
  }

  Share share = first_share(a, w);
  if (share.first >= end) return;  // (units of no tile)
  for (int at = max((int)start, share.first);;) {
    const int t = share.t, row_first = share.first, row_end = share.end;
    const int it0 = at - row_first, it1 = min(end, row_end) - row_first;
    at = min(end, row_end);
    const int visible = min(share.visible, it1 * kTileKeys);  // to the end of this share
    const int32_t* pages = a.table + (int64_t)share.request * a.width;

    // this wave's part of the queries: step i covers elements 16 (part + NP i) ..; the third parts of the band's
    bf16x8 qf[KS], ql[KS], q3[KS - KC];
    {
      const int64_t q = ((int64_t)t * a.H + (nh > 0 ? h0 + min(n, nh - 1) : 0)) * kRow + 8 * g + 16 * part;
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        qf[i] = *reinterpret_cast<const bf16x8*>((const bf16*)a.qa + q + 16 * NP * i);
        ql[i] = *reinterpret_cast<const bf16x8*>((const bf16*)a.qa_lo + q + 16 * NP * i);
        if (i >= KC) q3[i >= KC ? i - KC : 0] = *reinterpret_cast<const bf16x8*>((const bf16*)a.qa_low2 + q + 16 * NP * i);
      }
    }
    f32x16 oacc[NB];
    float m = -INFINITY, lsum;

    // Where a tile's rows are: each lane looks up the page of row n, and the copies take the rows' places
    // from the lanes. A key past the share's end, or without a page (bad), is copied from zeros.
    int win = 0, win_end;  // first page of the window, and the first key past it
    auto page_of = [&](int key) { return (int)((uint64_t)(uint32_t)key * a.page_magic >> a.page_shift); };
    auto refill = [&](int it) {  // the window reaches tile `it`
      const int k0 = it * kTileKeys;
      if (k0 < visible && min(k0 + kTileKeys, visible) > win_end) {
        win = page_of(k0);
        win_end = (int)min((int64_t)(win + kPages) * a.page, (int64_t)INT32_MAX);
        const int have = page_of(visible - 1) + 1;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = fresh_lane(); i < kPages; i += 64) win_ids[i] = win + i < have ? pages[win + i] : -1;
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
    };
    int key_page, key_id;
    auto look = [&](int it) {
      const int key = it * kTileKeys + (fresh_lane() & 31);
      key_page = key < visible ? page_of(key) : win;
      key_id = win_ids[key_page - win];
    };
    struct Rows { int lo, hi, band_lo, band_hi; uint32_t bad; };  // (band: of row 8 wave + lane / 8)
    const char* zeros = (const char*)kZeroRow;
    asm volatile("" : "+s"(zeros));
    auto rows_of = [&](int it) {  // (of the tile that was looked up last)
      const int l = fresh_lane(), key = it * kTileKeys + (l & 31);
      const bool live = key < visible, ok = live && (unsigned)key_id < (unsigned)a.n_pages;
      const int64_t off = 2 * ((int64_t)key_id * a.page_stride + (int64_t)(key - key_page * a.page) * kRow);
      const uintptr_t src = ok ? (uintptr_t)a.cache + off : (uintptr_t)zeros;
      const int lo = (int)(uint32_t)src, hi = (int)(uint32_t)(src >> 32), r = 8 * wave + (l >> 3);
      return Rows{lo, hi, __shfl(lo, r), __shfl(hi, r), (uint32_t)__ballot(live && !ok)};
    };
    // This wave's quarter of a tile's copies: rows wave, wave + 4, .. and an eighth of the band. The place of the
    // j-th is taken some instructions before it.
    constexpr int NMAIN = kTileKeys / 4, NCOPY = NMAIN + 1;
    auto place = [&](const Rows& x, int j) -> const void* {
      const int r = wave + 4 * (j < NMAIN ? j : 0);
      int lo = __builtin_amdgcn_readlane(x.lo, r), hi = __builtin_amdgcn_readlane(x.hi, r);
      asm volatile("" : "+s"(lo), "+s"(hi));  // (here, not where it is used)
      return (const void*)((uintptr_t)(uint32_t)lo | ((uintptr_t)(uint32_t)hi << 32));
    };
    auto copy = [&](const Rows& x, const void* place, uint32_t tile, int j) {
      // swz<16>(wave + 4 j) is swz<16>(wave) and two bits of j
      if (j < NMAIN) copy_row<NT>(place, at_copy ^ (16 * swz<16>(4 * j)), tile + 2 * wave * kDc, 8 * j * kDc);
      else copy_lanes<NT>((const char*)((uintptr_t)(uint32_t)x.band_lo | ((uintptr_t)(uint32_t)x.band_hi << 32)) + at_band, tile + 1024 * wave, 2 * kMain);
    };
    auto fetch = [&](int it, uint32_t tile) {  // a whole tile at once
      refill(it);
      look(it);
      const Rows x = rows_of(it);
      const void* base[NCOPY];
#pragma unroll
      for (int j = 0; j < NCOPY; ++j) base[j] = place(x, j);
      asm volatile("s_nop 0");
#pragma unroll
      for (int j = 0; j < NCOPY; ++j) copy(x, base[j], tile, j);
      return x.bad;
    };
    auto k_frag = [&](uint32_t tile, int i) {
      return i < KC ? lds_at<bf16x8>(((tile + at_k) ^ (32 * (NP * i % 8))) + 256 * (NP * i / 8))
                    : lds_at<bf16x8>((tile + at_b) ^ (32 * NP * (i - KC)));
    };
    auto v_frag = [&](uint32_t tile, int i) {  // column block i % NB, keys 16 (i / NB) ..
      const uint32_t flip = 64 * (NP * (i % NB) % 4), add = 256 * (NP * (i % NB) / 4) + 32 * kDc * (i / NB);
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(uintptr_t)(((tile + at_v) ^ flip) + add));
      const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(uintptr_t)(((tile + at_v8) ^ flip) + add));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    // fragments are read PF (PV) steps ahead, in a pinned order
    constexpr int PF = 4, PV = 4, NV = 2 * NB;
    struct Ahead { bf16x8 k[PF], v[PV]; };
    auto read_k = [&](uint32_t tile, Ahead& x) {
#pragma unroll
      for (int i = 0; i < PF; ++i) x.k[i] = k_frag(tile, i);
    };
    auto read_v = [&](uint32_t tile, Ahead& x) {
#pragma unroll
      for (int i = 0; i < PV; ++i) x.v[i] = v_frag(tile, i);
    };
    // This wave's part of a tile's scores, the first fragments read before; `beside(j)` runs beside product j < 2 KS.
    auto products = [&](uint32_t tile, const Ahead& x, f32x16& s, auto&& beside) {
      bf16x8 k[PF + 1];
#pragma unroll
      for (int i = 0; i < PF; ++i) k[i] = x.k[i];
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        if (i + PF < KS) k[(i + PF) % (PF + 1)] = k_frag(tile, i + PF);
        score_step(s, k[i % (PF + 1)], qf[i], i == 0);
        __builtin_amdgcn_sched_barrier(0);
        beside(2 * i);
        __builtin_amdgcn_sched_barrier(0);
        score_step_low(s, k[i % (PF + 1)], ql[i]);
        if (i >= KC) score_step_low(s, k[i % (PF + 1)], q3[i >= KC ? i - KC : 0]);
        __builtin_amdgcn_sched_barrier(0);
        beside(2 * i + 1);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    // This wave's part of a tile's scores to the others. Keys that are not to be seen get -infinity here, keys
    // without a page NaN: neither is changed by the other parts' sums of zeros.
    auto give = [&](int turn, int it, uint32_t bad, f32x16& s) {
      scores_done(s);
      const int lim = visible - it * kTileKeys;
      if (lim < kTileKeys || bad) {
        const int g = fresh_lane() >> 5;  // (and keeps the branch)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int k = (r >> 2) * 8 + (r & 3) + 4 * g;
          s[r] = k < lim ? (bad >> k & 1 ? NAN : s[r]) : -INFINITY;
        }
      }
      const int l = fresh_lane();
#pragma unroll
      for (int rr = 0; rr < 4; ++rr)
        sums[((turn * 4 + wave) * 4 + rr) * 64 + l] = f32x4{s[4 * rr], s[4 * rr + 1], s[4 * rr + 2], s[4 * rr + 3]};
    };
    // The parts of a tile's scores, added up in order (two of them: the other one to this wave's), so that
    // every wave of the group has the same bits.
    constexpr int NX = NP == 2 ? 1 : NP;
    struct Parts { f32x4 v[NX][4]; };
    auto read_parts = [&](int turn) {
      Parts p;
      const int l = fresh_lane();
#pragma unroll
      for (int u = 0; u < NX; ++u)
#pragma unroll
        for (int rr = 0; rr < 4; ++rr) p.v[u][rr] = sums[((turn * 4 + (NP == 2 ? wave ^ HG : hg + HG * u)) * 4 + rr) * 64 + l];
      return p;
    };
    auto add_parts = [&](const Parts& p, int rr, f32x16& s) {
      f32x4 v = p.v[0][rr];
      if constexpr (NP == 2) v += f32x4{s[4 * rr], s[4 * rr + 1], s[4 * rr + 2], s[4 * rr + 3]};
#pragma unroll
      for (int u = 1; u < NX; ++u) v += p.v[u][rr];
#pragma unroll
      for (int e = 0; e < 4; ++e) s[4 * rr + e] = v[e];
    };
    auto raise = [&](f32x16 s, int turn) {  // m to a tile's maximum, of its parts
      const Parts parts = read_parts(turn);
      float mx = -INFINITY;
#pragma unroll
      for (int rr = 0; rr < 4; ++rr) {
        add_parts(parts, rr, s);
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[4 * rr + e]);
      }
      m = fmaxf(m, wave_xor32_max(mx) * a.scale_log2);
    };
    // O with a tile's probabilities hi + lo, two column blocks at a time, so that no product waits for the
    // one before it; `beside(i)` runs beside pair i < NB. When the tile's last fragment has been read: `read`.
    auto accumulate = [&](uint32_t tile, const Ahead& x, const bf16x8 (&pf)[2], const bf16x8 (&pl)[2], auto&& beside, auto&& read) {
      bf16x8 v[PV + 2];
#pragma unroll
      for (int i = 0; i < PV; ++i) v[i] = x.v[i];
#pragma unroll
      for (int i = 0; i < NV; i += 2) {
        if (i + PV < NV) {
          v[(i + PV) % (PV + 2)] = v_frag(tile, i + PV);
          v[(i + PV + 1) % (PV + 2)] = v_frag(tile, i + PV + 1);
        }
        if (i + PV == NV) read();
        const bf16x8 &v0 = v[i % (PV + 2)], &v1 = v[(i + 1) % (PV + 2)];
        mma(oacc[i % NB], v0, pf[i / NB]);
        mma(oacc[i % NB + 1], v1, pf[i / NB]);
        mma(oacc[i % NB], v0, pl[i / NB]);
        mma(oacc[i % NB + 1], v1, pl[i / NB]);
        beside(i / 2);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    // All tiles of the share; once more with its maximum where the first tile's does not do
    for (bool again = false;; again = true) {
#pragma unroll
      for (int i = 0; i < NB; ++i) oacc[i] = f32x16{};
      lsum = 0.f;
      win_end = 0;
      lds_barrier();  // the tiles and parts before are read
      const uint32_t bad0 = fetch(it0, ring);
      uint32_t bad1 = fetch(it0 + 1, ring + 2 * kTile);
      refill(it0 + 2);
      look(it0 + 2);
      Rows rows = rows_of(it0 + 2);
      wait_vmem_le<NCOPY>();
      lds_barrier();
      f32x16 s;
      Ahead ahead;
      read_k(ring, ahead);
      products(ring, ahead, s, [](int) {});
      give(0, it0, bad0, s);
      wait_vmem();
      lds_barrier();
      if (!again) raise(s, 0);
      bool high = m == -INFINITY;
      const float m_use = m == -INFINITY ? 0.f : m;
      read_k(ring + 2 * kTile, ahead);
      uint32_t tile0 = ring, tile1 = ring + 2 * kTile, tile2 = ring + 4 * kTile;  // of tiles it, it + 1, it + 2
      for (int it = it0, turn = 0; it < it1; ++it, turn ^= 1) {
        f32x16 next;
        bf16x8 pf[2], pl[2];
        Parts parts;
        float ps = 0.f;
        const void* base;
        auto piece = [&](int i) {  // of the softmax of tile `it`
          if (i == 0) {
            parts = read_parts(turn);
          } else if (i >= 6 && i < 10) {
            add_parts(parts, i - 6, s);
#pragma unroll
            for (int r = 4 * (i - 6); r < 4 * (i - 5); ++r) s[r] = here(s[r]);
          } else if (i >= 10 && i < 27) {
            const int r = i - 10;  // (an exponential's result is used a product later)
            if (r > 0) ps = here(ps + s[r - 1]);
            if (r < 16) s[r] = here(fast_exp2(__builtin_fmaf(s[r], a.scale_log2, -m_use)));
            if (r == 8 || r == 16) pf[r / 8 - 1] = here(acc_to_frag<bf16>(s, r / 8 - 1));  // (its halves are taken from it, too)
          } else if (i >= 27 && i < 35) {
            const int kk = (i - 27) / 4, e0 = (i - 27) % 4 * 2;
            s[8 * kk + e0] = here(s[8 * kk + e0] - to_f32(pf[kk][e0]));
            s[8 * kk + e0 + 1] = here(s[8 * kk + e0 + 1] - to_f32(pf[kk][e0 + 1]));
            if (e0 == 6) pl[kk] = here(acc_to_frag<bf16>(s, kk));
          } else if (i == 35) {
            read_v(tile0, ahead);
          }
        };
        products(tile1, ahead, next, [&](int j) {
          constexpr int EVERY = 2 * KS / NCOPY;
          if (j % EVERY == 0) base = place(rows, j / EVERY);
          if (j % EVERY == 1) copy(rows, base, tile2, j / EVERY);
#pragma unroll
          for (int i = 36 / (2 * KS) * j; i < 36 / (2 * KS) * (j + 1); ++i) piece(i);
        });
        give(turn ^ 1, it + 1, bad1, next);
        bad1 = rows.bad;
        lsum += ps;
        high |= ps > __builtin_exp2f(kHead);
        refill(it + 3);
        accumulate(
            tile0, ahead, pf, pl,
            [&](int i) {
              if (i == 0) look(it + 3);
              if (i == NB - 3) {
                rows = rows_of(it + 3);
                asm volatile("" : "+v"(rows.lo), "+v"(rows.hi));
              }
            },
            [&]() {
              wait_vmem();
              lds_barrier();  // every wave's copies of tile it + 2 and part of tile it + 1's scores; tile it is read
              read_k(tile2, ahead);
            });
        s = next;
        const uint32_t free = tile0;
        tile0 = tile1, tile1 = tile2, tile2 = free;
      }
      if (again) break;
      const bool any = __ballot(high) != 0;
      if (l == 0) s_high[wave] = any;
      lds_barrier();
      if (!(s_high[0] | s_high[1] | s_high[2] | s_high[3])) break;
      win_end = 0;
      for (int it = it0; it < it1; ++it) {  // the maximum alone, a tile after the other
        lds_barrier();  // the tile and the parts before are read
        const uint32_t bad = fetch(it, ring);
        wait_vmem();
        lds_barrier();
        f32x16 s;
        Ahead ahead;
        read_k(ring, ahead);
        products(ring, ahead, s, [](int) {});
        give(0, it, bad, s);
        lds_barrier();
        raise(s, 0);
      }
    }

    // lane: head n, columns 32 (part + NP i) + 8 (r / 4) + 4 g + r % 4
    const bool whole = it0 == 0 && it1 == row_end - row_first;
    const float ltot = wave_xor32_sum(lsum), f = whole ? 1.f / ltot : 1.f;
    const int h = h0 + n;
    if (n < nh) {
      float* o = whole ? a.obar + ((int64_t)t * a.H + h) * kDc
                       : a.part_o + ((int64_t)partial_place(w, per, row_first) * a.H + h) * kDc;
      o += 32 * part + 4 * g;
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int rr = 0; rr < 4; ++rr)
          *reinterpret_cast<f32x4*>(o + 32 * NP * i + 8 * rr) =
              f32x4{oacc[i][4 * rr] * f, oacc[i][4 * rr + 1] * f, oacc[i][4 * rr + 2] * f, oacc[i][4 * rr + 3] * f};
      if (part == 0 && g == 0) {
        if (!whole) {
          float* ml = a.part_ml + 2 * ((int64_t)partial_place(w, per, row_first) * a.H + h);
          ml[0] = m;
          ml[1] = ltot;
        } else if (a.lse) {
          a.lse[(int64_t)t * a.H + h] = (m + fast_log2(ltot)) * kLn2;
        }
      }
    }
    if (at >= end) return;
    share = next_share(a, t, at);
    at = share.first;
    if (at >= end) return;
  }
}

// Where each row has a request of its own, a tile's copies pass the caches by (a hint: nt); successive rows of one
// request read the same pages again, from there. Us of a call with the hint and without: 64 requests x up to
// 8192 keys, 16 heads 95 and 103; 61, 128 heads 199 and 207; 64 x 4000, 64 heads 89 and 92; but 4 tokens for each
// of 64 requests, 16 heads 289 and 275, 512 tokens of one request over 8192 keys 872 and 726.
template <int HG>
__global__ __launch_bounds__(256, 1) void wide_kernel(PagedArgs a, int head_blocks) {
  constexpr int kFew = SplitCfg<bf16, 4>::LDS;
  __shared__ __attribute__((aligned(256))) unsigned char smem[kLds > kFew ? kLds : kFew];
  __shared__ int32_t s_page[4][kPages];
  __shared__ int s_high[4];
  // the head blocks of a worker follow each other on one XCD: its L2 serves all but the first
  const int id = blockIdx.x, hb = id / 8 % head_blocks, w = id / (8 * head_blocks) * 8 + id % 8;
  const int per = uniform(a.sched[0]), total = uniform(a.sched[1]), groups = uniform(a.sched[2]);
  const int hb0 = hb * a.heads_per_wg, hb1 = min(a.H, hb0 + a.heads_per_wg);
  if (groups > 0) {  // few tiles
    const int hf = hb0 + 32 * (w / 8 % groups);
    if (w / (8 * groups) < a.workers / (8 * groups) && hf < hb1)
      split_shares<bf16, 4>(a, smem, w / (8 * groups) * 8 + w % 8, hf, min(32, hb1 - hf), per, total);
  } else if (uniform(a.sched[4])) {
    wide_shares<HG, false>(a, smem, s_page, s_high, w, hb0, hb1, per, total);
  } else {
    wide_shares<HG, true>(a, smem, s_page, s_high, w, hb0, hb1, per, total);
  }
}

}  // namespace

void launch_paged_wide(const PagedArgs& a, int head_blocks, hipStream_t st) {
  const unsigned wgs = (unsigned)(head_blocks * a.workers);
  if (a.heads_per_wg > 32) wide_kernel<2><<<wgs, 256, 0, st>>>(a, head_blocks);
  else wide_kernel<1><<<wgs, 256, 0, st>>>(a, head_blocks);
}

}  // namespace laga
