// Split attention over the paged cache for bf16 with d_c = 512 and d_rope = 64: a wave owns 32
// heads over the whole row, so every byte of a tile that it reads from LDS feeds 32 heads and
// no partial scores cross waves. (paged_attn.hip has the form for any width.)
#define LAGA_LDS_DMA_ASM 1
#include "paged_split.hpp"

namespace laga {
namespace {

// A workgroup's four waves are HG groups of 32 heads x KP = 4 / HG parts of the keys. HG = 4, more than
// 32 heads: the waves share a tile, and a ring of four of them in LDS (with two groups x two parts for 33
// to 64 heads, a tile for each part and one stage ahead, 64 requests x 4000 keys took 180 us, so 80).
// HG = 1: each wave takes every fourth tile, fills and reads its one stage by itself, the other
// three waves' copies and products overlap with its wait, and the parts meet at the row's end.
//   S^T = K Q^T, O^T += C^T P^T, a lane per head, as in the general kernel
// Registers: Q (36 fragments of a row's 576 elements), the low halves of its band, and O (512 columns
// x 32 heads) in the accumulation registers. The low halves of q W_k^T have no room: their effect on
// lse is added to first order where the rows are joined, as scale * lo . o (the second is below 1e-6).
constexpr int kDc = 512, kDr = 64, kRow = kDc + kDr;
constexpr int kMain = kTileKeys * kDc, kBand = kTileKeys * kDr, kTile = kMain + kBand;  // elements
// The softmax's reference is the maximum of the part's first tile and stays, so that no sum is ever rescaled
// (O would have to leave the accumulation registers for it): bf16 and fp32 hold 2^kHead as
// they hold 1, and probabilities, sums and their parts keep their precision. Where a later score passes it by
// more, the row's share is swept again, for its maximum and then with it.
constexpr float kHead = 64.f;
constexpr int kPages = 128;  // page ids of a row that a wave keeps in LDS

// A product of the chain S^T. Written out, because S^T has to stay in ordinary registers (the
// accumulation ones are all O's); scores_done waits until the chain's last product is written.
__device__ __forceinline__ void score_step(f32x16& s, const bf16x8& k, const bf16x8& q, bool first) {
  if (first) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(k), "v"(q));
  else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(k), "v"(q));
}
__device__ __forceinline__ void scores_done(f32x16& s) { asm volatile("s_nop 15\n\ts_nop 15" : "+v"(s)); }

// Direct copies of 1 KB (common.hpp, g2lds16_so and g2lds16). NT: the data are used by this workgroup alone, and
// pass the caches by (6.9 against 5.9 TB/s for a pool read once, 334 MB).
template <bool NT>
__device__ __forceinline__ void copy_row(const void* at, uint32_t off, void* lds) {
  const void* base = uniform((const char*)at);
  if constexpr (!NT) return g2lds16_so(base, off, lds);
  const uint32_t m = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)lds);
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(off), "s"(base), "s"(m)
               : "memory", "m0");
}
template <bool NT>
__device__ __forceinline__ void copy_lanes(const void* g, void* lds) {
  if constexpr (!NT) return g2lds16(g, lds);
  const uint32_t m = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)lds);
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" ::"v"(g), "s"(m) : "memory", "m0");
}
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}
template <typename V>
__device__ __forceinline__ V lds_at(uint32_t address) {
  return *(__attribute__((address_space(3))) const V*)(uintptr_t)address;
}

template <int HG, bool NT>
__global__ __launch_bounds__(256, 1) void wide_kernel(PagedArgs a, int head_blocks) {
  static_assert(HG == 1 || HG == 4);
  constexpr int KP = 4 / HG;
  __shared__ __attribute__((aligned(16))) bf16 ring[4 * kTile];
  static_assert(SplitCfg<bf16, 4>::LDS <= (int)sizeof(ring), "the general form's LDS");
  __shared__ int32_t s_page[4][kPages];
  __shared__ bf16x8 s_low[4][kDr / 32][64];
  __shared__ float s_m[4][32], s_l[4][32];
  __shared__ int s_high[4];

  const int l = threadIdx.x & 63, n = l & 31, g = l >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hg = wave % HG, kp = wave / HG;
  // the head blocks of a worker follow each other on one XCD: its L2 serves all but the first
  const int id = blockIdx.x, hb = id / 8 % head_blocks, w = id / (8 * head_blocks) * 8 + id % 8;
  const int per = uniform(a.sched[0]), total = uniform(a.sched[1]), groups = uniform(a.sched[2]);
  const int hb0 = hb * a.heads_per_wg, hb1 = min(a.H, hb0 + a.heads_per_wg);
  if (groups > 0) {  // few tiles
    const int hf = hb0 + 32 * (w / 8 % groups);
    if (w / (8 * groups) < a.workers / (8 * groups) && hf < hb1)
      split_shares<bf16, 4>(a, (unsigned char*)ring, w / (8 * groups) * 8 + w % 8, hf, min(32, hb1 - hf), per, total);
    return;
  }
  const int h0 = hb0 + 32 * hg, nh = min(32, hb1 - h0);  // nh <= 0: this wave only copies
  const int64_t start = (int64_t)w * per;
  if (start >= total) return;
  const int end = (int)min((int64_t)total, start + per);
  int32_t* win_ids = s_page[wave];

  Share share = first_share(a, w);
  if (share.first >= end) return;  // (units of no tile)
  for (int at = max((int)start, share.first);;) {
    const int t = share.t, row_first = share.first, row_end = share.end;
    const int it0 = at - row_first, it1 = min(end, row_end) - row_first;
    at = min(end, row_end);
    const int visible = min(share.visible, it1 * kTileKeys);  // to the end of this share
    const int32_t* pages = a.table + (int64_t)share.request * a.width;

    // (half of the band's low halves in LDS: with all in registers one of Q's would spill)
    bf16x8 qf[kRow / 16], ql[kDr / 32];
    {
      const int64_t q = ((int64_t)t * a.H + (nh > 0 ? h0 + min(n, nh - 1) : 0)) * kRow + 8 * g;
#pragma unroll
      for (int i = 0; i < kRow / 16; ++i) qf[i] = *reinterpret_cast<const bf16x8*>((const bf16*)a.qa + q + 16 * i);
#pragma unroll
      for (int i = 0; i < kDr / 16; ++i) {
        const bf16x8 x = *reinterpret_cast<const bf16x8*>((const bf16*)a.qa_lo + q + kDc + 16 * i);
        if (i < kDr / 32) ql[i] = x;
        else s_low[wave][i - kDr / 32][l] = x;
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    }
    f32x16 oacc[kDc / 32];
    float m = -INFINITY, lsum;
    bool high;
    int win;
    auto page_of = [&](int key) { return (int)((uint64_t)(uint32_t)key * a.page_magic >> a.page_shift); };
    // This wave's share of the copies of tile `it` into buf; returns the tile's keys with no page.
    // Rows are 1152 bytes apart where the tile lies in one page; else, and in a row's last tile (and with
    // HG = 1, whose copies wait for memory and not for their addresses), each row's place comes
    // from the lane of its key.
    constexpr int NMAIN = kTileKeys / HG, NCOPY = NMAIN + 4 / HG;
    auto copy = [&](const char* flat, bf16* buf, int j, int l) {  // the j-th, of a tile that lies in one page
      if (j < NMAIN) {
        const int r = hg + HG * j;
        copy_row<NT>(flat + r * 2 * kRow, (uint32_t)((l ^ swz<16>(r)) * 16), buf + r * kDc);
      } else {
        const int i = hg + HG * (j - NMAIN), r = l >> 3;  // (rows 8 apart are swizzled by the flip of one bit)
        copy_row<NT>(flat + 8 * i * 2 * kRow + 2 * kDc, r * 2 * kRow + ((l & 7) ^ swz<8>(r) ^ (i & 1)) * 16,
                     buf + kMain + i * 512);
      }
    };
    const char* flat = nullptr;  // the tile's first row, where the copies are left to the caller
    int ahead = 0;               // and the id of its first page, read from the window beforehand
    auto look = [&](int it) { ahead = win_ids[min((uint32_t)(page_of(it * kTileKeys) - win), kPages - 1u)]; };
    auto fetch = [&](int it, bf16* buf, bool at_once) -> uint32_t {
      const int l = fresh_lane(), n = l & 31;
      const int k0 = it * kTileKeys, p0 = page_of(k0), o0 = k0 - p0 * a.page;
      if (k0 < visible && (win < 0 || page_of(min(k0 + kTileKeys, visible) - 1) >= win + kPages)) {
        win = p0;
        const int have = page_of(visible - 1) + 1;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = l; i < kPages; i += 64) win_ids[i] = win + i < have ? pages[win + i] : -1;
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (!at_once) look(it);
      }
      flat = nullptr;
      if (HG > 1 && k0 + kTileKeys <= visible && o0 + kTileKeys <= a.page) {
        const int pid = uniform(at_once ? win_ids[p0 - win] : ahead);
        if ((unsigned)pid < (unsigned)a.n_pages) {
          const char* base = uniform((const char*)((const bf16*)a.cache + (int64_t)pid * a.page_stride + (int64_t)o0 * kRow));
          if (at_once) {
#pragma unroll
            for (int j = 0; j < NCOPY; ++j) copy(base, buf, j, l);
          } else {
            flat = base;
          }
          return 0;
        }
      }
      const int key = k0 + n;
      const bool live = key < visible;
      const int pg = live ? page_of(key) : win, off = live ? key - pg * a.page : 0;
      const int pid = win_ids[pg - win];  // (0 of the last window for a tile past the end)
      const bool ok = live && (unsigned)pid < (unsigned)a.n_pages;
      const bf16* src =
          ok ? (const bf16*)a.cache + (int64_t)pid * a.page_stride + (int64_t)off * kRow : (const bf16*)kZeroRow;
      const int lo = (int)(uint32_t)(uintptr_t)src, hi = (int)(uint32_t)((uintptr_t)src >> 32);
#pragma unroll
      for (int j = 0; j < NMAIN; ++j) {
        const int r = hg + HG * j;
        const uintptr_t base = (uintptr_t)(uint32_t)__builtin_amdgcn_readlane(lo, r) |
                               ((uintptr_t)(uint32_t)__builtin_amdgcn_readlane(hi, r) << 32);
        copy_row<NT>((const void*)base, (uint32_t)((l ^ swz<16>(r)) * 16), buf + r * kDc);
      }
#pragma unroll
      for (int j = 0; j < 4 / HG; ++j) {
        const int i = hg + HG * j, r = 8 * i + (l >> 3);
        const uintptr_t base = (uintptr_t)(uint32_t)__shfl(lo, r) | ((uintptr_t)(uint32_t)__shfl(hi, r) << 32);
        copy_lanes<NT>((const bf16*)base + kDc + (((l & 7) ^ swz<8>(r)) * 8), buf + kMain + i * 512);
      }
      return (uint32_t)__ballot(live && !ok);
    };
    // fragments are read PF (PV) products ahead, in a pinned order
    constexpr int PF = HG == 4 ? 3 : 5, NQ = kRow / 16, PV = 4, NV = 2 * (kDc / 32);
    // Chunk c of a tile's row r is at c ^ swz<16>(r) (c part; c ^ swz<8>(r) in the band). This lane
    // reads the fragment of contraction step i in row n at (k ^ 32 (i % 8)) + 256 (i / 8), of
    // the band's step i at b ^ 32 i, and for the transposing reads of column block i, rows vr
    // and vr + 8, at (v ^ 64 (i % 4)) + 256 (i / 4) and likewise v8.
    struct Reads { uint32_t k, b, v, v8; };
    auto reads_of = [&](const bf16* buf) {
      const uint32_t at = lds_address(buf);
      const int l = fresh_lane(), n = l & 31, g = l >> 5;
      const int sl = l & 15, vr = 4 * g + (sl >> 2), vc = 2 * ((l >> 4) & 1) + ((sl & 3) >> 1);
      return Reads{at + 2 * n * kDc + ((g ^ swz<16>(n)) * 16), at + 2 * (kMain + n * kDr) + ((g ^ swz<8>(n)) * 16),
                   at + 2 * vr * kDc + ((vc ^ swz<16>(vr)) * 16) + 8 * (sl & 1),
                   at + 2 * (vr + 8) * kDc + ((vc ^ swz<16>(vr + 8)) * 16) + 8 * (sl & 1)};
    };
    auto k_frag = [&](const Reads& x, int i) {
      return i < kDc / 16 ? lds_at<bf16x8>((x.k ^ (32 * (i % 8))) + 256 * (i / 8)) : lds_at<bf16x8>(x.b ^ (32 * (i - kDc / 16)));
    };
    auto v_frag = [&](const Reads& x, int i) {  // column block i % 16, keys 16 (i / 16) ..
      const uint32_t flip = 64 * (i % 4), add = 256 * (i % 16 / 4) + 32 * kDc * (i / 16);
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(uintptr_t)((x.v ^ flip) + add));
      const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(uintptr_t)((x.v8 ^ flip) + add));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    // S^T of a tile; `beside(i)` runs beside product i
    auto products = [&](const Reads& x, f32x16& s, auto&& beside) {
      constexpr int B0 = kDc / 16, B1 = B0 + kDr / 32;  // the band's steps; those with low halves in LDS
      bf16x8 k[PF + 1], low[kDr / 32];
      const uint32_t low_at = lds_address(s_low[wave]) + 16 * fresh_lane();
#pragma unroll
      for (int i = 0; i < PF; ++i) k[i] = k_frag(x, i);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        if (i + PF < NQ) k[(i + PF) % (PF + 1)] = k_frag(x, i + PF);
        if (i + PF >= NQ && i + PF - NQ < kDr / 32) low[i + PF - NQ] = lds_at<bf16x8>(low_at + 1024 * (i + PF - NQ));
        score_step(s, k[i % (PF + 1)], qf[i], i == 0);
        if (i >= B0) score_step(s, k[i % (PF + 1)], i < B1 ? ql[i < B1 ? i - B0 : 0] : low[i < B1 ? 0 : i - B1], false);
        beside(i);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    auto mask = [&](int it, uint32_t bad, f32x16& s) {
      const int lim = visible - it * kTileKeys;
      if (lim < kTileKeys || bad) {
        const int g = fresh_lane() >> 5;  // (and keeps the branch)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int k = (r >> 2) * 8 + (r & 3) + 4 * g;
          s[r] = k < lim ? (bad >> k & 1 ? NAN : s[r]) : -INFINITY;
        }
      }
    };
    // a tile's scores, and its largest over the lane's head
    auto scores = [&](int it, const Reads& x, uint32_t bad, f32x16& s) {
      products(x, s, [](int) {});
      scores_done(s);
      mask(it, bad, s);
      float mx = -INFINITY;
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[r]);
      return wave_xor32_max(mx) * a.scale_log2;
    };
    // O with a tile's probabilities hi + lo, two column blocks at a time, so that no product waits for the
    // one before it; `beside(i)` runs beside product i
    auto accumulate = [&](const Reads& x, const bf16x8 (&pf)[2], const bf16x8 (&pl)[2], auto&& beside) {
      bf16x8 v[PV + 2];
#pragma unroll
      for (int i = 0; i < PV; ++i) v[i] = v_frag(x, i);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < NV; i += 2) {
        if (i + PV < NV) {
          v[(i + PV) % (PV + 2)] = v_frag(x, i + PV);
          v[(i + PV + 1) % (PV + 2)] = v_frag(x, i + PV + 1);
        }
        const bf16x8 &v0 = v[i % (PV + 2)], &v1 = v[(i + 1) % (PV + 2)];
        mma(oacc[i % 16], v0, pf[i / 16]);
        beside(2 * i);
        mma(oacc[i % 16 + 1], v1, pf[i / 16]);
        beside(2 * i + 1);
        mma(oacc[i % 16], v0, pl[i / 16]);
        beside(2 * i + 2);
        mma(oacc[i % 16 + 1], v1, pl[i / 16]);
        beside(2 * i + 3);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    // O and the sums with a tile's probabilities
    auto update = [&](int it, const bf16* buf, uint32_t bad) {
      const Reads x = reads_of(buf);
      f32x16 s;
      const float mx = scores(it, x, bad, s);
      m = m == -INFINITY ? mx : m;  // (nothing but zeros or NaN is summed up so far)
      high |= __ballot(mx > m + kHead) != 0;
      const float m_use = m == -INFINITY ? 0.f : m;
      float ps = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[r] = fast_exp2(__builtin_fmaf(s[r], a.scale_log2, -m_use));
        ps += s[r];
      }
      lsum += ps;
      bf16x8 pf[2], pl[2];
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        pf[kk] = acc_to_frag<bf16>(s, kk);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[8 * kk + e] -= to_f32(pf[kk][e]);
        pl[kk] = acc_to_frag<bf16>(s, kk);
      }
      accumulate(x, pf, pl, [](int) {});
    };
    // the tiles of this wave's part, in order; a tile past the share's end (a part's last step) is
    // copied from zeros and all masked
    const int steps = (it1 - it0 + KP - 1) / KP;
    auto sweep = [&](auto&& body) {
      win = -1;
      lds_barrier();  // the tiles of the sweep before, and its parts, are read
      bf16* buf = ring + kp * kTile;
      for (int it = it0 + kp, i = 0; i < steps; ++i, it += KP) {
        if (HG > 1 && i > 0) lds_barrier();  // the tile before is read
        const uint32_t bad = fetch(it, buf, true);
        wait_vmem();
        if (HG > 1) lds_barrier();
        body(it, buf, bad);
      }
    };
    // The same for HG = 4, a tile ahead: the products of tile i + 1's scores run beside tile i's softmax,
    // the copies of tile i + 3 beside tile i's products with P (2 x 100000 keys, 128 heads: 98 us, a tile
    // after the other 103).
    auto sweep_ahead = [&](auto) {
      win = -1;
      lds_barrier();  // the tiles of the sweep before are read
      uint32_t bad0 = fetch(it0, ring, true), bad1 = fetch(it0 + 1, ring + kTile, true),
               bad2 = fetch(it0 + 2, ring + 2 * kTile, true);
      wait_vmem_le<2 * NCOPY>();
      lds_barrier();
      f32x16 s;
      products(reads_of(ring), s, [](int) {});
      scores_done(s);
      mask(it0, bad0, s);
      look(it0 + 3);
      for (int step = 0; step < steps; ++step) {
        const int it = it0 + step;
        wait_vmem_le<NCOPY>();
        lds_barrier();  // every wave's copies of tile it + 1; tile it - 1 is read
        const uint32_t bad3 = fetch(it + 3, ring + (step + 3 & 3) * kTile, false);
        f32x16 next;
        bf16x8 pf[2], pl[2];
        float mx = -INFINITY, ps = 0.f, m_use = 0.f;
        products(reads_of(ring + (step + 1 & 3) * kTile), next, [&](int i) {
          if (i < 8) {
            mx = fmaxf(mx, fmaxf(s[2 * i], s[2 * i + 1]));
          } else if (i == 8) {
            mx = wave_xor32_max(mx) * a.scale_log2;
          } else if (i == 9) {
            m = m == -INFINITY ? mx : m;  // (nothing but zeros or NaN is summed up so far)
            high |= __ballot(mx > m + kHead) != 0;
            m_use = m == -INFINITY ? 0.f : m;
          } else if (i < 26) {
            s[i - 10] = fast_exp2(__builtin_fmaf(s[i - 10], a.scale_log2, -m_use));
            ps += s[i - 10];
          } else if (i < 34) {
            const int kk = (i - 26) / 4, j = (i - 26) % 4;
            if (j == 0) pf[kk] = acc_to_frag<bf16>(s, kk);
            else if (j < 3)
#pragma unroll
              for (int e = 4 * (j - 1); e < 4 * j; ++e) s[8 * kk + e] -= to_f32(pf[kk][e]);
            else pl[kk] = acc_to_frag<bf16>(s, kk);
          }
        });
        lsum += ps;
        accumulate(reads_of(ring + (step & 3) * kTile), pf, pl, [&](int i) {
          if (i == 48) look(it + 4);
          if (i % 4 == 1 && i / 4 < NCOPY && flat) copy(flat, ring + (step + 3 & 3) * kTile, i / 4, fresh_lane());
        });
        asm volatile("" : "+v"(next));  // (its products are done long ago)
        mask(it + 1, bad1, next);
        s = next;
        bad1 = bad2;
        bad2 = bad3;
      }
      wait_vmem();
    };
    for (bool again = false;; again = true) {
#pragma unroll
      for (int i = 0; i < kDc / 32; ++i) oacc[i] = f32x16{};
      lsum = 0.f;
      high = false;
      if constexpr (HG == 4) sweep_ahead(0);
      else sweep(update);
      if (again) break;
      if (l == 0) s_high[wave] = high;
      lds_barrier();
      if (!(s_high[0] | s_high[1] | s_high[2] | s_high[3])) break;
      sweep([&](int it, const bf16* buf, uint32_t bad) {
        f32x16 s;
        m = fmaxf(m, scores(it, reads_of(buf), bad, s));
      });
    }

    // lane: head n, columns 32 i + 8 (r / 4) + 4 g + r % 4
    const bool whole = it0 == 0 && it1 == row_end - row_first;
    float ltot = wave_xor32_sum(lsum), f = 1.f;
    if constexpr (KP > 1) {
      if (g == 0) { s_m[wave][n] = m; s_l[wave][n] = ltot; }
      lds_barrier();  // (and every wave has read its tiles)
      float mx = -INFINITY;
#pragma unroll
      for (int u = 0; u < KP; ++u) mx = fmaxf(mx, s_m[u * HG + hg][n]);
      const float m_use = mx == -INFINITY ? 0.f : mx;
      ltot = 0.f;
#pragma unroll
      for (int u = 0; u < KP; ++u)
        ltot = __builtin_fmaf(s_l[u * HG + hg][n], fast_exp2(s_m[u * HG + hg][n] - m_use), ltot);
      f = fast_exp2(m - m_use);
      m = mx;
    }
    if (whole) f *= 1.f / ltot;
    const int h = h0 + n;
    float* o = whole ? a.obar + ((int64_t)t * a.H + h) * kDc
                     : a.part_o + ((int64_t)partial_place(w, per, row_first) * a.H + h) * kDc;
    o += 4 * g;
    if constexpr (KP == 1) {
      if (n < nh) {
#pragma unroll
        for (int i = 0; i < kDc / 32; ++i)
#pragma unroll
          for (int rr = 0; rr < 4; ++rr)
            *reinterpret_cast<f32x4*>(o + 32 * i + 8 * rr) =
                f32x4{oacc[i][4 * rr] * f, oacc[i][4 * rr + 1] * f, oacc[i][4 * rr + 2] * f, oacc[i][4 * rr + 3] * f};
      }
    } else {
      // parts of eight column blocks at a time through the tiles' LDS; each wave adds up its
      // 8 / KP blocks of them, parts in order
      f32x4* x = (f32x4*)ring;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if (half > 0) lds_barrier();
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int rr = 0; rr < 4; ++rr) {
            const f32x16& v = oacc[8 * half + i];
            x[((wave * 8 + i) * 4 + rr) * 64 + l] = f32x4{v[4 * rr] * f, v[4 * rr + 1] * f, v[4 * rr + 2] * f, v[4 * rr + 3] * f};
          }
        lds_barrier();
#pragma unroll
        for (int j = 0; j < 8 / KP; ++j) {
          const int i = kp * (8 / KP) + j;
#pragma unroll
          for (int rr = 0; rr < 4; ++rr) {
            f32x4 v = x[((hg * 8 + i) * 4 + rr) * 64 + l];
#pragma unroll
            for (int u = 1; u < KP; ++u) v += x[(((u * HG + hg) * 8 + i) * 4 + rr) * 64 + l];
            if (n < nh) *reinterpret_cast<f32x4*>(o + 32 * (8 * half + i) + 8 * rr) = v;
          }
        }
      }
    }
    if (kp == 0 && g == 0 && n < nh) {
      if (!whole) {
        float* ml = a.part_ml + 2 * ((int64_t)partial_place(w, per, row_first) * a.H + h);
        ml[0] = m;
        ml[1] = ltot;
      } else if (a.lse) {
        a.lse[(int64_t)t * a.H + h] = (m + fast_log2(ltot)) * kLn2;
      }
    }
    if (at >= end) return;
    share = next_share(a, t, at);
    at = share.first;
    if (at >= end) return;
  }
}

}  // namespace

void launch_paged_wide(const PagedArgs& a, int head_blocks, hipStream_t st) {
  const unsigned wgs = (unsigned)(head_blocks * a.workers);
  if (head_blocks > 1) wide_kernel<4, false><<<wgs, 256, 0, st>>>(a, head_blocks);
  else if (a.heads_per_wg > 32) wide_kernel<4, true><<<wgs, 256, 0, st>>>(a, head_blocks);
  else wide_kernel<1, true><<<wgs, 256, 0, st>>>(a, head_blocks);
}

}  // namespace laga
