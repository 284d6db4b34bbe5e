// Split attention over a paged cache held in 8 bits: rows of e4m3 numbers, with a power of two for the latent and one
// for the shared key of each position. (paged_attn.hip has the call's other launches.)
//
// The products run on fp16 operands, 16x16x32 at a time: an e4m3 number is an fp16 number, and two fp16 parts of a
// query value hold 22 bits of it (three bf16 parts would hold 24, for half as many products again). With key j's
// powers 2^c_j and 2^k_j
//
//   z_j = scale (2^c_j A_j + 2^k_j B_j),  A = qa . c8,  B = q_rope . k8,  O += (p_j 2^(c_j + d)) c8_j
//
// so the powers never meet a number of 8 bits: they are added to the exponents of A, B and p.
#define LAGA_LDS_DMA_ASM 1
#include "paged_dev.hpp"

namespace laga {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;
typedef __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 f16x2;
typedef __attribute__((__vector_size__(4 * sizeof(int)))) int i32x4;
typedef __attribute__((__vector_size__(2 * sizeof(int)))) int i32x2;

__device__ __forceinline__ void mma16(f32x4& acc, const f16x8& a, const f16x8& b) {
  acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, acc, 0, 0, 0);
}
// 8 e4m3 numbers in fp16, exactly
__device__ __forceinline__ f16x8 widen(int lo, int hi) {
  f16x8 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned x = i < 2 ? lo : hi;
    const f16x2 v = __builtin_bit_cast(f16x2, i % 2 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.f, true)
                                                    : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.f, false));
    y[2 * i] = v[0];
    y[2 * i + 1] = v[1];
  }
  return y;
}

// Rows are NK steps of 64 numbers of the latent and one of the band, zeros up to them. Of a workgroup's four waves
//   HG have 16 heads each, with both parts of their queries and O in registers;
//   CS = 2 halve the columns of O above d_c = 512, and both form all scores;
//   KW take a tile of 32 keys each, the next KW tiles after it, and put their sums together at a share's end.
// So a wave never waits for another's partial scores, and with 16 heads for no other wave at all.
template <int NK, int HG>
struct Q8Cfg {
  static constexpr int CS = NK > 8 ? 2 : 1;
  static constexpr int SW = HG * CS;           // waves that share a tile
  static constexpr int KW = 4 / SW;
  static constexpr int P = 4 * NK + 4;         // 16-byte chunks of an LDS row; 4 modulo 8, see kTurns
  static constexpr int NI = kTileKeys * P / 64;  // copies of 64 chunks per tile
  static constexpr int NJ = (NI + SW - 1) / SW;  // of each wave, at most; NI / SW at least
  static constexpr int TILE = kTileKeys * P * 16, STAGE = TILE + 256;  // the keys' exponents after their rows
  static constexpr int kFit = 150 * 1024 / STAGE / KW;
  static constexpr int NS = kFit < 8 ? kFit : 8;
  static constexpr int NB = 4 * NK / CS;       // blocks of 16 columns of a wave
  static constexpr int kRing = KW * NS * STAGE, kSums = KW > 1 ? 4 * NB * 64 * 16 : 0;
  static constexpr int LDS = kRing > kSums ? kRing : kSums;
  static_assert(SW * KW == 4 && NS >= 2 && P % 8 == 4);
};
constexpr int kIds = 128;  // page ids of a row that a wave keeps in LDS

// Chunk c of row r is at c ^ f(r), f(r) = entry r / 4 of kTurns: at a pitch of 4 chunks modulo 8 the four rows r % 4 begin a
// quarter round the banks apart, and f deals the rows of one r % 4 to its four chunks, in both readings: 16 bytes
// of 16 rows, two neighbouring chunks over the half-waves, and 16 bytes of the 8 rows 4 g .. + 3 and 16 + 4 g .. + 3
// in each quarter-wave g.
constexpr unsigned kTurns = 0u << 0 | 2u << 2 | 3u << 4 | 1u << 6 | 1u << 8 | 3u << 10 | 2u << 12 | 0u << 14;
__device__ __forceinline__ int turn_of(int row) { return kTurns >> (row >> 2) * 2 & 3; }

// A probability's fp16 reference: the running maximum is raised only where a score passes it by kRise, and p
// goes into the product as p 2^(c_j + d + kLift), d such that no p 2^(c_j + d) passes 2^kRise: 2^14 at most, and 11 bits
// down to 2^-28 of that.
constexpr float kRise = 8.f;
constexpr int kLift = 6;

__device__ __forceinline__ float quad_max(float x) {  // over the four lanes of a head
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float quad_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}
// 2 bytes per lane to LDS, 4 bytes apart
__device__ __forceinline__ void copy_short(const void* g, uint32_t to) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_ushort %0, off" ::"v"(g), "s"(to) : "memory", "m0");
}

// The share of worker w, for heads h0 .. h0 + heads (at most 16 HG). FINE: p in two parts.
template <int NK, int HG, bool FINE>
__device__ __forceinline__ void q8_shares(const PagedArgs& a, unsigned char* smem, int32_t (*s_ids)[kIds], int (*s_bad)[8],
                                          float (*s_ml)[2][16], int w, int h0, int heads, int per, int total) {
  using C = Q8Cfg<NK, HG>;
  constexpr int CS = C::CS, SW = C::SW, KW = C::KW, P = C::P, NI = C::NI, NJ = C::NJ, NS = C::NS, NB = C::NB;
  const int l = threadIdx.x & 63, n = l & 15, g = l >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kw = wave / SW, sr = wave % SW, hg = sr / CS, cs = sr % CS;
  const int W = a.d_c + a.d_rope;
  const int64_t start = (int64_t)w * per;
  if (start >= total) return;
  const int end = (int)min((int64_t)total, start + per);
  Share share = first_share(a, w);
  if (share.first >= end) return;  // (units of no tile)
  const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)smem + kw * NS * C::STAGE;
  int32_t* ids = s_ids[wave];

  // of a tile at LDS address x: rows n and 16 + n of K, from chunk g on; rows key(g, (l & 15) / 2) of C^T, chunk i % 4
  uint32_t at_k[2], at_v[4];
  {
    const int q = l & 15, vr = 4 * g + (q >> 1 & 3) + 16 * (q >> 3);
#pragma unroll
    for (int b = 0; b < 2; ++b) at_k[b] = (16 * b + n) * P * 16 + ((g ^ turn_of(16 * b + n)) * 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) at_v[i] = vr * P * 16 + ((i ^ turn_of(vr)) * 16) + 8 * (q & 1) + cs * NB * 16;
  }
  // copy j's lane: its row of the tile, and where in a cached row its chunk is
  constexpr uint32_t kNoPlace = ~0u;
  int row_of[NJ];
  uint32_t place[NJ];
#pragma unroll
  for (int jj = 0; jj < NJ; ++jj) {
    const int p = min(sr + SW * jj, NI - 1) * 64 + l, row = p / P, c = (p - row * P) ^ turn_of(row);
    row_of[jj] = row;
    place[jj] = c < 4 * NK ? (16 * c < a.d_c ? 16 * c : kNoPlace)
                           : (16 * (c - 4 * NK) < a.d_rope ? a.d_c + 16 * (c - 4 * NK) : kNoPlace);
  }

  for (int at = max((int)start, share.first);;) {
    const int t = share.t, row_first = share.first, row_end = share.end;
    const int it0 = at - row_first, it1 = min(end, row_end) - row_first;
    at = min(end, row_end);
    const int visible = min((int64_t)share.visible, (int64_t)it1 * kTileKeys);  // to the end of this share
    const int32_t* pages = a.table + (int64_t)share.request * a.width;

    // the queries of head n: of step i and half u elements 64 i + 16 g + 8 u .., scaled to 2^9 .. 2^10 at most
    f16x8 qh[NK + 1][2], ql[NK + 1][2];
    int e_c, e_k;
    {
      const int64_t th = (int64_t)t * a.H + h0 + min(16 * hg + n, heads - 1);
      const int blocks = qa_blocks(a.d_c);
      const float* tops = a.qa_max + th * blocks;
      float top = 0.f;
      for (int i = 0; i + 1 < blocks; ++i) top = fmaxf(top, tops[i]);
      auto power = [](float x) { return x > 0.f ? max(__builtin_amdgcn_frexp_expf(x), -126) - 10 : 0; };
      e_c = power(top);
      e_k = power(tops[blocks - 1]);
      const float* q = (const float*)a.qa + th * W;
#pragma unroll
      for (int i = 0; i <= NK; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int c = (i < NK ? 64 * i : 0) + 16 * g + 8 * u;
          const bool there = c < (i < NK ? a.d_c : a.d_rope);
          const float* from = q + (i < NK ? 0 : a.d_c) + (there ? c : 0);
          const f32x4 x0 = *reinterpret_cast<const f32x4*>(from), x1 = *reinterpret_cast<const f32x4*>(from + 4);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float x = there ? __builtin_ldexpf(e < 4 ? x0[e & 3] : x1[e & 3], i < NK ? -e_c : -e_k) : 0.f;
            const _Float16 hi = (_Float16)x;
            qh[i][u][e] = hi;
            ql[i][u][e] = (_Float16)(x - (float)hi);
          }
        }
    }
    f32x4 oacc[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) oacc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, lsum = 0.f;  // m a whole number
    int d = 0;                        // O has p 2^(c_j + d + kLift)

    int win = 0, win_end = 0;  // first page of the window, and the first key past it
    auto page_of = [&](int key) { return (int)((uint64_t)(uint32_t)key * a.page_magic >> a.page_shift); };
    // The copies of tile `it` into stage st. A key past the share's end, or without a page (bad), is copied from zeros.
    auto fetch = [&](int it, int st) {
      const int k0 = it * kTileKeys;
      if (min(k0 + kTileKeys, visible) > win_end) {
        win = page_of(k0);
        win_end = (int)min((int64_t)(win + kIds) * a.page, (int64_t)INT32_MAX);
        const int have = page_of(visible - 1) + 1;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = l; i < kIds; i += 64) ids[i] = win + i < have ? pages[win + i] : -1;
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
      const int key = k0 + (l & 31);
      const bool live = key < visible;
      const int pg = live ? page_of(key) : win, id = ids[pg - win];
      const bool ok = live && (unsigned)id < (unsigned)a.n_pages;
      const int off = key - pg * a.page;
      const char* src = ok ? (const char*)a.cache + (int64_t)id * a.page_stride + (int64_t)off * W : (const char*)kZeroRow;
      const char* exps = ok ? (const char*)a.scales + 2 * ((int64_t)id * a.page + off) : (const char*)kZeroRow;
      const uint32_t bad = (uint32_t)__ballot(live && !ok);
      if (l == 0) s_bad[wave][st] = (int)bad;
      const uint32_t tile = ring + st * C::STAGE;
      const int lo = (int)(uint32_t)(uintptr_t)src, hi = (int)(uint32_t)((uintptr_t)src >> 32);
#pragma unroll
      for (int jj = 0; jj < NJ; ++jj) {
        if (NI % SW == 0 || sr + SW * jj < NI) {
          const uintptr_t base = (uintptr_t)(uint32_t)__shfl(lo, row_of[jj]) | ((uintptr_t)(uint32_t)__shfl(hi, row_of[jj]) << 32);
          g2lds16(place[jj] == kNoPlace ? (const char*)kZeroRow : (const char*)base + place[jj],
                  (void*)(uintptr_t)(tile + (sr + SW * jj) * 1024));
        }
      }
      if (sr == 0) copy_short(exps, uniform((int)(tile + C::TILE)));
    };

    lds_barrier();  // the tiles, sums and page ids before are read
    const int steps = (it1 - it0 + KW - 1) / KW;
    auto tile_of = [&](int s) { return it0 + KW * s + kw; };
    constexpr int kAhead = SW == 1 ? NS : NS - 1;  // tiles on their way at a step's begin
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (tile_of(i) < it1) fetch(tile_of(i), i);
    int st = 0;
    for (int s = 0; s < steps; ++s) {
      const int it = tile_of(s);
      // tile `it` has landed: only the tiles after it may be on their way
      if (tile_of(s + kAhead - 1) < it1) wait_vmem_le<(kAhead - 1) * (NI / SW + (SW == 1))>();
      else wait_vmem();
      asm volatile("" ::: "memory");  // (nothing is read before)
      if constexpr (SW > 1) {
        lds_barrier();  // ... every wave's copies, and the stage before is read
        if (tile_of(s + kAhead) < it1) fetch(tile_of(s + kAhead), st == 0 ? NS - 1 : st - 1);
      }
      if (it < it1) {
        const uint32_t tile = ring + st * C::STAGE;
        f32x4 sc[2], sk[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) sc[b] = sk[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i <= NK; ++i)
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const i32x4 x = *(__attribute__((address_space(3))) const i32x4*)(uintptr_t)(tile + at_k[b] + 64 * i);
            f32x4& acc = i < NK ? sc[b] : sk[b];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const f16x8 k = widen(x[2 * u], x[2 * u + 1]);
              mma16(acc, k, qh[i][u]);
              mma16(acc, k, ql[i][u]);
            }
          }
        // lane: head n, keys 16 b + 4 g + r
        int ec[2][4];
        float z[2][4];
        const int lim = visible - it * kTileKeys - 4 * g;
        const int bad = uniform(s_bad[wave][st]);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const i32x4 x = *(__attribute__((address_space(3))) const i32x4*)(uintptr_t)(tile + C::TILE + 64 * b + 16 * g);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            ec[b][r] = (x[r] & 255) - kScaleBias;
            const int ek = (x[r] >> 8 & 255) - kScaleBias;
            z[b][r] = a.scale_log2 * (__builtin_ldexpf(sc[b][r], ec[b][r] + e_c) + __builtin_ldexpf(sk[b][r], ek + e_k));
          }
        }
        if (lim + 4 * g < kTileKeys || bad) {
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int k = 16 * b + r;
              z[b][r] = k < lim ? (bad >> (k + 4 * g) & 1 ? NAN : z[b][r]) : -INFINITY;
            }
        }
        float m_use = m == -INFINITY ? 0.f : m, most = m == -INFINITY ? INFINITY : -INFINITY;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float over = z[b][r] - m_use;
            most = fmaxf(most, fmaxf(over, over + (float)(ec[b][r] + d)));
          }
        if (__ballot(most > kRise)) {
          // m to the whole number at or above every score, and d so that the largest p 2^(c_j + d) is at most 1
          float top = -INFINITY;
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r) top = fmaxf(top, z[b][r]);
          const float m_new = fmaxf(m, ceilf(quad_max(top)));
          m_use = m_new == -INFINITY ? 0.f : m_new;
          float lift = -1e5f;
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r) lift = fmaxf(lift, z[b][r] - m_use + (float)ec[b][r]);
          int ref = (int)ceilf(fminf(quad_max(lift), 1e5f));
          const float fall = m == -INFINITY ? -INFINITY : m - m_use;  // <= 0
          const int fell = (int)fmaxf(fall, -1e5f);
          if (m != -INFINITY) ref = max(ref, fell - d);
          const float f = m == -INFINITY ? 0.f : __builtin_ldexpf(1.f, fell - ref - d);
          if (m != -INFINITY) lsum = __builtin_ldexpf(lsum, fell);
#pragma unroll
          for (int i = 0; i < NB; ++i) oacc[i] *= f;
          d = -ref;
          m = m_new;
        }
        f16x8 ph, pl;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float p = fast_exp2(z[b][r] - m_use);
            lsum += p;
            const float x = __builtin_ldexpf(p, ec[b][r] + d + kLift);
            ph[4 * b + r] = (_Float16)x;
            if constexpr (FINE) pl[4 * b + r] = (_Float16)(x - (float)ph[4 * b + r]);
          }
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          const i32x2 x = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
              (__attribute__((address_space(3))) i32x2*)(uintptr_t)(tile + at_v[i % 4] + 64 * (i / 4)));
          const f16x8 v = widen(x[0], x[1]);
          mma16(oacc[i], v, ph);
          if constexpr (FINE) mma16(oacc[i], v, pl);
        }
      }
      if constexpr (SW == 1) {
        if (tile_of(s + NS) < it1) {
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this stage is read
          fetch(tile_of(s + NS), st);
        }
      }
      st = st + 1 == NS ? 0 : st + 1;
    }

    // lane: head n, columns 16 i + 4 g + r
    float ltot = quad_sum(lsum);
    int lower = -(d + kLift);
    const bool whole = it0 == 0 && it1 == row_end - row_first;
    if constexpr (KW > 1) {
      // the waves' sums under their common maximum
      lds_barrier();  // every tile is read
      if (g == 0) s_ml[wave][0][n] = m, s_ml[wave][1][n] = ltot;
      lds_barrier();
      float top = -INFINITY;
#pragma unroll
      for (int u = 0; u < KW; ++u) top = fmaxf(top, s_ml[u * SW + sr][0][n]);
      auto factor = [&](float x) { return x == -INFINITY ? 0.f : __builtin_ldexpf(1.f, (int)fmaxf(x - top, -1e5f)); };
      float sum = 0.f;
#pragma unroll
      for (int u = 0; u < KW; ++u) {
        const float lu = s_ml[u * SW + sr][1][n];
        sum += lu == 0.f ? 0.f : lu * factor(s_ml[u * SW + sr][0][n]);
      }
      const float f = factor(m);
      f32x4* sums = (f32x4*)smem;
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        f32x4 x;
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = __builtin_ldexpf(oacc[i][r], lower) * f;
        sums[(wave * NB + i) * 64 + l] = x;
      }
      m = top;
      ltot = sum;
      lds_barrier();
    }
    const int h = h0 + 16 * hg + n;
    const float f = whole ? 1.f / ltot : 1.f;
    if (16 * hg + n < heads) {
      const int64_t place_of = whole ? (int64_t)t * a.H + h : (int64_t)partial_place(w, per, row_first) * a.H + h;
      float* o = (whole ? a.obar : a.part_o) + place_of * a.d_c + 16 * NB * cs + 4 * g;
#pragma unroll
      for (int j = 0; j < NB / KW; ++j) {
        const int i = KW > 1 ? KW * j + kw : j;
        if (16 * (NB * cs + i) >= a.d_c) continue;
        f32x4 x;
        if constexpr (KW > 1) {
          const f32x4* sums = (const f32x4*)smem;
          x = sums[(sr * NB + i) * 64 + l];
#pragma unroll
          for (int u = 1; u < KW; ++u) x += sums[((u * SW + sr) * NB + i) * 64 + l];
        } else {
#pragma unroll
          for (int r = 0; r < 4; ++r) x[r] = __builtin_ldexpf(oacc[j][r], lower);
        }
        *reinterpret_cast<f32x4*>(o + 16 * i) = f32x4{x[0] * f, x[1] * f, x[2] * f, x[3] * f};
      }
      if (kw == 0 && cs == 0 && g == 0) {
        if (!whole) {
          a.part_ml[2 * place_of] = m;
          a.part_ml[2 * place_of + 1] = ltot;
        } else if (a.lse) {
          a.lse[place_of] = (m + fast_log2(ltot)) * kLn2;
        }
      }
    }
    if (at >= end) return;
    share = next_share(a, t, at);
    at = share.first;
    if (at >= end) return;
  }
}

template <int NK, int HG, bool FINE>
__global__ __launch_bounds__(256, 1) void q8_kernel(PagedArgs a, int head_blocks) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[Q8Cfg<NK, HG>::LDS];
  __shared__ int32_t s_ids[4][kIds];
  __shared__ int s_bad[4][8];
  __shared__ float s_ml[4][2][16];
  // the head blocks of a worker follow each other on one XCD: its L2 serves all but the first
  const int id = blockIdx.x, hb = id / 8 % head_blocks, w = id / (8 * head_blocks) * 8 + id % 8;
  const int h0 = hb * a.heads_per_wg;
  q8_shares<NK, HG, FINE>(a, smem, s_ids, s_bad, s_ml, w, h0, min(a.heads_per_wg, a.H - h0), uniform(a.sched[0]), uniform(a.sched[1]));
}

template <int NK, bool FINE>
void launch_q8(const PagedArgs& a, int head_blocks, hipStream_t st) {
  const unsigned wgs = (unsigned)(head_blocks * a.workers);
  if (a.heads_per_wg <= 16) q8_kernel<NK, 1, FINE><<<wgs, 256, 0, st>>>(a, head_blocks);
  else if (NK > 8 || a.heads_per_wg <= 32) q8_kernel<NK, 2, FINE><<<wgs, 256, 0, st>>>(a, head_blocks);
  else if constexpr (NK <= 8) q8_kernel<NK, 4, FINE><<<wgs, 256, 0, st>>>(a, head_blocks);
}

}  // namespace

template <typename T>
void launch_paged_split_q8(const PagedArgs& a, int head_blocks, hipStream_t st) {
  constexpr bool FINE = sizeof(T) == 4;
  if (a.d_c <= 128) launch_q8<2, FINE>(a, head_blocks, st);
  else if (a.d_c <= 256) launch_q8<4, FINE>(a, head_blocks, st);
  else if (a.d_c <= 512) launch_q8<8, FINE>(a, head_blocks, st);
  else launch_q8<16, FINE>(a, head_blocks, st);
}
template void launch_paged_split_q8<bf16>(const PagedArgs&, int, hipStream_t);
template void launch_paged_split_q8<float>(const PagedArgs&, int, hipStream_t);

}  // namespace laga
