// Split attention over a paged cache held in 8 bits: rows of e4m3 numbers, with a power of two for the latent and one
// for the shared key of each position. (paged_attn.hip has the call's other launches.)
//
// The products run on fp16 operands, 16x16x32 at a time: an e4m3 number is an fp16 number, and two fp16 parts of a
// query value, its part of the row (qa or the band) scaled by 2^-e or 2^-f to 2^15 at most, hold 22 bits of it down to 2^-17 of the
// part's largest and 2^-39 of that below (three bf16 parts would hold 24, for half as many products again). With key j's
// powers 2^c_j and 2^k_j
//
//   z_j = scale (2^(c_j + e) A_j + 2^(k_j + f) B_j),  A = 2^-e qa . c8,  B = 2^-f q_rope . k8,  O += (p_j 2^(c_j + d)) c8_j
//
// so the powers never meet a number of 8 bits. A lone wave per SIMD (its registers hold a head group's queries and sums) issues
// an instruction in 4 to 5 cycles, a 16 x 16 product takes the matrix unit 16 and a 32 x 32 one 32: two numbers' conversions
// beside each 16 x 16 product of the scores hide behind it, and O's four behind its pairs of products.
//
// Measured (d_c = 512, d_rope = 64, 578 bytes a key): 64 requests of up to 8192 keys, 16 heads, 47 us, 167 MB at 3.6 TB/s over
// the launch: bound by memory within a share, by the shares' starts and ends else (77 us from a
// cache in bf16). 61 requests, 128 heads: 218 us, 2 requests of up to 100000 keys 113 (169 and 89 in bf16): a step
// of 32 keys and 64 heads takes about 5700 cycles, 2180 of them products; an instruction is issued in 51 % of the cycles, 136
// conversions per wave among them. Tried there and slower, when p was one part and the split took 184 us: four waves to 32
// heads (240), scores beside the products of O (200; its registers are moved about), no gain from fewer exponentials or
// conflicts (there are none). (What a first part leaves, by one mixed fma in place of a conversion and a difference: 0.3 % of a call.)
#define LAGA_LDS_DMA_ASM 1
#include <type_traits>

#include "paged_dev.hpp"

namespace laga {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;
typedef __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 f16x2;
typedef __attribute__((__vector_size__(4 * sizeof(int)))) int i32x4;
typedef __attribute__((__vector_size__(2 * sizeof(int)))) int i32x2;

__device__ __forceinline__ void mma(f32x4& acc, const f16x8& a, const f16x8& b) {
  acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, acc, 0, 0, 0);
}
__device__ __forceinline__ void mma(f32x16& acc, const f16x8& a, const f16x8& b) {
  acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, acc, 0, 0, 0);
}
// e4m3 numbers in fp16, exactly: four of them into elements at .. at + 3, or eight
__device__ __forceinline__ void widen4(f16x8& y, int at, int x) {
  const f16x2 lo = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((unsigned)x, 1.f, false));
  const f16x2 hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((unsigned)x, 1.f, true));
  y[at] = lo[0], y[at + 1] = lo[1], y[at + 2] = hi[0], y[at + 3] = hi[1];
}

// A product of the scores' chains. Written out, because the queries are to stay in accumulation registers, which leaves the
// ordinary ones to O (a rescaled sum would travel from one kind to the other and back); scores_done waits until the
// last are written. (An operand that a vector instruction wrote may be read two wait states after it.)
template <bool FIRST, bool ACC>
__device__ __forceinline__ void score_step(f32x4& s, const f16x8& k, const f16x8& q) {
  if constexpr (FIRST && ACC) asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, 0" : "=&v"(s) : "v"(k), "a"(q));
  else if constexpr (FIRST) asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, 0" : "=&v"(s) : "v"(k), "v"(q));
  else if constexpr (ACC) asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+v"(s) : "v"(k), "a"(q));
  else asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+v"(s) : "v"(k), "v"(q));
}
template <bool FIRST>
__device__ __forceinline__ void score_step(f32x16& s, const f16x8& k, const f16x8& q) {
  if constexpr (FIRST) asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, 0" : "=&v"(s) : "v"(k), "a"(q));
  else asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+v"(s) : "v"(k), "a"(q));
}
__device__ __forceinline__ void scores_done(f32x4 (&a)[2], f32x4 (&b)[2]) {
  asm volatile("s_nop 15\n\ts_nop 3" : "+v"(a[0]), "+v"(a[1]), "+v"(b[0]), "+v"(b[1]));
}
__device__ __forceinline__ void scores_done(f32x16& a, f32x16& b) {
  asm volatile("s_nop 15\n\ts_nop 7" : "+v"(a), "+v"(b));
}

// Rows are NK steps of 64 numbers of the latent and one of the band, zeros up to them. A workgroup's four waves:
// HEADS = 16: KW = 4 tiles of 32 keys are under way at once, one to a wave, in products of 16 x 16; the waves put their
//   sums together at a share's end, and wait for each other nowhere else. Above d_c = 512, where the queries and O do
//   not fit in registers, all four share a tile: each forms all of its scores and has a quarter of O's columns.
// HEADS = 32 or 64: two waves have 32 heads, in products of 32 x 32, for which half as many numbers are widened as for
//   twice 16 heads. They share both products, each with every second half of the contraction and half of O's
//   columns, and exchange partial scores through LDS; with 32 heads two such pairs take a tile each.
// In every form a wave's registers hold its part of the queries, twice, and of O.
template <int NK, int HEADS>
struct Q8Cfg {
  static constexpr bool WIDE = HEADS > 16;
  static constexpr int HG = WIDE ? HEADS / 32 : 1;      // groups of heads
  static constexpr int CS = WIDE ? 2 : NK > 8 ? 4 : 1;  // waves of a group
  static constexpr int SW = HG * CS;                    // waves that share a tile
  static constexpr int KW = 4 / SW;                     // tiles under way at once
  static constexpr int CH = 4 * NK;            // 16-byte chunks of the latent in an LDS row
  static constexpr int RPC = 64 / CH;          // rows of a copy of 64 chunks
  static constexpr int NM = kTileKeys / RPC, NI = NM + 2;  // copies of a tile's latents; with those of its keys
  static constexpr int NJ = (NI + SW - 1) / SW;            // of each wave, at most; NI / SW at least
  static constexpr int BAND = kTileKeys * CH * 16, TILE = BAND + kTileKeys * 64;
  static constexpr int STAGE = TILE + 256;     // the keys' exponents after them
  static constexpr int kParts = WIDE ? 2 * 4 * 64 * 16 * 4 : 0;  // partial scores of two tiles
  static constexpr int kFit = (150 * 1024 - kParts) / STAGE / KW;
  static constexpr int NS = kFit < 8 ? kFit : 8;
  static constexpr int NB = WIDE ? NK : 4 * NK / CS;       // blocks of 32, or 16, columns of a wave
  static constexpr int kO = 4 * NK / (WIDE ? 1 : CS);      // f32x4 of O in a lane
  static constexpr int kRing = KW * NS * STAGE, kSums = KW > 1 ? 4 * kO * 64 * 16 : 0;
  static constexpr int LDS = kRing + kParts > kSums ? kRing + kParts : kSums;
  static_assert(SW * KW == 4 && NS >= (WIDE ? 3 : 2) && !(WIDE && NK > 8));
};
constexpr int kIds = 128;  // page ids of a row that a wave keeps in LDS

// Chunk c of a latent's row r is at c ^ turn(r), of a key's at c ^ band_turn(r). The banks repeat every 16 chunks. In 16 x 16
// products a pass of ds_read_b128 has rows {0 .. 3, 12 .. 15} at a chunk c and {4 .. 11} at c ^ 1, and a pass of the transposing
// 8-byte reads the 16 bytes at c of rows {0 .. 7, 16 .. 23} or the others; in 32 x 32 ones {0 .. 3, 12 .. 15, 20 .. 27} or the
// others at c, and {0 .. 3, 8 .. 11}, or those moved by 4 or 16, at c and c ^ 1. The turns keep each of these apart. They
// are linear in the bits of r, so that the rows of a copy and its number turn separately.
template <int NK, bool WIDE>
__host__ __device__ constexpr int turn(int r) {
  if (WIDE) return NK > 2 ? (r & 3) << 1 | (r >> 2 & 1) | (r & 8) : (r & 2) | (r >> 2 & 1) | (r & 8) >> 1;
  return NK > 2 ? (r & 15) ^ (r & 16) >> 1 : (r >> 1 & 7) ^ (r & 16) >> 2;
}
template <bool WIDE>
__host__ __device__ constexpr int band_turn(int r) {
  return WIDE ? r >> 3 & 3 : (r & 4) >> 1 ^ ((r & 8) >> 3) * 3;
}

// A probability's reference m, a whole number, is raised only where a score passes it by kRise, and p goes into the
// product as p 2^(c_j + d + kLift), d such that no p 2^(c_j + d) passes 2^kRise: 2^14 at most. As two fp16 parts, 22 bits of
// it or 2^-25: one part alone, 11 bits, left 5 to 11 % of the outputs in bf16 a rounding off the nearest (0.1 % now), at 9 % less
// time with 128 heads (205 us of 61 x up to 8192 keys, now 223), the same with 16 (60.0, 60.6).
constexpr float kRise = 8.f;
constexpr int kLift = 6;

// over the lanes of a head: four, or two
template <bool WIDE>
__device__ __forceinline__ float head_max(float x) {
  if (!WIDE) x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
template <bool WIDE>
__device__ __forceinline__ float head_sum(float x) {
  if (!WIDE) x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}
// 2 bytes per lane to LDS, 4 bytes apart
__device__ __forceinline__ void copy_short(const void* g, uint32_t to) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_ushort %0, off" ::"v"(g), "s"(to) : "memory", "m0");
}

// 16 bytes per lane to LDS that nothing else is likely to read (a hint)
__device__ __forceinline__ void copy_past(const void* g, uint32_t to) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" ::"v"(g), "s"(to) : "memory", "m0");
}

template <int N> struct Count { static constexpr int n = N; };
struct __attribute__((aligned(16))) Q8Lds {
  int32_t powers[4][64];  // of a tile's keys, c and then k, for each wave
  int32_t ids[4][kIds];
  int bad[4][8];        // keys of a stage's tile that have no page
  float ml[4][2][32];
};
// The share of worker w, for heads h0 .. h0 + heads (HEADS at most). FULL: d_c = 64 NK and d_rope = 64. PAST: nothing else reads
// the tiles.
template <int NK, int HEADS, bool FULL, bool PAST>
__device__ __forceinline__ void q8_shares(const PagedArgs& a, unsigned char* smem, Q8Lds& lds, int w, int h0, int heads, int per,
                                          int total) {
  using C = Q8Cfg<NK, HEADS>;
  constexpr bool WIDE = C::WIDE;
  constexpr int CS = C::CS, SW = C::SW, KW = C::KW, CH = C::CH, NI = C::NI, NJ = C::NJ, NS = C::NS, NB = C::NB;
  constexpr int GH = WIDE ? 32 : 16;  // heads of a group
  const int l = threadIdx.x & 63, n = l % GH, g = l / GH;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kw = wave / SW, sr = wave % SW, hg = sr % C::HG, cs = sr / C::HG;
  const int d_c = FULL ? 64 * NK : a.d_c, d_rope = FULL ? 64 : a.d_rope, W = d_c + d_rope;
  const int64_t start = (int64_t)w * per;
  if (start >= total) return;
  const int end = (int)min((int64_t)total, start + per);
  Share share = first_share(a, w);
  if (share.first >= end) return;  // (units of no tile)
  const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)smem + kw * NS * C::STAGE;
  int32_t* ids = lds.ids[wave];

  // Of a tile at LDS address x (a multiple of 256), with the row's turn in at_k, at_b and at_v:
  //   16 heads: step i of row 16 b + n of the latents is at ((x + at_k) ^ 64 (i + STEPS / 2 b modulo STEPS)) + 64 (the rest of i) + 16 b
  //     rows, of the keys at x + at_b + 16 b rows; chunk i of this wave's columns in the transposing reads of rows 4 g .. and
  //     16 + 4 g .. at ((x + at_v) ^ 16 (i modulo TURNS)) + 16 (the rest of i)
  //   32: step i of this wave's half of row n at ((x + at_k) ^ 32 i), of the keys at x + at_b; chunks 2 i and 2 i + 1 of this
  //     wave's columns in those of rows 16 k + 4 g .. and 16 k + 8 + 4 g .. at ((x + at_v) ^ 32 i) + 16 k rows
  constexpr int TURNS = NK > 2 ? 16 : 8, STEPS = TURNS / 4;
  constexpr bool BAND_ACC = NK <= 8;  // (the latent's queries alone fill the accumulation registers above)
  // Of this wave's jj-th copy, of RPC latents' rows: this lane's row is at_src + jj SW RPC, its chunk at_copy with the turn of
  // jj SW RPC; of a copy of 16 rows of keys at_key_src and at_band.
  uint32_t at_k, at_b, at_v, at_copy, at_band;
  int at_src, at_key_src;
  {
    const int q = l & 15;
    if constexpr (WIDE) {
      const int vr = 4 * g + (q >> 1 & 3) + 8 * (q >> 3), first = 2 * NK * cs, turned = first % TURNS, rest = first - turned;
      at_k = n * CH * 16 + ((turned + g ^ turn<NK, WIDE>(n)) + rest) * 16;
      at_b = C::BAND + n * 64 + ((2 * cs + g ^ band_turn<WIDE>(n)) * 16);
      at_v = vr * CH * 16 + ((turned + (l >> 4 & 1) ^ turn<NK, WIDE>(vr)) + rest) * 16 + 8 * (q & 1);
    } else {
      const int vr = 4 * g + (q >> 1 & 3) + 16 * (q >> 3);
      at_k = n * CH * 16 + ((g ^ turn<NK, WIDE>(n)) * 16);
      at_b = C::BAND + n * 64 + ((g ^ band_turn<WIDE>(n)) * 16);
      at_v = vr * CH * 16 + (turn<NK, WIDE>(vr) * 16) + 8 * (q & 1) + cs * NB * 16;
    }
    at_src = sr * C::RPC + l / CH;
    at_copy = (l % CH ^ turn<NK, WIDE>(at_src)) * 16;
    at_key_src = (sr & 1) * 16 + (l >> 2);
    at_band = d_c + min(((l & 3) ^ band_turn<WIDE>(at_key_src)) * 16, d_rope - 16);
  }

  for (int at = max((int)start, share.first);;) {
    const int t = share.t, row_first = share.first, row_end = share.end;
    const int it0 = at - row_first, it1 = min(end, row_end) - row_first;
    at = min(end, row_end);
    const int visible = min((int64_t)share.visible, (int64_t)it1 * kTileKeys);  // to the end of this share
    const int32_t* pages = a.table + (int64_t)share.request * a.width;

    float m = -INFINITY, lsum = 0.f;
    float rise = -INFINITY;  // kRise, once there is a reference
    int d = 0;

    int win = 0, win_end = 0;  // first page of the window, and the first key past it
    auto page_of = [&](int key) { return (int)((uint64_t)(uint32_t)key * a.page_magic >> a.page_shift); };
    // The copies of a tile. A key past the share's end, or without a page (bad), is copied from zeros. look: the page of
    // key l % 32; ready: where the copies come from and go; copy: the jj-th of this wave's, and with the first the keys'
    // exponents. (Chunks past a row's end repeat its last one: they meet zeros of the queries, and columns that are not
    // stored.)
    int look_id, look_pg;
    auto look = [&](int it) {
      const int k0 = it * kTileKeys;
      if (min(k0 + kTileKeys, visible) > win_end) {
        win = page_of(k0);
        win_end = (int)min((int64_t)(win + kIds) * a.page, (int64_t)INT32_MAX);
        const int have = page_of(visible - 1) + 1;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = fresh_lane(); i < kIds; i += 64) ids[i] = win + i < have ? pages[win + i] : -1;
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
      const int key = k0 + (fresh_lane() & 31);
      look_pg = key < visible ? page_of(key) : win;
      look_id = ids[look_pg - win];
    };
    bool asking = false;
    int src_lo = 0, src_hi = 0;  // where row l % 32 is
    int row_lo = 0, row_hi = 0;  // and this lane's row of the next copy
    uint32_t to = 0;
    constexpr int MAIN = C::NM / SW;  // of this wave's copies, those of latents
    static_assert(C::NM % SW == 0);
    auto next_row = [&](int jj) {
      const int r = jj < MAIN ? at_src + jj * SW * C::RPC : at_key_src + (SW == 1 ? (jj - MAIN) * 16 : 0);
      row_lo = __builtin_amdgcn_ds_bpermute(4 * r, src_lo);
      row_hi = __builtin_amdgcn_ds_bpermute(4 * r, src_hi);
    };
    auto ready = [&](int it, int stage) {
      const int key = it * kTileKeys + (fresh_lane() & 31);
      const bool live = key < visible, ok = live && (unsigned)look_id < (unsigned)a.n_pages;
      const int off = key - look_pg * a.page;
      const uintptr_t src = ok ? (uintptr_t)a.cache + (int64_t)look_id * a.page_stride + (int64_t)off * W : (uintptr_t)kZeroRow;
      src_lo = (int)(uint32_t)src;
      src_hi = (int)(uint32_t)(src >> 32);
      lds.bad[wave][stage] = (int)(uint32_t)__ballot(live && !ok);  // (the same from every lane)
      to = ring + stage * C::STAGE + sr * 1024;
      if (sr == 0)
        copy_short(ok ? (const char*)a.scales + 2 * ((int64_t)look_id * a.page + off) : (const char*)kZeroRow, uniform((int)(to + C::TILE)));
      next_row(0);
      asking = true;
    };
    auto copy = [&](int jj) {
      if (!asking || (SW == 4 && jj == MAIN && sr > 1)) return;
      const uint32_t chunk = at_copy ^ (turn<NK, WIDE>(jj * SW * C::RPC) * 16);
      const uint32_t off = jj < MAIN ? (FULL ? chunk : min(chunk, (uint32_t)d_c - 16)) : at_band;
      const uintptr_t row = (uintptr_t)(uint32_t)row_lo | ((uintptr_t)(uint32_t)row_hi << 32);
      const char* from = (const char*)row + off;
      const int at = (int)(to + SW * jj * 1024);
      if constexpr (PAST) copy_past(from, uniform(at));
      else g2lds16(from, (void*)(uintptr_t)(uint32_t)at);
      if (jj + 1 < NJ) next_row(jj + 1);
    };

    lds_barrier();  // the tiles, sums and page ids before are read
    const int steps = SW == 1 ? (it1 - it0 - kw + KW - 1) / KW : (it1 - it0 + KW - 1) / KW;
    // (with more than one wave to a tile, a last one perhaps past the share's end: rows of zeros without weight)
    auto tile_of = [&](int s) { return it0 + KW * s + kw; };
    // Tile s has landed: only the AFTER tiles that were asked for after it may be on their way.
    auto landed = [&](int s, auto after) {
      constexpr int AFTER = decltype(after)::n;
      if (s + AFTER < steps) wait_vmem_le<AFTER * (NI / SW + (SW == 1))>();
      else wait_vmem();
      if constexpr (SW > 1) lds_barrier();  // every wave's copies (and partial scores)
      else asm volatile("" ::: "memory");   // (nothing is read before)
    };
    // The queries of head n, each part scaled by 2^-e of its own to 2^14 .. 2^15 at most: of step i and half u elements 64 i + 16 g
    // + 8 u .., or of this wave's half 32 i + 16 g + 8 u ... They are read first, and widened while the first tiles are on their way.
    f16x8 qh[NK + 1][2], ql[NK + 1][2];
    int ec = 0, ek = 0;
    if (steps > 0) {
      const int64_t th = (int64_t)t * a.H + h0 + min(GH * hg + n, heads - 1);
      const int blocks = qa_blocks(d_c);
      const float* tops = a.qa_max + th * blocks;
      const f32x4* q = (const f32x4*)a.qa + (int64_t)t * (W / 4) * a.H + (th - (int64_t)t * a.H);
      auto at = [&](int i, int u) { return (WIDE ? 32 * (i < NK ? NK * cs + i : cs) : i < NK ? 64 * i : 0) + 16 * g + 8 * u; };
      auto there = [&](int i, int u) { return FULL || at(i, u) < (i < NK ? d_c : d_rope); };
      constexpr int TURN = 9;  // steps whose numbers are on their way at once
      f32x4 x[TURN][2][2];
      auto read = [&](int i0) {
#pragma unroll
        for (int i = i0; i < min(i0 + TURN, NK + 1); ++i)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const f32x4* from = q + (((i < NK ? 0 : d_c) + (there(i, u) ? at(i, u) : 0)) >> 2) * a.H;
            x[i - i0][u][0] = from[0];
            x[i - i0][u][1] = from[a.H];
          }
      };
      float top = 0.f;
      for (int i = 0; i < blocks - 1; ++i) top = fmaxf(top, tops[i]);
      const float band_top = tops[blocks - 1];
      read(0);
      look(tile_of(0));
      wait_vmem();
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll 1
      for (int i = 0; i < min(NS, steps); ++i) {
        if (i > 0) look(tile_of(i));
        ready(tile_of(i), i);
#pragma unroll
        for (int jj = 0; jj < NJ; ++jj) copy(jj);
      }
      asking = false;
      ec = top > 0.f ? __builtin_amdgcn_frexp_expf(top) - 15 : 0;
      ek = band_top > 0.f ? __builtin_amdgcn_frexp_expf(band_top) - 15 : 0;
#pragma unroll
      for (int i0 = 0; i0 <= NK; i0 += TURN) {
        if (i0 > 0) read(i0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = i0; i < min(i0 + TURN, NK + 1); ++i)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            typedef float f32x8 __attribute__((ext_vector_type(8)));
            const int up = there(i, u) ? -(i < NK ? ec : ek) : -1000;  // (to zero)
            f32x8 y, rest;
#pragma unroll
            for (int k = 0; k < 8; ++k) y[k] = __builtin_ldexpf(x[i - i0][u][k >> 2][k & 3], up);
            qh[i][u] = __builtin_convertvector(y, f16x8);
#pragma unroll
            for (int k = 0; k < 8; ++k) rest[k] = y[k] - (float)qh[i][u][k];
            ql[i][u] = __builtin_convertvector(rest, f16x8);
            if (i < NK || BAND_ACC) asm volatile("" : "+a"(qh[i][u]), "+a"(ql[i][u]));  // (whole)
            else asm volatile("" : "+v"(qh[i][u]), "+v"(ql[i][u]));
            __builtin_amdgcn_sched_barrier(0);
          }
      }
    }
    typedef std::conditional_t<WIDE, f32x16, f32x4> acc_t;
    acc_t oacc[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) oacc[i] = acc_t{};
    int st = 0;
    uint32_t tile = ring;
    constexpr int NZ = WIDE ? 16 : 8;  // scores of a lane
    i32x4 pc[NZ / 4];                  // c of their keys
    float z[NZ], p[NZ], x[NZ];
    // The powers are added up first, so that nothing passes fp32's range but a score that does
    auto score = [&](float A, int c, float B, int k) { return __builtin_ldexpf(A, c + ec) + __builtin_ldexpf(B, k + ek); };
    // this lane's r-th score is of key
    auto key_of = [&](int r) { return (WIDE ? 8 : 16) * (r >> 2) + 4 * g + (r & 3); };
    // Scores of tile s into p and what goes into the product, x, under the reference, which is raised where need be.
    auto weigh = [&](int s, int bad) {
      const int lim = visible - tile_of(s) * kTileKeys;
      if (lim < kTileKeys || bad) {
#pragma unroll
        for (int r = 0; r < NZ; ++r) z[r] = key_of(r) < lim ? (bad >> key_of(r) & 1 ? NAN : z[r]) : -INFINITY;
      }
      float most_t = -INFINITY, most_x = 0.f;
      auto under = [&](float m_use, int lift) {
#pragma unroll
        for (int r = 0; r < NZ; ++r) {
          const float t = __builtin_fmaf(z[r], a.scale_log2, -m_use);
          most_t = fmaxf(most_t, t);
          p[r] = fast_exp2(t);
          x[r] = __builtin_ldexpf(p[r], pc[r >> 2][r & 3] + lift);
          most_x = fmaxf(most_x, x[r]);
        }
      };
      under(m == -INFINITY ? 0.f : m, d + kLift);
      if (__ballot(most_t > rise || most_x > 0x1p14f)) {
        // m to the whole number at or above every score, and d so that the largest p 2^(c_j + d) is 1 at most
        float top = -INFINITY;
#pragma unroll
        for (int r = 0; r < NZ; ++r) top = fmaxf(top, z[r] * a.scale_log2);
        const float m_new = fmaxf(m, ceilf(head_max<WIDE>(top))), m_use = m_new == -INFINITY ? 0.f : m_new;
        float lift = -1e5f;
#pragma unroll
        for (int r = 0; r < NZ; ++r)
          lift = fmaxf(lift, __builtin_fmaf(z[r], a.scale_log2, -m_use) + (float)(pc[r >> 2][r & 3] + 1));
        int ref = (int)ceilf(fminf(head_max<WIDE>(lift), 1e5f));
        const int fell = m == -INFINITY ? -100000 : (int)fmaxf(m - m_use, -1e5f);
        if (m != -INFINITY) {
          ref = max(ref, fell - d);
          lsum = __builtin_ldexpf(lsum, fell);
        }
        ref = min(max(ref, -120), 129);
        const float f = m == -INFINITY ? 0.f : __builtin_ldexpf(1.f, fell - ref - d);
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          oacc[i] *= f;
          if (WIDE || i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
        d = -ref;
        m = m_new;
        rise = m == -INFINITY ? -INFINITY : kRise;
        under(m_use, d + kLift);
      }
#pragma unroll
      for (int r = 0; r < NZ; r += 4) lsum += (p[r] + p[r + 1]) + (p[r + 2] + p[r + 3]);
    };
    // eight of them as an operand, and what its rounding left
    auto operand = [&](int first, f16x8& hi, f16x8& lo) {
      typedef float f32x8 __attribute__((ext_vector_type(8)));
      f32x8 y;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = x[first + e];
      hi = __builtin_convertvector(y, f16x8);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] -= (float)hi[e];
      lo = __builtin_convertvector(y, f16x8);
    };
    // The keys' powers, by way of LDS to the lanes that need them; of which one is NaN (byte 255)
    auto give_powers = [&](int exps) {
      const int b = l < 32 ? exps & 255 : exps >> 8 & 255;
      lds.powers[wave][l] = b - kScaleBias;
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      const uint64_t nan = __ballot(b == 255);
      return (int)((uint32_t)nan | (uint32_t)(nan >> 32));
    };
    auto powers = [&](int of, int r) { return *reinterpret_cast<const i32x4*>(&lds.powers[wave][32 * of + key_of(r)]); };
    auto raw_at = [&](uint32_t at) { return *(__attribute__((address_space(3))) const i32x4*)(uintptr_t)at; };
    auto columns_at = [&](uint32_t at) { return __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2*)(uintptr_t)at); };
    constexpr int PER = (NJ + NK) / (NK + 1);  // copies beside a step
    static_assert(PER == 1 || PER == 2);
    int exps, bads;
    auto tile_first = [&]() {
      exps = *(__attribute__((address_space(3))) const int*)(uintptr_t)(tile + C::TILE + 4 * (fresh_lane() & 31));
      bads = lds.bad[wave][st];
    };
    // the copies of step s are those of the tile that takes the place of the one before its own
    auto ask = [&](int s) {
      if (s > 0 && s - 1 + NS < steps) ready(tile_of(s - 1 + NS), st == 0 ? NS - 1 : st - 1);
      else asking = false;
    };

    if constexpr (!WIDE) {
      auto k_read = [&](int i, int b) {
        return raw_at(i < NK ? ((tile + at_k) ^ (64 * ((i + b * STEPS / 2) % STEPS))) + 64 * (i / STEPS * STEPS) + 16 * b * CH * 16
                             : tile + at_b + 16 * b * 64);
      };
      auto v_read = [&](int i) { return columns_at(((tile + at_v) ^ (16 * (i % TURNS))) + 16 * (i / TURNS * TURNS)); };
      constexpr int RA = NK > 2 ? 3 : 2;  // steps whose numbers are on their way
      i32x4 raw[RA][2];
      auto k_first = [&]() {
#pragma unroll
        for (int i = 0; i < RA; ++i)
#pragma unroll
          for (int b = 0; b < 2; ++b) raw[i][b] = k_read(i, b);
        tile_first();
      };
      if (steps > 0) {
        landed(0, Count<NS - 1>{});
        k_first();
      }
      for (int s = 0; s < steps; ++s) {
        // Scores, step by step: beside the eight products of one step the next one's numbers are widened, later ones'
        // read, and now and then a copy is asked for.
        int bad = uniform(bads);
        ask(s);
        f32x4 sc[2], sk[2];
        i32x4 pk[2];
        f16x8 k[2][2][2];
#pragma unroll
        for (int j = 0; j < 8; ++j) widen4(k[0][j >> 2][j >> 1 & 1], 4 * (j & 1), raw[0][j >> 2][j & 3]);
        asm volatile("s_nop 1" : "+v"(k[0][0][0]), "+v"(k[0][1][0]), "+v"(k[0][0][1]), "+v"(k[0][1][1]));
#pragma unroll
        for (int i = 0; i <= NK; ++i) {
          f32x4(&acc)[2] = i < NK ? sc : sk;
          if (i + RA <= NK)
#pragma unroll
            for (int b = 0; b < 2; ++b) raw[i % RA][b] = k_read(i + RA, b);
          if (i == 0) {
            bad |= give_powers(exps);
          } else if (i == 1) {
#pragma unroll
            for (int b = 0; b < 2; ++b) pc[b] = powers(0, 4 * b), pk[b] = powers(1, 4 * b);
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int b = j & 1, u = j >> 2;
            const f16x8& q = j >> 1 & 1 ? ql[i][u] : qh[i][u];
            if (j < 2 && i == NK) score_step<true, BAND_ACC>(acc[b], k[i & 1][b][u], q);
            else if (i == NK) score_step<false, BAND_ACC>(acc[b], k[i & 1][b][u], q);
            else if (j < 2 && i == 0) score_step<true, true>(acc[b], k[i & 1][b][u], q);
            else score_step<false, true>(acc[b], k[i & 1][b][u], q);
            if (i < NK) {
              f16x8& y = k[i + 1 & 1][j >> 2][j >> 1 & 1];
              widen4(y, 4 * (j & 1), raw[(i + 1) % RA][j >> 2][j & 3]);
              if (j & 1) asm volatile("" : "+v"(y));  // (here, not where it is used)
            }
            __builtin_amdgcn_sched_barrier(0);
            if (j % (8 / PER) == 8 / PER - 1 && PER * i + j / (8 / PER) < NJ) copy(PER * i + j / (8 / PER));
          }
        }
        // O's first numbers, on their way beside the softmax
        constexpr int AHEAD = 4;
        i32x2 vr[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) vr[i] = v_read(i);
        scores_done(sc, sk);
#pragma unroll
        for (int r = 0; r < 8; ++r) z[r] = score(sc[r >> 2][r & 3], pc[r >> 2][r & 3], sk[r >> 2][r & 3], pk[r >> 2][r & 3]);
        weigh(s, bad);
        f16x8 ph, pl, v[2];
        operand(0, ph, pl);
        // O's products likewise, the numbers read AHEAD of them; when the tile's last are, the next tile's first
        widen4(v[0], 0, vr[0][0]);
        widen4(v[0], 4, vr[0][1]);
        auto o_step = [&](int i) {
          if (i + AHEAD < NB) vr[i % AHEAD] = v_read(i + AHEAD);
          mma(oacc[i], v[i & 1], ph);
          if (i + 1 < NB) {
            widen4(v[i + 1 & 1], 0, vr[(i + 1) % AHEAD][0]);
            widen4(v[i + 1 & 1], 4, vr[(i + 1) % AHEAD][1]);
          }
          mma(oacc[i], v[i & 1], pl);
          __builtin_amdgcn_sched_barrier(0);
        };
#pragma unroll
        for (int i = 0; i < NB - AHEAD; ++i) o_step(i);
        if (s + 1 < steps) {
          if constexpr (SW == 1) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this stage is read
          landed(s + 1, Count<NS - 2>{});  // (and by every wave)
          st = st + 1 == NS ? 0 : st + 1;
          tile = ring + st * C::STAGE;
          k_first();
          if (s + NS < steps) look(tile_of(s + NS));
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = NB - AHEAD; i < NB; ++i) o_step(i);
      }
    } else {
      f32x4* parts = (f32x4*)(smem + C::kRing);
      auto k_read = [&](int i) { return raw_at(i < NK ? (tile + at_k) ^ (32 * i) : tile + at_b); };
      constexpr int RA = 3;
      i32x4 raw[RA];
      auto k_first = [&]() {
#pragma unroll
        for (int i = 0; i < RA; ++i) raw[i] = k_read(i);
        tile_first();
      };
      // This wave's half of a tile's scores to z and to the other wave, as above.
      auto scores = [&](int turn_of) {
        f32x16 sc, sk;
        i32x4 pk[4];
        f16x8 k[2][2];
#pragma unroll
        for (int j = 0; j < 4; ++j) widen4(k[0][j >> 1], 4 * (j & 1), raw[0][j]);
        asm volatile("s_nop 1" : "+v"(k[0][0]), "+v"(k[0][1]));
#pragma unroll
        for (int i = 0; i <= NK; ++i) {
          f32x16& acc = i < NK ? sc : sk;
          if (i + RA <= NK) raw[i % RA] = k_read(i + RA);
          if (i == 0) {
            bads |= give_powers(exps);
          } else if (i == 1) {
#pragma unroll
            for (int r = 0; r < 4; ++r) pc[r] = powers(0, 4 * r), pk[r] = powers(1, 4 * r);
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const f16x8& q = j & 1 ? ql[i][j >> 1] : qh[i][j >> 1];
            if (j == 0 && (i == 0 || i == NK)) score_step<true>(acc, k[i & 1][j >> 1], q);
            else score_step<false>(acc, k[i & 1][j >> 1], q);
            if (i < NK) {
              f16x8& y = k[i + 1 & 1][j >> 1];
              widen4(y, 4 * (j & 1), raw[(i + 1) % RA][j]);
              if (j & 1) asm volatile("" : "+v"(y));  // (here, not where it is used)
            }
            __builtin_amdgcn_sched_barrier(0);
            if (j % (4 / PER) == 4 / PER - 1 && PER * i + j / (4 / PER) < NJ) copy(PER * i + j / (4 / PER));
          }
        }
        scores_done(sc, sk);
#pragma unroll
        for (int r = 0; r < 16; ++r) z[r] = score(sc[r], pc[r >> 2][r & 3], sk[r], pk[r >> 2][r & 3]);
#pragma unroll
        for (int r = 0; r < 4; ++r) parts[((turn_of * 4 + wave) * 4 + r) * 64 + l] = f32x4{z[4 * r], z[4 * r + 1], z[4 * r + 2], z[4 * r + 3]};
      };
      if (steps > 0) {
        landed(0, Count<NS - 1>{});
        k_first();
        asking = false;
        scores(0);
        landed(1, Count<NS - 2>{});
      }
      // Step s: tile s's weights and O, then the scores of the tile after it, whose copies have landed.
      for (int s = 0; s < steps; ++s) {
        const int bad = uniform(bads), other = wave ^ C::HG;
        f32x4 theirs[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) theirs[r] = parts[(((s & 1) * 4 + other) * 4 + r) * 64 + l];
        constexpr int AHEAD = 4;
        auto v_read = [&](int i) { return columns_at(((tile + at_v) ^ (32 * (i % NB))) + i / NB * 16 * CH * 16); };
        i32x2 vr[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) vr[i] = v_read(i);
#pragma unroll
        for (int r = 0; r < 16; ++r) z[r] += theirs[r >> 2][r & 3];
        weigh(s, bad);
        f16x8 ph[2], pl[2], v[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) operand(8 * k, ph[k], pl[k]);
        widen4(v[0], 0, vr[0][0]);
        widen4(v[0], 4, vr[0][1]);
#pragma unroll
        for (int i = 0; i < 2 * NB; ++i) {
          if (i + AHEAD < 2 * NB) vr[i % AHEAD] = v_read(i + AHEAD);
          mma(oacc[i % NB], v[i & 1], ph[i / NB]);
          if (i + 1 < 2 * NB) {
            widen4(v[i + 1 & 1], 0, vr[(i + 1) % AHEAD][0]);
            widen4(v[i + 1 & 1], 4, vr[(i + 1) % AHEAD][1]);
          }
          mma(oacc[i % NB], v[i & 1], pl[i / NB]);
          __builtin_amdgcn_sched_barrier(0);
        }
        if (s + 1 < steps) {
          const int was = st;
          st = st + 1 == NS ? 0 : st + 1;
          tile = ring + st * C::STAGE;
          k_first();
          // (the place of tile s - 1 is free: every wave has passed the barrier after it)
          if (s > 0 && s - 1 + NS < steps) ready(tile_of(s - 1 + NS), was == 0 ? NS - 1 : was - 1);
          else asking = false;
          scores(s + 1 & 1);
          if (s + NS < steps) look(tile_of(s + NS));
          landed(s + 2, Count<NS - 3>{});
        }
      }
    }

    // lane: head n, columns 16 i + 4 g + r of its wave's, or 32 i + 8 (r / 4) + 4 g + r % 4: O's f32x4 number j
    float ltot = head_sum<WIDE>(lsum);
    const int lower = -(d + kLift);
    auto quad_of = [&](int j) {
      if constexpr (WIDE) return f32x4{oacc[j >> 2][4 * (j & 3)], oacc[j >> 2][4 * (j & 3) + 1], oacc[j >> 2][4 * (j & 3) + 2], oacc[j >> 2][4 * (j & 3) + 3]};
      else return oacc[j];
    };
    const bool whole = it0 == 0 && it1 == row_end - row_first;
    const int h = h0 + GH * hg + n;
    const int64_t place_of = whole ? (int64_t)t * a.H + h : (int64_t)partial_place(w, per, row_first) * a.H + h;
    float* o = (whole ? a.obar : a.part_o) + place_of * d_c + 4 * g;
    auto column_of = [&](int j) { return WIDE ? 32 * (NB * cs + (j >> 2)) + 8 * (j & 3) : 16 * (NB * cs + j); };
    if (KW > 1 && it1 - it0 > 1) {
      // the waves' sums under their common maximum (a lone tile is the first wave's: 2.7 us less for 1000 keys, 16 heads, 10.9 now)
      f32x4* sums = (f32x4*)smem;
      lds_barrier();  // every tile is read
      if (g == 0) lds.ml[wave][0][n] = m, lds.ml[wave][1][n] = ltot;
      lds_barrier();
      float top = -INFINITY;
#pragma unroll
      for (int u = 0; u < KW; ++u) top = fmaxf(top, lds.ml[u * SW + sr][0][n]);
      auto factor = [&](float x) { return x == -INFINITY ? 0.f : __builtin_ldexpf(1.f, (int)fmaxf(x - top, -1e5f)); };
      float sum = 0.f;
#pragma unroll
      for (int u = 0; u < KW; ++u) {
        const float lu = lds.ml[u * SW + sr][1][n];
        sum += lu == 0.f ? 0.f : lu * factor(lds.ml[u * SW + sr][0][n]);
      }
      const float mine = __builtin_ldexpf(factor(m), lower);
#pragma unroll
      for (int j = 0; j < C::kO; ++j) sums[(wave * C::kO + j) * 64 + l] = quad_of(j) * mine;
      m = top;
      ltot = sum;
      const float f = whole ? 1.f / ltot : 1.f;
      lds_barrier();
      if (GH * hg + n < heads) {
#pragma unroll
        for (int i = 0; i < C::kO / KW; ++i) {
          const int j = KW * i + kw;
          if (!FULL && column_of(j) >= d_c) continue;
          f32x4 y = sums[(sr * C::kO + j) * 64 + l];
#pragma unroll
          for (int u = 1; u < KW; ++u) y += sums[((u * SW + sr) * C::kO + j) * 64 + l];
          *reinterpret_cast<f32x4*>(o + column_of(j)) = f32x4{y[0] * f, y[1] * f, y[2] * f, y[3] * f};
        }
      }
    } else if (kw == 0 && GH * hg + n < heads) {
      const float f = __builtin_ldexpf(whole ? 1.f / ltot : 1.f, lower);
#pragma unroll
      for (int j = 0; j < C::kO; ++j)
        if (FULL || column_of(j) < d_c) *reinterpret_cast<f32x4*>(o + column_of(j)) = quad_of(j) * f;
    }
    if (kw == 0 && cs == 0 && g == 0 && GH * hg + n < heads) {
      if (!whole) {
        a.part_ml[2 * place_of] = m;
        a.part_ml[2 * place_of + 1] = ltot;
      } else if (a.lse) {
        a.lse[place_of] = (m + fast_log2(ltot)) * kLn2;
      }
    }
    if (at >= end) return;
    share = next_share(a, t, at);
    at = share.first;
    if (at >= end) return;
  }
}

template <int NK, int HEADS, bool FULL>
__global__ __launch_bounds__(256, 1) void q8_kernel(PagedArgs a, int head_blocks) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[Q8Cfg<NK, HEADS>::LDS];
  __shared__ Q8Lds lds;
  // the head blocks of a worker follow each other on one XCD: its L2 serves all but the first
  const int id = blockIdx.x, hb = id / 8 % head_blocks, w = id / (8 * head_blocks) * 8 + id % 8;
  const int h0 = hb * a.heads_per_wg;
  const int heads = min(a.heads_per_wg, a.H - h0), per = uniform(a.sched[0]), total = uniform(a.sched[1]);
  // Copies past the caches (a hint), where no other row of the request and no other head block reads the tiles again. Us of a call
  // with it and without: 64 rows x up to 8192 keys, 16 heads 59 and 65, 256 x up to 4000, 8 heads 97 and 104, as in a model whose
  // other layers' caches are read in between; where the same cache is read call after call, from the last-level
  // cache, 41 and 39.5 (53 MB, 16 heads), 60 and 58 (106 MB, 8 heads), 60.3 and 57.4 (167 MB, 16 heads).
  if constexpr (HEADS <= 16 && NK <= 8)
    if (uniform(a.sched[4]) == 0 && heads == a.H) return q8_shares<NK, HEADS, FULL, true>(a, smem, lds, w, h0, heads, per, total);
  q8_shares<NK, HEADS, FULL, false>(a, smem, lds, w, h0, heads, per, total);
}

template <int NK, bool FULL>
void launch_q8(const PagedArgs& a, int head_blocks, hipStream_t st) {
  const unsigned wgs = (unsigned)(head_blocks * a.workers);
  if (a.heads_per_wg <= 16) q8_kernel<NK, 16, FULL><<<wgs, 256, 0, st>>>(a, head_blocks);
  else if constexpr (NK <= 8) {
    if (a.heads_per_wg <= 32) q8_kernel<NK, 32, FULL><<<wgs, 256, 0, st>>>(a, head_blocks);
    else q8_kernel<NK, 64, FULL><<<wgs, 256, 0, st>>>(a, head_blocks);
  }
}
// Widths that fill the steps need no care at a row's end. Us of a call with it and without: 1 x 1000 keys, 16 heads 20.9 and 22.2; 64 x
// up to 8192, 16 heads 59.0 and 60.6; 256 x up to 4000, 8 heads 95.9 and 98.4; with 128 heads no difference.
template <int NK>
void launch_q8(const PagedArgs& a, int head_blocks, hipStream_t st) {
  if (a.d_c == 64 * NK && a.d_rope == 64) launch_q8<NK, true>(a, head_blocks, st);
  else launch_q8<NK, false>(a, head_blocks, st);
}

}  // namespace

void launch_paged_split_q8(const PagedArgs& a, int head_blocks, hipStream_t st) {
  if (a.d_c <= 128) launch_q8<2>(a, head_blocks, st);
  else if (a.d_c <= 256) launch_q8<4>(a, head_blocks, st);
  else if (a.d_c <= 512) launch_q8<8>(a, head_blocks, st);
  else launch_q8<16>(a, head_blocks, st);
}

}  // namespace laga
