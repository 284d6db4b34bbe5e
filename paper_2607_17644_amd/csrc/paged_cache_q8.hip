// Rows of a paged cache held in 8 bits: written as they are quantised, and read back.
//
// Of each part x of a row (the normalised latent, the rotated key), with a its largest finite magnitude:
//   e = the least whole number with a <= 448 2^e (448 the largest e4m3 number), kLeastScale at least, kMostScale at most
//   byte j = e4m3(x_j 2^-e), to nearest, ties to even, at most 448 in magnitude; NaN where x_j is no finite number
// A power of two leaves every bit of the mantissa to the number, and its product with one is exact in bf16 and fp32.
#include <type_traits>

#include "common.hpp"
#include "paged.hpp"

namespace laga {
namespace {

typedef __attribute__((__vector_size__(2 * sizeof(int)))) int i32x2;
typedef __attribute__((__vector_size__(4 * sizeof(int)))) int i32x4;

// The row is formed in double precision: half a step of e4m3 decides over an eighth of the value, and in single precision
// some 40 of the 9.4 million bytes of 16384 tokens fall to the other side. What bounds a prompt's append is therefore its
// vector instructions (632 a wave of two tokens, in 67 % of the cycles): 16384 tokens 16.8 us, 19.5 before the place
// below (which was the number's bits shifted into fp32's), the largest magnitude in place of the largest exponent and the
// band's frequencies from the host; 13.0 to a cache in bf16. (Single precision with a check for numbers
// that are near such a place, and double for rows that have one, took 20.)
// The e of one number alone: of a part, the largest of its numbers'.
__device__ __forceinline__ int exponent_of(double x) {
  const uint64_t u = (uint64_t)__builtin_bit_cast(int64_t, x) & ~((uint64_t)1 << 63);
  const int e = (int)(u >> 52);
  return e == 2047 ? kLeastScale : e - 1023 - 8 + ((u & (((uint64_t)1 << 52) - 1)) > (uint64_t)3 << 50);
}
// x 2^-e at the nearest e4m3 number, even at ties: its last place is an eighth of its leading one, 2^-9 at least, and a
// sum with 1.5 2^52 of that place ends there. ANY: x may be infinite, or above 448 2^e.
template <bool ANY>
__device__ __forceinline__ float eighth(double x, double down) {
  const double y = x * down;
  const uint32_t hi = (uint32_t)((uint64_t)__builtin_bit_cast(int64_t, y) >> 32);
  const double place = __builtin_bit_cast(double, (uint64_t)(max(hi & 0x7ff00000u, (1023u - 6) << 20) + (49u << 20 | 1u << 19)) << 32);
  float f = (float)((y + place) - place);
  if constexpr (ANY) f = !(__builtin_fabs(y) < __builtin_inf()) ? __builtin_nanf("") : __builtin_amdgcn_fmed3f(f, -448.f, 448.f);
  return __builtin_copysignf(f, __builtin_bit_cast(float, hi));
}
template <bool ANY>
__device__ __forceinline__ int four(const double* x, double down) {
  int y = __builtin_amdgcn_cvt_pk_fp8_f32(eighth<ANY>(x[0], down), eighth<ANY>(x[1], down), 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(eighth<ANY>(x[2], down), eighth<ANY>(x[3], down), y, true);
}
__device__ __forceinline__ int within(int e) { return min(max(e, kLeastScale), kMostScale); }

constexpr int kWaves = 4;  // per workgroup
// A wave per token and turn, a chunk of 8 numbers per lane (CH above 512); then its lanes take a pair of the
// shared key each, of 64 / (d_rope / 2) tokens at a time.
template <typename T, int TPW, int CH>
__global__ __launch_bounds__(64 * kWaves) void append_q8_kernel(AppendQ8Args args) {
  const AppendArgs& a = args.a;
  const int l = threadIdx.x & 63;
  const int64_t t0 = ((int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6)) * TPW;
  if (t0 >= a.T) return;  // wave-uniform; the kernel has no barrier
  const int nch = a.d_c / 8, width = a.d_c + a.d_rope;
  uint8_t* cache = (uint8_t*)a.cache;
  auto row_of = [&](int slot) {
    const int pg = (int)((uint64_t)(uint32_t)slot * args.page_magic >> args.page_shift);
    return cache + pg * a.page_stride + (int64_t)(slot - pg * a.page) * width;
  };

  float v[TPW][CH][8];
  int slot[TPW];
#pragma unroll
  for (int i = 0; i < TPW; ++i) {
    slot[i] = __builtin_amdgcn_readfirstlane(t0 + i < a.T ? a.slot[t0 + i] : -1);
    if ((unsigned)slot[i] >= (unsigned)a.n_slots) slot[i] = -1;
    const T* x = (const T*)a.latent + (t0 + i < a.T ? t0 + i : t0) * a.latent_stride;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int ch = l + 64 * k;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][k][e] = 0.f;
      if (ch < nch) load8(x + 8 * ch, v[i][k]);
    }
  }
  float g[CH][8];
#pragma unroll
  for (int k = 0; k < CH; ++k) {
#pragma unroll
    for (int e = 0; e < 8; ++e) g[k][e] = 1.f;
    if (a.gamma && l + 64 * k < nch) load8((const T*)a.gamma + 8 * (l + 64 * k), g[k]);
  }
  double sum[TPW], y[TPW][CH][8];
  int most[TPW];
#pragma unroll
  for (int i = 0; i < TPW; ++i) {
    sum[i] = 0.;
#pragma unroll
    for (int k = 0; k < CH; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[i] = __builtin_fma((double)v[i][k][e], (double)v[i][k][e], sum[i]);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1)
#pragma unroll
    for (int i = 0; i < TPW; ++i) sum[i] += __shfl_xor(sum[i], o);
  bool any = false;
#pragma unroll
  for (int i = 0; i < TPW; ++i) {
    const double r = rsqrt(__builtin_fma(sum[i], args.mean, (double)a.eps));
    double top = 0.;
#pragma unroll
    for (int k = 0; k < CH; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        y[i][k][e] = (double)v[i][k][e] * r * (double)g[k][e];
        top = __builtin_fmax(top, __builtin_fabs(y[i][k][e]));
      }
    most[i] = exponent_of(top);
    if (__ballot(top == __builtin_inf())) {
      any = true;
      most[i] = kLeastScale;
#pragma unroll
      for (int k = 0; k < CH; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) most[i] = max(most[i], exponent_of(y[i][k][e]));
    }
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1)
#pragma unroll
    for (int i = 0; i < TPW; ++i) most[i] = max(most[i], __shfl_xor(most[i], o));
#pragma unroll
  for (int i = 0; i < TPW; ++i) any = any || most[i] >= kMostScale;
  auto write = [&](auto is_any) {
#pragma unroll
    for (int i = 0; i < TPW; ++i) {
      if (slot[i] < 0) continue;  // wave-uniform
      const int e = within(most[i]);
      const double down = __builtin_ldexp(1., -e);
#pragma unroll
      for (int k = 0; k < CH; ++k)
        if (l + 64 * k < nch)
          *reinterpret_cast<i32x2*>(row_of(slot[i]) + 8 * (l + 64 * k)) =
              i32x2{four<decltype(is_any)::value>(y[i][k], down), four<decltype(is_any)::value>(y[i][k] + 4, down)};
      if (l == 0) args.scales[2 * (int64_t)slot[i]] = (uint8_t)(e + kScaleBias);
    }
  };
  if (any) write(std::true_type{});  // (the same on all lanes)
  else write(std::false_type{});

  const int pairs = a.d_rope / 2, p = l & pairs - 1, log2_pairs = __ffs(pairs) - 1;  // a power of two, 32 at most
  const double freq = args.freq[p];
  for (int i = l >> log2_pairs; i < TPW; i += 64 >> log2_pairs) {
    const int64_t t = t0 + i;
    if (t >= a.T) break;
    const int s = a.slot[t];
    if ((unsigned)s >= (unsigned)a.n_slots) continue;
    double turns = (double)(a.position_offset + a.position[t]) * freq, cs, sn;
    turns -= rint(turns);
    sincospi(2. * turns, &sn, &cs);
    const T* x = (const T*)a.kpe + t * a.kpe_stride + 2 * p;
    const double x0 = to_f32(x[0]), x1 = to_f32(x[1]);
    const double y[2] = {x0 * cs - x1 * sn, x0 * sn + x1 * cs};
    int most = max(exponent_of(y[0]), exponent_of(y[1]));
    for (int o = 1; o < pairs; o <<= 1) most = max(most, __shfl_xor(most, o));  // (the lanes of a token are all here)
    const int e = within(most);
    const double down = __builtin_ldexp(1., -e);
    *reinterpret_cast<uint16_t*>(row_of(s) + a.d_c + 2 * p) =
        (uint16_t)__builtin_amdgcn_cvt_pk_fp8_f32(eighth<true>(y[0], down), eighth<true>(y[1], down), 0, false);
    if (p == 0) args.scales[2 * (int64_t)s + 1] = (uint8_t)(e + kScaleBias);
  }
}

// Rows back as numbers: a workgroup looks up the places of `rows` of them, then each thread takes 16 numbers of a row at a
// time, several on their way at once.
constexpr int kReadThreads = 256, kReadRows = 32;
template <typename T>
__global__ __launch_bounds__(kReadThreads) void read_q8_kernel(ReadQ8Args a, int rows) {
  __shared__ const uint8_t* s_src[kReadRows];
  __shared__ float s_power[kReadRows][2];
  const int64_t t0 = (int64_t)blockIdx.x * rows;
  const int have = (int)min((int64_t)rows, a.T - t0), W = a.d_c + a.d_rope;
  if ((int)threadIdx.x < have) {
    const int64_t t = t0 + threadIdx.x;
    const int pos = a.position[t];
    const uint8_t* src = nullptr;
    int exps = kScaleBias | kScaleBias << 8;
    if (pos >= 0) {
      exps = 255 | 255 << 8;
      const int64_t r = a.row_request ? a.row_request[t] : t;
      if ((uint64_t)r < (uint64_t)a.R && pos < a.width * a.page) {
        const int pg = (int)((uint64_t)(uint32_t)pos * a.page_magic >> a.page_shift), off = pos - pg * a.page;
        const int id = a.table[r * a.width + pg];
        if ((unsigned)id < (unsigned)a.n_pages) {
          src = a.cache + id * a.page_stride + (int64_t)off * W;
          exps = *reinterpret_cast<const uint16_t*>(a.scales + 2 * ((int64_t)id * a.page + off));
        }
      }
    }
    s_src[threadIdx.x] = src;
    // (byte 0: 2^-127; 255: NaN)
    for (int k = 0; k < 2; ++k) {
      const int b = exps >> 8 * k & 255;
      s_power[threadIdx.x][k] = __builtin_bit_cast(float, b << 23 | ((b + 1 & 254) == 0 ? 1 << 22 : 0));
    }
  }
  __syncthreads();
  const int nch = W / 16;
#pragma unroll 4
  for (int x = threadIdx.x; x < have * nch; x += kReadThreads) {
    const int i = x / nch, c = 16 * (x - i * nch);
    const uint8_t* src = s_src[i];
    i32x4 b = {};  // a row that is not there: 0, times 1 or NaN
    if (src) b = *reinterpret_cast<const i32x4*>(src + c);
    const float power = s_power[i][c >= a.d_c];
    T* to = c < a.d_c ? (T*)a.c_kv + (t0 + i) * a.d_c + c : (T*)a.k_pe + (t0 + i) * a.d_rope + (c - a.d_c);
#pragma unroll
    for (int k = 0; k < 4; k += 2) {
      typedef float f32x2 __attribute__((ext_vector_type(2)));
      float y[8];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(b[k + u], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(b[k + u], true);
        y[4 * u] = lo[0] * power;
        y[4 * u + 1] = lo[1] * power;
        y[4 * u + 2] = hi[0] * power;
        y[4 * u + 3] = hi[1] * power;
      }
      store8(to + 4 * k, y);
    }
  }
}

template <typename T, int TPW>
void launch_append_q8_t(const AppendQ8Args& a, hipStream_t st) {
  const int per = kWaves * TPW;
  const unsigned wgs = (unsigned)(((int64_t)a.a.T + per - 1) / per);
  if (a.a.d_c <= 512) append_q8_kernel<T, TPW, 1><<<wgs, 64 * kWaves, 0, st>>>(a);
  else append_q8_kernel<T, TPW, 2><<<wgs, 64 * kWaves, 0, st>>>(a);
}

}  // namespace

// Two tokens a wave share the band's frequencies and the lanes of its turn, once the waves fill the GPU: 16384 tokens 16.8 us,
// 18.5 with one, 17.5 with four; 64 tokens 4.8 with one.
template <typename T>
hipError_t launch_append_q8(const AppendQ8Args& a, hipStream_t st) {
  if (a.a.T <= 16 * kCus) launch_append_q8_t<T, 1>(a, st);
  else launch_append_q8_t<T, 2>(a, st);
  return hipGetLastError();
}

// Rows per workgroup: as many as keep their places in LDS where that still gives every CU four; else few, for more copies at once.
// 78246 rows of d_c = 512 and d_rope = 64 in bf16 (136 MB) 35 us, 3.9 TB/s; stores that pass the caches by took 46. 130 rows 3.3 us.
template <typename T>
hipError_t launch_read_q8(const ReadQ8Args& a, hipStream_t st) {
  const int rows = a.T >= 4 * kCus * kReadRows ? kReadRows : 4;
  read_q8_kernel<T><<<(unsigned)(((int64_t)a.T + rows - 1) / rows), kReadThreads, 0, st>>>(a, rows);
  return hipGetLastError();
}

template hipError_t launch_append_q8<bf16>(const AppendQ8Args&, hipStream_t);
template hipError_t launch_append_q8<float>(const AppendQ8Args&, hipStream_t);
template hipError_t launch_read_q8<bf16>(const ReadQ8Args&, hipStream_t);
template hipError_t launch_read_q8<float>(const ReadQ8Args&, hipStream_t);

}  // namespace laga
