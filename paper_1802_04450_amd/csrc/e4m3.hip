// 8-bit matrices: a row is cut into blocks of 128 along the contraction, a block holds numbers with 4 bits of exponent and 3 of
// fraction and one power of two.  Conversion there and back, and the product by groups.
//
// Why powers of two: the numbers are floating-point themselves, so a scale that is not one gains nothing but a fraction of a bit
// of range at the lower end, while the matrix instructions of gfx950 multiply by a power of two per 32 values on their own - the
// sums need no scaling afterwards.
#include "experts.h"
#include "grouped_tiles.h"

namespace sceig {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

// ---- conversion -------------------------------------------------------------------------------------------------------
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 ... 127
// v 2^e for -254 <= e <= 254 in two exact steps (an end result below the normal range is rounded once).
__device__ __forceinline__ float scaled(float v, int e) {
  const int h = e >> 1;
  return v * power_of_two(h) * power_of_two(e - h);
}

// 16 lanes a block, 8 values a lane.  The exponent is the smallest E >= -127 with max |v| <= 448 * 2^E over the finite values
// (E = 0 for a block of zeros): 448 = 1.75 * 2^8, so it comes from the bits of the largest value and nothing saturates.  Each
// value is rounded once, to the nearest with ties to even; what is not finite becomes the type's NaN.
template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void quantize_kernel(const T* __restrict__ x, int64_t ldx, int64_t rows, int K, int blocks_row,
                                                       uint8_t* __restrict__ q, int64_t ldq, uint8_t* __restrict__ scale,
                                                       int64_t lds) {
  const int64_t block = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  const int lane = threadIdx.x & 15;
  const int64_t row = block / blocks_row;
  if (row >= rows) return;
  const int b = (int)(block - row * blocks_row);
  const int j = b * kScaleBlock + lane * 8;
  float v[8];
  const T* p = x + row * ldx + j;
  if (WIDE) {
    constexpr int E = 16 / (int)sizeof(T);
    typedef T Part __attribute__((ext_vector_type(E)));
#pragma unroll
    for (int u = 0; u < 8; u += E) {
      if (j + u < K) {
        const Part part = *reinterpret_cast<const Part*>(p + u);
#pragma unroll
        for (int e = 0; e < E; ++e) v[u + e] = static_cast<float>(part[e]);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[u + e] = 0.0f;
      }
    }
  } else {
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = j + u < K ? static_cast<float>(p[u]) : 0.0f;
  }
  float most = 0.0f;
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    const float a = fabsf(v[u]);
    most = a < INFINITY ? fmaxf(most, a) : most;
  }
#pragma unroll
  for (int s = 1; s < 16; s <<= 1) most = fmaxf(most, __shfl_xor(most, s));
  int e = 0;
  if (most > 0.0f) {
    int shift = 0;
    float m = most;
    if (m < 1.1754944e-38f) {  // below the normal range: its bits after a shift into it
      m *= 16777216.0f;
      shift = 24;
    }
    const uint32_t bits = __float_as_uint(m);
    e = (int)(bits >> 23) - 127 - shift - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = e < -127 ? -127 : e;
  }
  uint32_t word[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float s[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) s[u] = scaled(v[h * 4 + u], -e);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(s[0], s[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(s[2], s[3], w, true);
    word[h] = (uint32_t)w;
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (!(fabsf(v[h * 4 + u]) < INFINITY)) word[h] |= 0x7fu << (8 * u);
  }
  if (reinterpret_cast<uintptr_t>(q) % 8 == 0 && ldq % 8 == 0) {
    *reinterpret_cast<uint2*>(q + row * ldq + j) = make_uint2(word[0], word[1]);
  } else {
#pragma unroll
    for (int u = 0; u < 8; ++u) q[row * ldq + j + u] = (uint8_t)(word[u >> 2] >> (8 * (u & 3)));
  }
  if (lane == 0) scale[row * lds + b] = (uint8_t)(e + 127);
}

// 8 values a thread.
template <typename T>
__global__ __launch_bounds__(256) void dequantize_kernel(const uint8_t* __restrict__ q, int64_t ldq, const uint8_t* __restrict__ scale,
                                                         int64_t lds, int64_t rows, int K, int parts, T* __restrict__ x, int64_t ldx) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = at / parts;
  if (row >= rows) return;
  const int j = (int)(at - row * parts) * 8;
  const int code = scale[row * lds + j / kScaleBlock];
  uint32_t word[2];
  if (reinterpret_cast<uintptr_t>(q) % 8 == 0 && ldq % 8 == 0) {
    const uint2 w = *reinterpret_cast<const uint2*>(q + row * ldq + j);
    word[0] = w.x;
    word[1] = w.y;
  } else {
    word[0] = word[1] = 0;
    for (int u = 0; u < 8; ++u) word[u >> 2] |= (uint32_t)q[row * ldq + j + u] << (8 * (u & 3));
  }
  float v[8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    v[h * 4 + 0] = __builtin_amdgcn_cvt_f32_fp8(word[h], 0);
    v[h * 4 + 1] = __builtin_amdgcn_cvt_f32_fp8(word[h], 1);
    v[h * 4 + 2] = __builtin_amdgcn_cvt_f32_fp8(word[h], 2);
    v[h * 4 + 3] = __builtin_amdgcn_cvt_f32_fp8(word[h], 3);
  }
#pragma unroll
  for (int u = 0; u < 8; ++u) v[u] = code == 255 ? NAN : scaled(v[u], code - 127);
  T* out = x + row * ldx + j;
  constexpr int E = 16 / (int)sizeof(T);
  if (j + 8 <= K && reinterpret_cast<uintptr_t>(x) % 16 == 0 && ldx % E == 0) {
    typedef T Part __attribute__((ext_vector_type(E)));
#pragma unroll
    for (int u = 0; u < 8; u += E) {
      Part p;
#pragma unroll
      for (int e = 0; e < E; ++e) p[e] = static_cast<T>(v[u + e]);
      *reinterpret_cast<Part*>(out + u) = p;
    }
  } else {
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (j + u < K) out[u] = static_cast<T>(v[u]);
  }
}

// ---- product ------------------------------------------------------------------------------------------------------------
// A 64 x 64 tile of y by four waves, 32 x 32 each, one block of the contraction (128 bytes a row) at a time through LDS.  A lane
// of the matrix instruction takes 32 consecutive values of one row and the exponent byte of their block.
//
// The 8-bit matrix instructions add eight neighbouring products with a common exponent before they go to 32 bits: what lies 2^-14
// below the largest of the eight is cut off (measured: 256 + 2^-5 is kept, 256 + 2^-6 is not, and is where the two products are
// eight apart).  On random data that is 5.5e-5 of the result's size, which 16-bit results (2e-4, 1.7e-3 from their own rounding)
// do not show.  32-bit results would, so they take the factors as bf16, which holds every 8-bit number, with sums in 32 bits
// throughout and each block's powers of two multiplied in afterwards.
constexpr int kTile = 64;
constexpr int kPitch = kScaleBlock + 16;

template <typename T>
__global__ __launch_bounds__(256) void e4m3_any_kernel(E4m3Args a, int cols) {
  __shared__ __attribute__((aligned(16))) uint8_t xt[kTile * kPitch], wt[kTile * kPitch];
  const RowTile t = find_tile<kTile>(a.offsets, a.groups, a.rows, cols);
  if (t.group < 0) return;
  const bool empty = t.group == a.groups;
  const int c0 = t.col * kTile, cn = min(kTile, a.N - c0);
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int wr = (wave >> 1) * 32, wc = (wave & 1) * 32;
  // a thread loads two chunks of 16 bytes of each factor: rows tid / 8 and tid / 8 + 32
  int64_t xrow[2];
  const uint8_t *xp[2], *wp[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = (tid >> 3) + h * 32;
    xrow[h] = !empty && r < t.count ? source_row(a.order, t.begin + r, a.slots, a.xrows) : -1;
    xp[h] = xrow[h] < 0 ? nullptr : a.x + xrow[h] * a.ldx + (tid & 7) * 16;
    wp[h] = !empty && r < cn ? a.w + (int64_t)t.group * a.ldg + (int64_t)(c0 + r) * a.ldw + (tid & 7) * 16 : nullptr;
  }
  // the scales of the rows whose values the lane hands to the matrix instructions
  const uint8_t *xsp[2], *wsp[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = wr + h * 16 + (lane & 15), c = wc + h * 16 + (lane & 15);
    const int64_t src = !empty && r < t.count ? source_row(a.order, t.begin + r, a.slots, a.xrows) : -1;
    xsp[h] = src < 0 ? nullptr : a.xs + src * a.ldxs;
    wsp[h] = !empty && c < cn ? a.ws + (int64_t)t.group * a.ldgs + (int64_t)(c0 + c) * a.ldws : nullptr;
  }
  f32x4 acc[2][2];
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int v = 0; v < 2; ++v) acc[u][v] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const i32x4 zero = {0, 0, 0, 0};
  const int steps = empty ? 0 : a.Kp / kScaleBlock;
  for (int b = 0; b < steps; ++b) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = ((tid >> 3) + h * 32) * kPitch + (tid & 7) * 16;
      *reinterpret_cast<i32x4*>(xt + at) = xp[h] ? *reinterpret_cast<const i32x4*>(xp[h] + b * kScaleBlock) : zero;
      *reinterpret_cast<i32x4*>(wt + at) = wp[h] ? *reinterpret_cast<const i32x4*>(wp[h] + b * kScaleBlock) : zero;
    }
    __syncthreads();
    i32x8 fx[2], fw[2];
    int sx[2], sw[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const i32x4* px = reinterpret_cast<const i32x4*>(xt + (wr + h * 16 + (lane & 15)) * kPitch + (lane >> 4) * 32);
      const i32x4* pw = reinterpret_cast<const i32x4*>(wt + (wc + h * 16 + (lane & 15)) * kPitch + (lane >> 4) * 32);
      fx[h] = __builtin_shufflevector(px[0], px[1], 0, 1, 2, 3, 4, 5, 6, 7);
      fw[h] = __builtin_shufflevector(pw[0], pw[1], 0, 1, 2, 3, 4, 5, 6, 7);
      sx[h] = xsp[h] ? xsp[h][b] : 127;
      sw[h] = wsp[h] ? wsp[h][b] : 127;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int v = 0; v < 2; ++v)
        acc[u][v] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw[v], fx[u], acc[u][v], 0, 0, 0, sw[v], 0, sx[u]);
    __syncthreads();
  }
  T* y = static_cast<T*>(a.y);
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int row = wr + u * 16 + (lane & 15);
    if (row >= t.count) continue;
    T* out = y + (t.begin + row) * a.ldy + c0;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const int col = wc + v * 16 + (lane >> 4) * 4;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (col + i < cn) out[col + i] = static_cast<T>(acc[u][v][i]);
    }
  }
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
// 8 numbers as bf16
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The same tile with the factors as bf16 in LDS.
constexpr int kWidePitch = kScaleBlock + 8;

__global__ __launch_bounds__(256) void e4m3_wide_kernel(E4m3Args a, int cols) {
  __shared__ __attribute__((aligned(16))) __bf16 xt[kTile * kWidePitch], wt[kTile * kWidePitch];
  const RowTile t = find_tile<kTile>(a.offsets, a.groups, a.rows, cols);
  if (t.group < 0) return;
  const bool empty = t.group == a.groups;
  const int c0 = t.col * kTile, cn = min(kTile, a.N - c0);
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int wr = (wave >> 1) * 32, wc = (wave & 1) * 32;
  const uint8_t *xp[2], *wp[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = (tid >> 3) + h * 32;
    const int64_t src = !empty && r < t.count ? source_row(a.order, t.begin + r, a.slots, a.xrows) : -1;
    xp[h] = src < 0 ? nullptr : a.x + src * a.ldx + (tid & 7) * 16;
    wp[h] = !empty && r < cn ? a.w + (int64_t)t.group * a.ldg + (int64_t)(c0 + r) * a.ldw + (tid & 7) * 16 : nullptr;
  }
  // the scales of the results that the lane gets: two rows, twice four columns
  const uint8_t *xsp[2], *wsp[2][4];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = wr + h * 16 + (lane & 15), c = wc + h * 16 + (lane >> 4) * 4;
    const int64_t src = !empty && r < t.count ? source_row(a.order, t.begin + r, a.slots, a.xrows) : -1;
    xsp[h] = src < 0 ? nullptr : a.xs + src * a.ldxs;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      wsp[h][i] = !empty && c + i < cn ? a.ws + (int64_t)t.group * a.ldgs + (int64_t)(c0 + c + i) * a.ldws : nullptr;
  }
  f32x4 acc[2][2];
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int v = 0; v < 2; ++v) acc[u][v] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const int steps = empty ? 0 : a.Kp / kScaleBlock;
  for (int b = 0; b < steps; ++b) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = ((tid >> 3) + h * 32) * kWidePitch + (tid & 7) * 16;
      const uint4 x = xp[h] ? *reinterpret_cast<const uint4*>(xp[h] + b * kScaleBlock) : make_uint4(0, 0, 0, 0);
      const uint4 w = wp[h] ? *reinterpret_cast<const uint4*>(wp[h] + b * kScaleBlock) : make_uint4(0, 0, 0, 0);
      *reinterpret_cast<bf16x8*>(xt + at) = widen(x.x, x.y);
      *reinterpret_cast<bf16x8*>(xt + at + 8) = widen(x.z, x.w);
      *reinterpret_cast<bf16x8*>(wt + at) = widen(w.x, w.y);
      *reinterpret_cast<bf16x8*>(wt + at + 8) = widen(w.z, w.w);
    }
    __syncthreads();
    f32x4 part[2][2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int v = 0; v < 2; ++v) part[u][v] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int e = 0; e < kScaleBlock; e += 32) {
      bf16x8 fx[2], fw[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        fx[h] = *reinterpret_cast<const bf16x8*>(xt + (wr + h * 16 + (lane & 15)) * kWidePitch + e + (lane >> 4) * 8);
        fw[h] = *reinterpret_cast<const bf16x8*>(wt + (wc + h * 16 + (lane & 15)) * kWidePitch + e + (lane >> 4) * 8);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int v = 0; v < 2; ++v) part[u][v] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[v], fx[u], part[u][v], 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int sx = xsp[u] ? xsp[u][b] : 127;
#pragma unroll
      for (int v = 0; v < 2; ++v)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int sw = wsp[v][i] ? wsp[v][i][b] : 127;
          acc[u][v][i] += sx == 255 || sw == 255 ? NAN : ldexpf(part[u][v][i], sx + sw - 254);
        }
    }
    __syncthreads();
  }
  float* y = static_cast<float*>(a.y);
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int row = wr + u * 16 + (lane & 15);
    if (row >= t.count) continue;
    float* out = y + (t.begin + row) * a.ldy + c0;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const int col = wc + v * 16 + (lane >> 4) * 4;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (col + i < cn) out[col + i] = acc[u][v][i];
    }
  }
}

template <typename T>
hipError_t quantize_typed(const T* x, int64_t ldx, int64_t rows, int K, uint8_t* q, int64_t ldq, uint8_t* scale, int64_t lds,
                          hipStream_t st) {
  constexpr int E = 16 / (int)sizeof(T);
  const int blocks_row = (K + kScaleBlock - 1) / kScaleBlock;
  const int64_t grid = (rows * blocks_row + 15) / 16;
  if (grid > 0x7fffffff) return hipErrorInvalidConfiguration;
  if (reinterpret_cast<uintptr_t>(x) % 16 == 0 && ldx % E == 0 && K % E == 0)
    quantize_kernel<T, true><<<(uint32_t)grid, 256, 0, st>>>(x, ldx, rows, K, blocks_row, q, ldq, scale, lds);
  else
    quantize_kernel<T, false><<<(uint32_t)grid, 256, 0, st>>>(x, ldx, rows, K, blocks_row, q, ldq, scale, lds);
  return hipGetLastError();
}

template <typename T>
hipError_t dequantize_typed(const uint8_t* q, int64_t ldq, const uint8_t* scale, int64_t lds, int64_t rows, int K, T* x, int64_t ldx,
                            hipStream_t st) {
  const int parts = (K + 7) / 8;
  const int64_t grid = (rows * parts + 255) / 256;
  if (grid > 0x7fffffff) return hipErrorInvalidConfiguration;
  dequantize_kernel<T><<<(uint32_t)grid, 256, 0, st>>>(q, ldq, scale, lds, rows, K, parts, x, ldx);
  return hipGetLastError();
}

template <typename T>
hipError_t product_typed(const E4m3Args& a, hipStream_t st) {
  const int cols = (a.N + kTile - 1) / kTile;
  const int64_t blocks = tile_bound(a.rows, a.groups, kTile, cols);
  if (blocks > 0x7fffffff) return hipErrorInvalidConfiguration;
  if constexpr (sizeof(T) == 4)
    e4m3_wide_kernel<<<(uint32_t)blocks, 256, 0, st>>>(a, cols);
  else
    e4m3_any_kernel<T><<<(uint32_t)blocks, 256, 0, st>>>(a, cols);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_blocks(const void* x, int dtype, int64_t ldx, int64_t rows, int K, uint8_t* q, int64_t ldq,
                                  uint8_t* scale, int64_t lds, hipStream_t st) {
  if (rows == 0) return hipSuccess;
  if (dtype == kF32) return quantize_typed(static_cast<const float*>(x), ldx, rows, K, q, ldq, scale, lds, st);
  if (dtype == kBF16) return quantize_typed(static_cast<const __bf16*>(x), ldx, rows, K, q, ldq, scale, lds, st);
  return quantize_typed(static_cast<const _Float16*>(x), ldx, rows, K, q, ldq, scale, lds, st);
}

hipError_t launch_dequantize_blocks(const uint8_t* q, int64_t ldq, const uint8_t* scale, int64_t lds, int64_t rows, int K,
                                    void* x, int dtype, int64_t ldx, hipStream_t st) {
  if (rows == 0) return hipSuccess;
  if (dtype == kF32) return dequantize_typed(q, ldq, scale, lds, rows, K, static_cast<float*>(x), ldx, st);
  if (dtype == kBF16) return dequantize_typed(q, ldq, scale, lds, rows, K, static_cast<__bf16*>(x), ldx, st);
  return dequantize_typed(q, ldq, scale, lds, rows, K, static_cast<_Float16*>(x), ldx, st);
}

hipError_t launch_grouped_product_e4m3(const E4m3Args& a, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  if (a.dtype == kF32) return product_typed<float>(a, st);
  if (a.dtype == kBF16) return product_typed<__bf16>(a, st);
  return product_typed<_Float16>(a, st);
}

}  // namespace sceig
