// The product of every group of rows with its cluster's matrix, and the gradients of both factors, in 16 and 32 bits.
#include "experts.h"
#include "grouped_tiles.h"

namespace sceig {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// What the matrix instructions take: a chunk is 16 bytes of a row along the contraction.
template <typename T>
struct Matrix;
template <>
struct Matrix<__bf16> {
  static constexpr int kChunk = 8;
  typedef __bf16 Chunk __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x4 mma(Chunk a, Chunk b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Matrix<_Float16> {
  static constexpr int kChunk = 8;
  typedef _Float16 Chunk __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x4 mma(Chunk a, Chunk b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Matrix<float> {
  static constexpr int kChunk = 4;
  typedef float Chunk __attribute__((ext_vector_type(4)));
  // Four instructions of depth 4.  Which value of the contraction an instruction takes from a lane does not matter as long as
  // both factors take the same: the j-th takes the j-th of the lane's chunk.
  static __device__ __forceinline__ f32x4 mma(Chunk a, Chunk b, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
};

// ---- any strides, any alignment ------------------------------------------------------------------------------------------
// out(r, c) = sum over e of R(r, e) C(c, e), a 64 x 64 tile of out by four waves, 32 x 32 each.  The contraction goes through
// LDS in steps of four chunks; the next step's chunks are loaded while this one's products run.
constexpr int kTile = 64;

enum { kProduct = 0, kTransposed = 1, kGradient = 2 };

// Eight (four) consecutive values from p on, of which `left` exist.
template <typename T, bool WIDE>
__device__ __forceinline__ typename Matrix<T>::Chunk load_chunk(const T* p, int left) {
  typedef typename Matrix<T>::Chunk Chunk;
  constexpr int CH = Matrix<T>::kChunk;
  Chunk v;
#pragma unroll
  for (int u = 0; u < CH; ++u) v[u] = static_cast<T>(0.0f);
  if (left <= 0) return v;
  if constexpr (WIDE) return *reinterpret_cast<const Chunk*>(p);  // lengths are whole chunks there
#pragma unroll
  for (int u = 0; u < CH; ++u)
    if (u < left) v[u] = p[u];
  return v;
}

template <typename T, int FORM, bool WIDE>
__global__ __launch_bounds__(256) void grouped_any_kernel(const T* __restrict__ rmat, const T* __restrict__ cmat, T* __restrict__ out,
                                                          const int32_t* __restrict__ offsets, const int32_t* __restrict__ order,
                                                          int64_t ldr, int64_t ldc, int64_t ldg, int64_t ldo, int64_t ldog,
                                                          int64_t rows, int64_t xrows, int groups, int slots, int outr, int outc,
                                                          int depth, int row_tiles, int col_tiles) {
  typedef typename Matrix<T>::Chunk Chunk;
  constexpr int CH = Matrix<T>::kChunk;
  constexpr int BK = 4 * CH;
  constexpr int LD = BK + CH;  // a row of a tile in LDS: one chunk more, so that the rows do not all begin in one bank
  __shared__ T rs[kTile * LD], cs[kTile * LD];
  int group, r0, rn, c0;
  int64_t pbegin = 0, pcount = 0;
  if (FORM == kGradient) {
    group = blockIdx.x / (row_tiles * col_tiles);
    const int at = blockIdx.x - group * (row_tiles * col_tiles);
    r0 = at / col_tiles * kTile;
    c0 = at % col_tiles * kTile;
    rn = min(kTile, outr - r0);
    const GroupRange g = group_range(offsets, groups, rows, group);
    pbegin = g.begin;
    pcount = g.end - g.begin;
  } else {
    const RowTile t = find_tile<kTile>(offsets, groups, rows, col_tiles);
    if (t.group < 0) return;
    group = t.group;
    r0 = 0;
    pbegin = t.begin;
    rn = t.count;
    c0 = t.col * kTile;
  }
  const int cn = min(kTile, outc - c0);
  const bool empty = FORM != kGradient && group == groups;
  const int64_t length = empty ? 0 : (FORM == kGradient ? pcount : depth);
  const T* cbase = FORM == kGradient || empty ? cmat : cmat + (int64_t)group * ldg;

  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int wr = (wave >> 1) * 32, wc = (wave & 1) * 32;
  f32x4 acc[2][2];
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < 2; ++b) acc[a][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  // A thread's chunk: of row `tid / 4` where rows run along the contraction, else of step tid / (64 / CH) of the contraction.
  constexpr int PER = kTile / CH;
  const int along_row = tid >> 2, along_e = (tid & 3) * CH;
  const int across_e = tid / PER, across_col = tid % PER * CH;
  int64_t rrow = -1;
  if (FORM != kGradient && along_row < rn) rrow = source_row(order, pbegin + along_row, slots, xrows);

  auto load = [&](int64_t e0, Chunk& r, Chunk& c) {
    if (FORM != kGradient) {
      const int64_t e = e0 + along_e;
      r = load_chunk<T, WIDE>(rmat + (rrow < 0 ? 0 : rrow * ldr + e), rrow < 0 ? 0 : (int)min((int64_t)CH, length - e));
    } else {
      const int64_t e = e0 + across_e;
      const int left = e < length ? min(CH, outr - (r0 + across_col)) : 0;
      r = load_chunk<T, WIDE>(rmat + (left > 0 ? (pbegin + e) * ldr + r0 + across_col : 0), left);
    }
    if (FORM == kProduct) {
      const int64_t e = e0 + along_e;
      const int left = along_row < cn ? (int)min((int64_t)CH, length - e) : 0;
      c = load_chunk<T, WIDE>(cbase + (left > 0 ? (int64_t)(c0 + along_row) * ldc + e : 0), left);
    } else {
      const int64_t e = e0 + across_e;
      int left = e < length ? min(CH, outc - (c0 + across_col)) : 0;
      int64_t at = 0;
      if (left > 0) {
        at = FORM == kGradient ? source_row(order, pbegin + e, slots, xrows) : e;
        if (at < 0) left = 0;
      }
      c = load_chunk<T, WIDE>(cbase + (left > 0 ? at * ldc + c0 + across_col : 0), left);
    }
  };
  auto store = [&](T* tile, const Chunk& v, bool along) {
    if (along) {
      *reinterpret_cast<Chunk*>(tile + along_row * LD + along_e) = v;
    } else {
#pragma unroll
      for (int u = 0; u < CH; ++u) tile[(across_col + u) * LD + across_e] = v[u];
    }
  };

  Chunk r, c;
  if (length > 0) load(0, r, c);
  for (int64_t e0 = 0; e0 < length; e0 += BK) {
    store(rs, r, FORM != kGradient);
    store(cs, c, FORM == kProduct);
    __syncthreads();
    if (e0 + BK < length) load(e0 + BK, r, c);
    Chunk fr[2], fc[2];
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      fr[a] = *reinterpret_cast<const Chunk*>(rs + (wr + a * 16 + (lane & 15)) * LD + (lane >> 4) * CH);
      fc[a] = *reinterpret_cast<const Chunk*>(cs + (wc + a * 16 + (lane & 15)) * LD + (lane >> 4) * CH);
    }
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int b = 0; b < 2; ++b) acc[a][b] = Matrix<T>::mma(fc[b], fr[a], acc[a][b]);  // a lane gets four neighbours of a row
    __syncthreads();
  }

  T* obase = FORM == kGradient ? out + (int64_t)group * ldog : out;
#pragma unroll
  for (int a = 0; a < 2; ++a) {
    const int row = wr + a * 16 + (lane & 15);
    if (row >= rn) continue;
    T* orow = obase + ((FORM == kGradient ? (int64_t)r0 : pbegin) + row) * ldo + c0;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int col = wc + b * 16 + (lane >> 4) * 4;
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (col + u < cn) orow[col + u] = static_cast<T>(acc[a][b][u]);
    }
  }
}

template <typename T>
bool whole_chunks(const void* p, int64_t ld) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % Matrix<T>::kChunk == 0;
}

template <typename T>
hipError_t product_typed(const GroupedArgs& a, bool transpose, hipStream_t st) {
  constexpr int CH = Matrix<T>::kChunk;
  const int outc = transpose ? a.K : a.N, depth = transpose ? a.N : a.K;
  const T *x = static_cast<const T*>(a.x), *w = static_cast<const T*>(a.w);
  T* y = static_cast<T*>(a.y);
  const int cols = (outc + kTile - 1) / kTile;
  const int64_t blocks = tile_bound(a.rows, a.groups, kTile, cols);
  if (blocks > 0x7fffffff) return hipErrorInvalidConfiguration;
  const bool wide = whole_chunks<T>(a.x, a.ldx) && whole_chunks<T>(a.w, a.ldw) && a.ldg % CH == 0 && a.K % CH == 0 && a.N % CH == 0;
#define SC_LAUNCH(FORM, WIDE)                                                                                                   \
  grouped_any_kernel<T, FORM, WIDE><<<(uint32_t)blocks, 256, 0, st>>>(x, w, y, a.offsets, a.order, a.ldx, a.ldw, a.ldg, a.ldy, 0, \
                                                                      a.rows, a.xrows, a.groups, a.slots, 0, outc, depth, 0, cols)
  if (transpose && wide) SC_LAUNCH(kTransposed, true);
  else if (transpose) SC_LAUNCH(kTransposed, false);
  else if (wide) SC_LAUNCH(kProduct, true);
  else SC_LAUNCH(kProduct, false);
#undef SC_LAUNCH
  return hipGetLastError();
}

template <typename T>
hipError_t gradient_typed(const GradientArgs& a, hipStream_t st) {
  constexpr int CH = Matrix<T>::kChunk;
  const T *dy = static_cast<const T*>(a.dy), *x = static_cast<const T*>(a.x);
  T* dw = static_cast<T*>(a.dw);
  const int rt = (a.N + kTile - 1) / kTile, ct = (a.K + kTile - 1) / kTile;
  const int64_t blocks = (int64_t)a.groups * rt * ct;
  if (blocks > 0x7fffffff) return hipErrorInvalidConfiguration;
  const bool wide = whole_chunks<T>(a.x, a.ldx) && whole_chunks<T>(a.dy, a.lddy) && a.K % CH == 0 && a.N % CH == 0;
#define SC_LAUNCH(WIDE)                                                                                                        \
  grouped_any_kernel<T, kGradient, WIDE><<<(uint32_t)blocks, 256, 0, st>>>(dy, x, dw, a.offsets, a.order, a.lddy, a.ldx, 0, a.ldw, \
                                                                           a.ldg, a.rows, a.xrows, a.groups, a.slots, a.N, a.K, 0, \
                                                                           rt, ct)
  if (wide) SC_LAUNCH(true);
  else SC_LAUNCH(false);
#undef SC_LAUNCH
  return hipGetLastError();
}

}  // namespace

hipError_t launch_grouped_product(const GroupedArgs& a, bool transpose, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  if (a.dtype == kF32) return product_typed<float>(a, transpose, st);
  if (a.dtype == kBF16) return product_typed<__bf16>(a, transpose, st);
  return product_typed<_Float16>(a, transpose, st);
}

hipError_t launch_grouped_gradient(const GradientArgs& a, hipStream_t st) {
  if (a.dtype == kF32) return gradient_typed<float>(a, st);
  if (a.dtype == kBF16) return gradient_typed<__bf16>(a, st);
  return gradient_typed<_Float16>(a, st);
}

}  // namespace sceig
