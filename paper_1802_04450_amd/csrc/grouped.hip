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

// ---- few rows a group ----------------------------------------------------------------------------------------------------------
// Every matrix that is met is read once, from memory straight into the registers of the wave that needs it, and that is what
// bounds it.  A wave has 16 columns and RF * 16 rows; KS of a workgroup's four waves share the columns, each with every KS-th
// run of RUN chunks of the contraction, and their sums are added in order at the end: as few columns as there are, enough
// waves are at work.  A run of the matrix is on its way while one is used.  Rows of any alignment: a lane's 16 bytes may begin anywhere.
constexpr int kThinRun = 4;

template <typename T>
__device__ __forceinline__ typename Matrix<T>::Chunk load_any(const T* p, int64_t left) {
  typedef typename Matrix<T>::Chunk Chunk;
  constexpr int CH = Matrix<T>::kChunk;
  Chunk v;
  if (left >= CH) {
    __builtin_memcpy(&v, p, sizeof(v));
  } else {
#pragma unroll
    for (int u = 0; u < CH; ++u) v[u] = u < left ? p[u] : static_cast<T>(0.0f);
  }
  return v;
}

template <typename T, int RF, int KS>
__global__ __launch_bounds__(256) void grouped_thin_kernel(GroupedArgs a, int col_tiles, int whole_stores) {
  typedef typename Matrix<T>::Chunk Chunk;
  constexpr int CH = Matrix<T>::kChunk, CT = 4 / KS, BK = 4 * CH;
  __shared__ f32x4 part[KS > 1 ? (KS - 1) * CT * RF * 64 : 1];
  const RowTile t = find_tile<RF * 16>(a.offsets, a.groups, a.rows, col_tiles);
  if (t.group < 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int ks = wave % KS, ct = wave / KS;
  const int c0 = (t.col * CT + ct) * 16;
  const int sub = lane & 15, quad = lane >> 4;
  const int64_t K = t.group == a.groups ? 0 : a.K;
  f32x4 acc[RF];
#pragma unroll
  for (int r = 0; r < RF; ++r) acc[r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  if (K > 0 && c0 < a.N) {
    const T* w = static_cast<const T*>(a.w) + (int64_t)t.group * a.ldg + (int64_t)min(c0 + sub, a.N - 1) * a.ldw + quad * CH;
    const T* x[RF];
#pragma unroll
    for (int r = 0; r < RF; ++r) {
      const int row = r * 16 + sub;
      const int64_t src = row < t.count ? source_row(a.order, t.begin + row, a.slots, a.xrows) : -1;
      x[r] = src < 0 ? nullptr : static_cast<const T*>(a.x) + src * a.ldx + quad * CH;
    }
    const int64_t step = (int64_t)KS * kThinRun * BK;
    Chunk next[kThinRun];
    int64_t e0 = (int64_t)ks * kThinRun * BK;
#pragma unroll
    for (int u = 0; u < kThinRun; ++u) next[u] = load_any<T>(w + e0 + u * BK, K - (e0 + u * BK + quad * CH));
    for (; e0 < K; e0 += step) {
      Chunk now[kThinRun];
#pragma unroll
      for (int u = 0; u < kThinRun; ++u) now[u] = next[u];
      const int64_t e1 = e0 + step;
      if (e1 < K) {
#pragma unroll
        for (int u = 0; u < kThinRun; ++u) next[u] = load_any<T>(w + e1 + u * BK, K - (e1 + u * BK + quad * CH));
      }
#pragma unroll
      for (int r = 0; r < RF; ++r) {
        if (r * 16 < t.count) {
          Chunk f[kThinRun];
#pragma unroll
          for (int u = 0; u < kThinRun; ++u)
            f[u] = load_any<T>(x[r] + e0 + u * BK, x[r] ? K - (e0 + u * BK + quad * CH) : 0);
#pragma unroll
          for (int u = 0; u < kThinRun; ++u) acc[r] = Matrix<T>::mma(now[u], f[u], acc[r]);
        }
      }
    }
  }
  if (KS > 1) {
    if (ks > 0) {
#pragma unroll
      for (int r = 0; r < RF; ++r) part[(((ks - 1) * CT + ct) * RF + r) * 64 + lane] = acc[r];
    }
    __syncthreads();
    if (ks > 0) return;
#pragma unroll
    for (int q = 0; q < KS - 1; ++q)
#pragma unroll
      for (int r = 0; r < RF; ++r) acc[r] += part[((q * CT + ct) * RF + r) * 64 + lane];
  }
  typedef T Quad __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int r = 0; r < RF; ++r) {
    const int row = r * 16 + sub, col = c0 + quad * 4;
    if (row >= t.count || col >= a.N) continue;
    T* out = static_cast<T*>(a.y) + (t.begin + row) * a.ldy + col;
    Quad q;
#pragma unroll
    for (int u = 0; u < 4; ++u) q[u] = static_cast<T>(acc[r][u]);
    if (whole_stores) {
      *reinterpret_cast<Quad*>(out) = q;
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (col + u < a.N) out[u] = q[u];
    }
  }
}

// ---- whole 16-byte pieces, 16-bit types --------------------------------------------------------------------------------------
// A BM x BN tile by WR x WC waves.  The contraction goes through LDS in steps of 64, in five buffers that hold a step of one
// operand each: while two are read, three are filled, the columns' operand two steps ahead and the rows' one and a half.  Pieces go
// straight from memory into LDS.  An operand whose rows run along the contraction (`along`) lies in LDS row by row, 128 bytes
// each, an operand whose rows run across it (`across`) step by step; the latter is turned by the transposing LDS read.
// The 16-byte pieces of a row are permuted by the row's number, so that the rows (or steps)
// that a read touches at once lie in different banks; as the loads write LDS in lane order it is the source address that is
// permuted.
__device__ uint4 zero_piece[1];

typedef short short4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4v LdsShort4;

// 16 bytes a lane from src to dst + 16 * lane, dst the same for the wave.  Written as an instruction of its own because the compiler
// counts the builtin as an access that may return out of order and then waits for every LDS read at once; it returns nothing in a
// register, and meet() waits for it.
__device__ __forceinline__ void piece_to_lds(const void* src, void* dst) {
  const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(LdsVoid*)dst);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(at), "v"(src) : "memory");
}
constexpr int kStep = 64;

// How the pieces of a row change places: of a row of the rows' operand by the 16-byte piece, of the columns' operand too, but in
// the order in which its fragments take the rows; of step e of an `across` operand by 32 bytes.
__device__ __forceinline__ int row_shift(int r) { return r & 7; }
__device__ __forceinline__ int col_shift(int c) { return ((c >> 3) & 3) | ((c << 1) & 4); }
__device__ __forceinline__ int across_shift(int e) { return (e & 3) | ((e >> 1) & 4); }

// Column (from the wave's first) of value i of column fragment b.  A lane gets values 4 q ... 4 q + 3 of every fragment (q = lane /
// 16); so that those of two fragments are eight neighbours, one 16-byte store, the columns are dealt out in this order.
__device__ __forceinline__ int fragment_col(int b, int i) { return (b >> 1) * 32 + (i >> 2) * 8 + (b & 1) * 4 + (i & 3); }

template <typename T>
__device__ __forceinline__ typename Matrix<T>::Chunk along_piece(const T* tile, int r, int shift, int piece) {
  return *reinterpret_cast<const typename Matrix<T>::Chunk*>(tile + r * kStep + ((piece ^ shift) << 3));
}
// Values first + 0 ... 3 (this lane's part of the columns) of steps e and e + 4, turned.
template <typename T, int EXT>
__device__ __forceinline__ typename Matrix<T>::Chunk across_piece(const T* tile, int col, int e) {
  union {
    short4v part[2];
    typename Matrix<T>::Chunk whole;
  } u;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const T* p = tile + (e + 4 * h) * EXT + (((col >> 4) ^ across_shift(e + 4 * h)) << 4) + (col & 15);
    u.part[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4*)p);
  }
  return u.whole;
}

// Workgroups take one tile after the other: while the last two steps of a tile run, the first two of the next are fetched, and a
// tile's results are stored while the next one's products run.  For that every tile has at least two steps, a gradient's three, as
// the rows of x that a step takes are looked up a step before they are fetched; steps behind the contraction's end hold zeros.
template <typename T, int FORM, int BM, int BN, int WR, int WC>
__global__ __launch_bounds__(WR * WC * 64) void grouped_tile_kernel(
    const T* __restrict__ rmat, const T* __restrict__ cmat, T* __restrict__ out, const int32_t* __restrict__ offsets,
    const int32_t* __restrict__ order, int64_t ldr, int64_t ldc, int64_t ldg, int64_t ldo, int64_t ldog, int64_t rows,
    int64_t xrows, int groups, int slots, int outr, int outc, int depth, int row_tiles, int col_tiles) {
  typedef typename Matrix<T>::Chunk Chunk;
  typedef T Part __attribute__((ext_vector_type(8)));
  constexpr int NW = WR * WC;
  constexpr int FR = BM / WR / 16, FC = BN / WC / 16;
  constexpr bool R_ALONG = FORM != kGradient, C_ALONG = FORM == kProduct;
  constexpr int LR = BM / 8 / NW, LC = BN / 8 / NW;  // loads of 1 KB a wave and step
  static_assert(LR * 8 * NW == BM && LC * 8 * NW == BN && FR % 4 == 0 && FC % 2 == 0, "");
  constexpr int BUFFERS = 5, BUFFER = (BM > BN ? BM : BN) * kStep;
  __shared__ __attribute__((aligned(1024))) T lds[BUFFERS * BUFFER];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = wave / WC * (BM / WR), wc = wave % WC * (BN / WC);
  const T* const zero = reinterpret_cast<const T*>(zero_piece);

  // ---- the tiles ----
  struct Tile {
    int group, r0, rn, c0, cn;
    int64_t pbegin;
    int length;
  };
  const TileWalk<BM> walk(offsets, FORM == kGradient ? 0 : groups, rows, FORM == kGradient ? 1 : col_tiles);
  const GroupOrder by_length(offsets, FORM == kGradient ? groups : 0, rows);
  const int per_group = row_tiles * col_tiles;  // gradient
  // A gradient's tiles take as long as their groups are.  From the longest group to the shortest they are dealt out to all
  // workgroups, to and fro.
  const int64_t count =
      FORM == kGradient ? ((int64_t)groups * per_group + gridDim.x - 1) / gridDim.x : walk.count;
  auto tile_at = [&](int64_t i, Tile& t) {  // false: there is none (only the last one of a gradient)
    if (FORM == kGradient) {
      const int64_t at = i * gridDim.x + (i & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
      if (at >= (int64_t)groups * per_group) return false;
      const int g = (int)(at / per_group), in = (int)(at - (int64_t)g * per_group);
      t.group = by_length.at(g);
      t.r0 = in / col_tiles * BM;
      t.c0 = in % col_tiles * BN;
      t.rn = min(BM, outr - t.r0);
      const GroupRange r = group_range(offsets, groups, rows, t.group);
      t.pbegin = r.begin;
      t.length = (int)(r.end - r.begin);
    } else {
      const RowTile r = walk.at(i);
      t.group = r.group;
      t.r0 = 0;
      t.rn = r.count;
      t.pbegin = r.begin;
      t.c0 = r.col * BN;
      t.length = depth;
    }
    t.cn = min(BN, outc - t.c0);
    return true;
  };

  // ---- what a lane loads ----
  // `along` a fixed row, `across` a fixed column of its operand, and one step after the other of it.  Rows and columns outside the
  // tile take the last one's values, which nothing stores; steps beyond the contraction's end come from a piece of zeros.
  const T *rp[LR], *cp[LC];
  const int along_r = lane >> 3;  // row within the eight that a load brings
  int re[LR], ce[LC];
#pragma unroll
  for (int u = 0; u < LR; ++u) re[u] = R_ALONG ? ((lane & 7) ^ row_shift(along_r)) * 8
                                               : (wave * LR + u) * (512 / BM) + lane / (BM / 8);
#pragma unroll
  for (int u = 0; u < LC; ++u) ce[u] = C_ALONG ? ((lane & 7) ^ col_shift((wave * LC + u) * 8 + along_r)) * 8
                                               : (wave * LC + u) * (512 / BN) + lane / (BN / 8);
  int32_t look[FORM == kGradient ? LC : LR];  // source rows: of the next tile, of the gradient's next step
  auto look_up_rows = [&](const Tile& t) {
    if (FORM != kGradient) {
#pragma unroll
      for (int u = 0; u < LR; ++u)
        look[u] = (int32_t)source_row(order, t.pbegin + min((wave * LR + u) * 8 + along_r, t.rn - 1), slots, xrows);
    }
  };
  auto look_up_step = [&](int64_t pbegin, int rest) {  // a step from grouped row pbegin on, `rest` rows are left
    if (FORM == kGradient) {
#pragma unroll
      for (int u = 0; u < LC; ++u) look[u] = ce[u] < rest ? (int32_t)source_row(order, pbegin + ce[u], slots, xrows) : -1;
    }
  };
  auto mask_rows = [&](int left) {  // the last step: what lies behind the end
#pragma unroll
    for (int u = 0; u < LR; ++u) rp[u] = re[u] < left ? rp[u] : zero;
  };
  auto mask_cols = [&](int left) {
#pragma unroll
    for (int u = 0; u < LC; ++u) cp[u] = ce[u] < left ? cp[u] : zero;
  };
  auto begin_rows = [&](const Tile& t) {
#pragma unroll
    for (int u = 0; u < LR; ++u) {
      if (R_ALONG)
        rp[u] = rmat + (look[u] < 0 ? 0 : look[u]) * ldr + re[u];
      else
        rp[u] = rmat + (t.pbegin + re[u]) * ldr + t.r0 + min((lane % (BM / 8) ^ (across_shift(re[u]) << 1)) * 8, t.rn - 8);
    }
    if (t.length < kStep) mask_rows(t.length);
  };
  auto col_of = [&](int c0, int cn, int u) { return c0 + min((lane % (BN / 8) ^ (across_shift(ce[u]) << 1)) * 8, cn - 8); };
  auto step_cols = [&](int c0, int cn) {  // gradient: the rows that were looked up
#pragma unroll
    for (int u = 0; u < LC; ++u) cp[u] = look[u] < 0 ? zero : cmat + look[u] * ldc + col_of(c0, cn, u);
  };
  auto begin_cols = [&](const Tile& t) {
    if (FORM == kGradient) {
      step_cols(t.c0, t.cn);
      return;
    }
    const T* base = cmat + (int64_t)t.group * ldg;
#pragma unroll
    for (int u = 0; u < LC; ++u) {
      if (C_ALONG)
        cp[u] = base + (int64_t)(t.c0 + min((wave * LC + u) * 8 + along_r, t.cn - 1)) * ldc + ce[u];
      else
        cp[u] = base + ce[u] * ldc + col_of(t.c0, t.cn, u);
    }
    if (t.length < kStep) mask_cols(t.length);
  };
  auto fetch_row = [&](int u, int buffer) { piece_to_lds(rp[u], lds + buffer * BUFFER + (wave * LR + u) * 512); };
  auto fetch_col = [&](int u, int buffer) { piece_to_lds(cp[u], lds + buffer * BUFFER + (wave * LC + u) * 512); };

  f32x4 acc[FR][FC];
  auto clear = [&]() {
#pragma unroll
    for (int a = 0; a < FR; ++a)
#pragma unroll
      for (int b = 0; b < FC; ++b) acc[a][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  };
  int sub = lane & 15, quad = lane >> 4;
  auto col_fragments = [&](int buffer, int kk, Chunk (&f)[FC]) {
    const T* tile = lds + buffer * BUFFER;
#pragma unroll
    for (int b = 0; b < FC; ++b) {
      if (C_ALONG) {
        const int c = wc + fragment_col(b, sub);
        f[b] = along_piece(tile, c, col_shift(c), kk * 4 + quad);
      } else {
        f[b] = across_piece<T, BN>(tile, wc + fragment_col(b, (sub & 3) * 4), kk * 32 + quad * 8 + (sub >> 2));
      }
    }
  };
  auto row_fragments = [&](int buffer, int kk, int pair, Chunk (&f)[2]) {
    const T* tile = lds + buffer * BUFFER;
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      const int r = wr + (pair * 2 + a) * 16;
      if (R_ALONG)
        f[a] = along_piece(tile, r + sub, row_shift(r + sub), kk * 4 + quad);
      else
        f[a] = across_piece<T, BM>(tile, r + (sub & 3) * 4, kk * 32 + quad * 8 + (sub >> 2));
    }
  };
  auto multiply = [&](int pair, const Chunk (&fr)[2], const Chunk (&fc)[FC]) {
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int b = 0; b < FC; ++b) acc[pair * 2 + a][b] = Matrix<T>::mma(fc[b], fr[a], acc[pair * 2 + a][b]);
  };
  auto store = [&](const Tile& t) {
    T* base = FORM == kGradient ? out + (int64_t)t.group * ldog + (int64_t)t.r0 * ldo : out + t.pbegin * ldo;
    const int64_t known = xrows * slots;
#pragma unroll
    for (int a = 0; a < FR; ++a) {
      const int row = wr + a * 16 + sub;
      if (row >= t.rn) continue;
      T* orow = base + row * ldo + t.c0;
      const bool none = FORM != kGradient && order && (uint32_t)order[t.pbegin + row] >= known;  // a row of zeros
#pragma unroll
      for (int b = 0; b < FC; b += 2) {
        const int col = wc + fragment_col(b, quad * 4);
        if (col < t.cn) {  // widths are whole pieces
          Part q;
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            q[u] = static_cast<T>(none ? 0.0f : acc[a][b][u]);
            q[u + 4] = static_cast<T>(none ? 0.0f : acc[a][b + 1][u]);
          }
          *reinterpret_cast<Part*>(orow + col) = q;
        }
      }
    }
  };

  // A step in two halves of PAIRS phases of two row fragments each; while a phase's products run the next one's values come out of
  // LDS and a few loads are issued (all at once they hold the waves up for as long as they take to issue).  In the first half
  // these are the columns' operand of the step after the next; in the second one, after a meeting behind which nobody reads this
  // step's columns' operand any more, the rows' operand of that step into its place.  Before the last phase the waves meet again:
  // there this step's rows' operand has been read by all as well, and all of the next step has arrived.
  constexpr int PAIRS = FR / 2, CL = LC / PAIRS;
  static_assert(CL * PAIRS == LC, "");
  constexpr int EARLY = PAIRS > 2 ? LR / PAIRS * (PAIRS - 2) : 0;  // loads of the rows' operand before the second meeting
  Tile tile, next;
  int64_t index = 0;
  if (count > 0 && tile_at(0, tile)) {
    clear();
    Chunk fr[2][2], fc[2][FC];
    constexpr int LEAST = FORM == kGradient ? 3 : 2;
    auto steps_of = [&](const Tile& t) { return max(LEAST, (t.length + kStep - 1) / kStep); };
    int left = steps_of(tile);                            // steps of this tile
    int fleft = left, ftail = tile.length;                // steps and rest of the contraction where the pointers stand
    int fc0 = tile.c0, fcn = tile.cn;                     // and its columns
    int64_t lbegin = tile.pbegin;                         // the same where rows are looked up, a step further
    int lleft = left, ltail = tile.length;
    bool more;
    auto look_further = [&]() {
      if (FORM != kGradient) return;
      if (--lleft > 0) {
        lbegin += kStep;
        ltail -= kStep;
      } else if (more) {
        lleft = steps_of(next);
        lbegin = next.pbegin;
        ltail = next.length;
      } else {
        lleft = 1;
        ltail = 0;
      }
      look_up_step(lbegin, ltail);
    };
    auto advance = [&]() {
      if (--fleft > 0) {
        ftail -= kStep;
#pragma unroll
        for (int u = 0; u < LR; ++u) rp[u] += R_ALONG ? (int64_t)kStep : kStep * ldr;
        if (FORM == kGradient) {
          step_cols(fc0, fcn);
        } else {
#pragma unroll
          for (int u = 0; u < LC; ++u) cp[u] += C_ALONG ? (int64_t)kStep : kStep * ldc;
        }
        if (ftail < kStep) {
          mask_rows(ftail);
          if (FORM != kGradient) mask_cols(ftail);
        }
      } else if (more) {
        begin_rows(next);
        begin_cols(next);
        fleft = steps_of(next);
        ftail = next.length;
        fc0 = next.c0;
        fcn = next.cn;
      } else {  // nothing more: the same again, which nothing uses
        fleft = 1;
      }
      look_further();
    };
    auto look_ahead = [&]() {
      more = index + 1 < count && tile_at(index + 1, next);
      if (more) look_up_rows(next);
    };
    int cnow = 0, rnow = 1, cnext = 2, rnext = 3, ahead = 4;  // buffers of this step, of the next one, and the free one
    look_up_rows(tile);
    look_up_step(lbegin, ltail);
    begin_rows(tile);
    begin_cols(tile);
    look_ahead();
    look_further();
#pragma unroll
    for (int f = 0; f < 2; ++f) {
#pragma unroll
      for (int u = 0; u < LC; ++u) fetch_col(u, f ? cnext : cnow);
#pragma unroll
      for (int u = 0; u < LR; ++u) fetch_row(u, f ? rnext : rnow);
      advance();
    }
    meet<LR + LC>();
    col_fragments(cnow, 0, fc[0]);
    row_fragments(rnow, 0, 0, fr[0]);
    for (;;) {
      asm volatile("" : "+v"(sub), "+v"(quad));  // LDS addresses are made anew in every step: there are no registers to keep them
#pragma unroll
      for (int p = 0; p < PAIRS; ++p) {
        __builtin_amdgcn_sched_barrier(0);
        if (p + 1 < PAIRS) {
          row_fragments(rnow, 0, p + 1, fr[(p + 1) & 1]);
        } else {
          col_fragments(cnow, 1, fc[1]);
          row_fragments(rnow, 1, 0, fr[0]);
        }
#pragma unroll
        for (int u = 0; u < CL; ++u) fetch_col(p * CL + u, ahead);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
        multiply(p, fr[p & 1], fc[0]);
        __builtin_amdgcn_s_setprio(0);
      }
#pragma unroll
      for (int p = 0; p < PAIRS; ++p) {
        __builtin_amdgcn_sched_barrier(0);
        if (p == 1 && PAIRS > 2) read_by_all();
        if (p + 1 < PAIRS) {
          row_fragments(rnow, 1, p + 1, fr[(p + 1) & 1]);
        } else {
          meet<LC + EARLY>();
          col_fragments(cnext, 0, fc[0]);
          row_fragments(rnext, 0, 0, fr[0]);
        }
        if (p >= 1 && p + 1 < PAIRS) {
#pragma unroll
          for (int u = 0; u < LR / PAIRS; ++u) fetch_row((p - 1) * (LR / PAIRS) + u, cnow);
        }
        if (p + 1 == PAIRS) {
#pragma unroll
          for (int u = EARLY; u < LR; ++u) fetch_row(u, cnow);
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
        multiply(p, fr[p & 1], fc[1]);
        __builtin_amdgcn_s_setprio(0);
      }
      const int free = rnow, filled = cnow;
      cnow = cnext;
      rnow = rnext;
      cnext = ahead;
      rnext = filled;
      ahead = free;
      if (--left == 0) {
        store(tile);
        if (!more) break;
        clear();
        ++index;
        tile = next;
        left = steps_of(tile);
        look_ahead();
      }
      advance();
    }
    arrived();  // nothing may still be on its way into LDS when the workgroup gives it back
  }

  if (FORM != kGradient) {  // rows behind the last group
    const GroupRange g = group_range(offsets, groups, rows, groups);
    const int parts = outc / 8;
    const int64_t count = (g.end - g.begin) * parts;
    Part q;
#pragma unroll
    for (int u = 0; u < 8; ++u) q[u] = static_cast<T>(0.0f);
    for (int64_t i = (int64_t)blockIdx.x * (NW * 64) + tid; i < count; i += (int64_t)gridDim.x * (NW * 64))
      *reinterpret_cast<Part*>(out + (g.begin + i / parts) * ldo + i % parts * 8) = q;
  }
}

template <typename T>
bool whole_chunks(const void* p, int64_t ld) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % Matrix<T>::kChunk == 0;
}

template <typename T, int RF>
hipError_t thin_typed(const GroupedArgs& a, hipStream_t st) {
  const int tiles = (a.N + 15) / 16;
  const int64_t met = a.rows < a.groups ? a.rows : a.groups;  // groups with rows, at most
  // about 2,048 waves at work
  const int ks = met * tiles >= 2048 ? 1 : met * tiles >= 1024 ? 2 : 4;
  const int cols = (tiles + 4 / ks - 1) / (4 / ks);
  const int64_t blocks = tile_bound(a.rows, a.groups, RF * 16, cols);
  if (blocks > 0x7fffffff) return hipErrorInvalidConfiguration;
  const int whole = a.N % 4 == 0 && a.ldy % 4 == 0 && reinterpret_cast<uintptr_t>(a.y) % (4 * sizeof(T)) == 0;
  if (ks == 1)
    grouped_thin_kernel<T, RF, 1><<<(uint32_t)blocks, 256, 0, st>>>(a, cols, whole);
  else if (ks == 2)
    grouped_thin_kernel<T, RF, 2><<<(uint32_t)blocks, 256, 0, st>>>(a, cols, whole);
  else
    grouped_thin_kernel<T, RF, 4><<<(uint32_t)blocks, 256, 0, st>>>(a, cols, whole);
  return hipGetLastError();
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
  const bool tiled = sizeof(T) == 2 && wide && whole_chunks<T>(a.y, a.ldy);
  if (!transpose) {
    // Up to 8 rows a group the matrices are what takes time, and the kernel for few rows reads them as fast as any (64 groups of
    // 1024 x 2048 in 16 bits, 64 rows 53 us, tiles 57; 512 rows 73 and 72; in 32 bits 72, tiles of 64 x 64 91).  Beyond, tiles read
    // them less often (1,024 rows 89 and 72), but where there are few of them a good part of the chip has nothing to do (256 rows,
    // 4 groups of 2048 x 2048 32 us, tiles 49).
    const int side = tiled ? 256 : kTile;
    const int64_t row_tiles = a.rows / side + a.groups, tiles = (row_tiles < a.rows ? row_tiles : a.rows) * ((a.N + side - 1) / side);
    if (a.rows <= (int64_t)8 * a.groups) return thin_typed<T, 1>(a, st);
    if (tiles < (tiled ? 128 : 512) && a.rows <= (int64_t)64 * a.groups)
      return a.rows <= (int64_t)24 * a.groups ? thin_typed<T, 2>(a, st) : thin_typed<T, 4>(a, st);
  }
  if constexpr (sizeof(T) == 2) {
    if (tiled) {
      constexpr int BM = 256, BN = 256;
      const int wcols = (outc + BN - 1) / BN;
      const int64_t n = tile_bound(a.rows, a.groups, BM, wcols);
      const uint32_t grid = (uint32_t)(n < 256 ? n : 256);
      if (transpose)
        grouped_tile_kernel<T, kTransposed, BM, BN, 2, 4><<<grid, 512, 0, st>>>(
            x, w, y, a.offsets, a.order, a.ldx, a.ldw, a.ldg, a.ldy, 0, a.rows, a.xrows, a.groups, a.slots, 0, outc, depth, 0, wcols);
      else
        grouped_tile_kernel<T, kProduct, BM, BN, 2, 4><<<grid, 512, 0, st>>>(
            x, w, y, a.offsets, a.order, a.ldx, a.ldw, a.ldg, a.ldy, 0, a.rows, a.xrows, a.groups, a.slots, 0, outc, depth, 0, wcols);
      return hipGetLastError();
    }
  }
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
  if constexpr (sizeof(T) == 2) {
    if (wide && whole_chunks<T>(a.dw, a.ldw) && a.ldg % CH == 0) {
      constexpr int BM = 256, BN = 256;
      const int wr = (a.N + BM - 1) / BM, wc = (a.K + BN - 1) / BN;
      const int64_t n = (int64_t)a.groups * wr * wc;
      grouped_tile_kernel<T, kGradient, BM, BN, 2, 4><<<(uint32_t)(n < 256 ? n : 256), 512, 0, st>>>(
          dy, x, dw, a.offsets, a.order, a.lddy, a.ldx, 0, a.ldw, a.ldg, a.rows, a.xrows, a.groups, a.slots, a.N, a.K, 0, wr, wc);
      return hipGetLastError();
    }
  }
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
