// The assignment of rows to clusters and what goes with it: the t best clusters of every row with their softmax weights, the
// rows grouped by cluster, the gradient of the scores, and the weighted sum that brings a row's t results together again.
#include "experts.h"

#include <math.h>

namespace sceig {
namespace {

constexpr int kThreads = 256;
constexpr int kWave = 64;
constexpr float kNone = -INFINITY;

// ---- the assignment ---------------------------------------------------------------------------------------------------
// LANES lanes hold a row, lane l its scores l * VPL ... l * VPL + VPL - 1: of lanes that hold the same largest score the first
// then holds the lowest index, and the loads are wide.
template <int LANES>
__device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int s = 1; s < LANES; s <<= 1) v = fmaxf(v, __shfl_xor(v, s));
  return v;
}
template <int LANES>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int s = 1; s < LANES; s <<= 1) v += __shfl_xor(v, s);
  return v;
}

template <typename T, int VPL, bool WIDE>
__device__ __forceinline__ void load_scores(const T* row, const uint8_t* allowed, int first, int k, float (&v)[VPL]) {
  constexpr int E = WIDE ? (VPL * (int)sizeof(T) < 16 ? VPL : 16 / (int)sizeof(T)) : 1;  // scores a load
  typedef T Part __attribute__((ext_vector_type(E)));
  typedef uint8_t Bytes __attribute__((ext_vector_type(E)));
#pragma unroll
  for (int c = 0; c < VPL; c += E) {
    if (first + c < k) {
      if constexpr (E == 1) {
        v[c] = static_cast<float>(row[first + c]);
        if (allowed && !allowed[first + c]) v[c] = kNone;
      } else {
        const Part p = *reinterpret_cast<const Part*>(row + first + c);
#pragma unroll
        for (int u = 0; u < E; ++u) v[c + u] = static_cast<float>(p[u]);
        if (allowed) {
          const Bytes b = *reinterpret_cast<const Bytes*>(allowed + first + c);
#pragma unroll
          for (int u = 0; u < E; ++u) v[c + u] = b[u] ? v[c + u] : kNone;
        }
      }
#pragma unroll
      for (int u = 0; u < E; ++u) v[c + u] = v[c + u] > kNone ? v[c + u] : kNone;  // NaN too
    } else {
#pragma unroll
      for (int u = 0; u < E; ++u) v[c + u] = kNone;
    }
  }
}

// A workgroup takes `chunk` rows (a multiple of the rows that it holds at once) and leaves in hist[blockIdx.x * k + c] how many
// of their choices are cluster c.
template <typename T, int LANES, int VPL, bool WIDE>
__global__ __launch_bounds__(kThreads) void route_kernel(const T* __restrict__ scores, int64_t ld,
                                                         const uint8_t* __restrict__ allowed, int64_t lda, int64_t n, int k, int t,
                                                         int normalize, int chunk, int32_t* __restrict__ idx,
                                                         float* __restrict__ weight, int32_t* __restrict__ hist) {
  extern __shared__ int32_t count[];
  for (int c = threadIdx.x; c < k; c += kThreads) count[c] = 0;
  __syncthreads();
  constexpr int ROWS = kThreads / LANES;
  const int lane = threadIdx.x & (LANES - 1);
  const int first = lane * VPL;
  const int shift = (threadIdx.x & (kWave - 1)) & ~(LANES - 1);
  const int64_t end = min(n, (int64_t)(blockIdx.x + 1) * chunk);
  for (int64_t i = (int64_t)blockIdx.x * chunk + threadIdx.x / LANES; i < end; i += ROWS) {
    float v[VPL];
    load_scores<T, VPL, WIDE>(scores + i * ld, allowed ? allowed + i * lda : nullptr, first, k, v);
    float top = 0.0f, total = 0.0f, mine = 0.0f;
    int at = -1;
    for (int s = 0; s < t; ++s) {
      float best = v[0];
#pragma unroll
      for (int c = 1; c < VPL; ++c) best = fmaxf(best, v[c]);
      const float m = group_max<LANES>(best);
      if (s == 0) {
        top = m > kNone ? m : 0.0f;
        if (!normalize) {
          float sum = 0.0f;
#pragma unroll
          for (int c = 0; c < VPL; ++c) sum += expf(v[c] - top);
          total = group_sum<LANES>(sum);
        }
      }
      uint64_t who = __ballot(best == m && m > kNone) >> shift;
      if constexpr (LANES < 64) who &= (1ull << LANES) - 1;
      const bool found = who != 0;
      const int owner = found ? __ffsll((unsigned long long)who) - 1 : 0;
      int c0 = 0;
      if (found && lane == owner) {
        bool hit = false;
#pragma unroll
        for (int c = 0; c < VPL; ++c) {
          if (!hit && v[c] == m) {
            hit = true;
            c0 = c;
            v[c] = kNone;
          }
        }
        atomicAdd(&count[first + c0], 1);
      }
      const int chosen = __shfl(c0, shift + owner) + owner * VPL;
      const float e = expf(m - top);
      if (normalize && found) total += e;
      if (lane == s && found) {
        at = chosen;
        mine = e;
      }
    }
    if (lane < t) {
      idx[i * t + lane] = at;
      weight[i * t + lane] = at >= 0 ? mine / total : 0.0f;
    }
  }
  __syncthreads();
  for (int c = threadIdx.x; c < k; c += kThreads) hist[(int64_t)blockIdx.x * k + c] = count[c];
}

// hist[b * k + c] becomes the number of choices of cluster c in the workgroups before b; totals[c] their number in all.
__global__ __launch_bounds__(kThreads) void route_scan_kernel(int32_t* __restrict__ hist, int blocks, int k,
                                                              int32_t* __restrict__ totals) {
  const int c = blockIdx.x * kThreads + threadIdx.x;
  if (c >= k) return;
  int32_t sum = 0;
  for (int b = 0; b < blocks; ++b) {
    const int32_t h = hist[(int64_t)b * k + c];
    hist[(int64_t)b * k + c] = sum;
    sum += h;
  }
  totals[c] = sum;
}

// One wave a chunk puts the chunk's slots in their places, 64 at a time in slot order: a lane's place is what its cluster has
// taken so far plus the lanes before it with the same cluster, found by one ballot for every bit of the cluster's number.
__global__ __launch_bounds__(kWave) void route_place_kernel(const int32_t* __restrict__ idx, int64_t n, int k, int t, int chunk,
                                                            const int32_t* __restrict__ hist, const int32_t* __restrict__ totals,
                                                            int32_t* __restrict__ offsets, int32_t* __restrict__ order,
                                                            int32_t* __restrict__ place) {
  extern __shared__ int32_t next[];
  const int lane = threadIdx.x;
  int32_t before = 0;
  for (int c0 = 0; c0 < k; c0 += kWave) {  // exclusive sum of the totals
    const int c = c0 + lane;
    const int32_t own = c < k ? totals[c] : 0;
    int32_t sum = own;
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) {
      const int32_t o = __shfl_up(sum, s);
      if (lane >= s) sum += o;
    }
    if (c < k) {
      next[c] = before + sum - own + hist[(int64_t)blockIdx.x * k + c];
      if (blockIdx.x == 0) offsets[c] = before + sum - own;
    }
    before += __shfl(sum, kWave - 1);
  }
  if (blockIdx.x == 0 && lane == 0) offsets[k] = before;
  __syncthreads();
  int bits = 0;
  while ((1 << bits) < k) ++bits;
  const int64_t begin = (int64_t)blockIdx.x * chunk * t, end = min(n, (int64_t)(blockIdx.x + 1) * chunk) * t;
  for (int64_t f0 = begin; f0 < end; f0 += kWave) {
    const int64_t f = f0 + lane;
    const int32_t c = f < end ? idx[f] : -1;
    uint64_t same = __ballot(c >= 0);
    for (int b = 0; b < bits; ++b) {
      const bool set = (c >> b) & 1;
      const uint64_t m = __ballot(set);
      same &= set ? m : ~m;
    }
    if (c >= 0) {
      const int rank = __popcll(same & ((1ull << lane) - 1));
      const int32_t p = next[c] + rank;
      place[f] = p;
      order[p] = (int32_t)f;
      if ((same >> lane) == 1ull) next[c] = p + 1;  // the last of them; after every lane has read, in program order
    } else if (f < end) {
      place[f] = -1;
    }
    if (f < end && f >= before) order[f] = -1;
    __syncthreads();
  }
}

int route_chunk(int64_t n, int k) {
  // At most 1,024 workgroups, and counters of at most 2^20 words for all of them: the scan reads them all.
  int64_t blocks = (int64_t)(1 << 20) / k;
  if (blocks > 1024) blocks = 1024;
  if (blocks < 1) blocks = 1;
  const int64_t rows = (n + blocks - 1) / blocks;
  return (int)((rows + 15) / 16 * 16);
}
int route_blocks(int64_t n, int k) { return (int)((n + route_chunk(n, k) - 1) / route_chunk(n, k)); }

template <typename T, int LANES, int VPL>
hipError_t route_typed(const T* scores, int64_t ld, const uint8_t* allowed, int64_t lda, int64_t n, int k, int t, bool normalize,
                       int32_t* idx, float* weight, int32_t* hist, hipStream_t st) {
  constexpr int E = VPL * (int)sizeof(T) < 16 ? VPL : 16 / (int)sizeof(T);
  const bool wide = k % E == 0 && ld % E == 0 && reinterpret_cast<uintptr_t>(scores) % (E * sizeof(T)) == 0 &&
                    (!allowed || (lda % E == 0 && reinterpret_cast<uintptr_t>(allowed) % E == 0));
  const int chunk = route_chunk(n, k), blocks = route_blocks(n, k);
  const size_t lds = sizeof(int32_t) * k;
  if (wide)
    route_kernel<T, LANES, VPL, true><<<blocks, kThreads, lds, st>>>(scores, ld, allowed, lda, n, k, t, normalize, chunk, idx,
                                                                    weight, hist);
  else
    route_kernel<T, LANES, VPL, false><<<blocks, kThreads, lds, st>>>(scores, ld, allowed, lda, n, k, t, normalize, chunk, idx,
                                                                     weight, hist);
  return hipGetLastError();
}

template <typename T>
hipError_t route_sized(const T* s, int64_t ld, const uint8_t* a, int64_t lda, int64_t n, int k, int t, bool norm, int32_t* idx,
                       float* w, int32_t* hist, hipStream_t st) {
  if (k <= 16) return route_typed<T, 16, 1>(s, ld, a, lda, n, k, t, norm, idx, w, hist, st);
  if (k <= 32) return route_typed<T, 16, 2>(s, ld, a, lda, n, k, t, norm, idx, w, hist, st);
  if (k <= 64) return route_typed<T, 16, 4>(s, ld, a, lda, n, k, t, norm, idx, w, hist, st);
  if (k <= 128) return route_typed<T, 16, 8>(s, ld, a, lda, n, k, t, norm, idx, w, hist, st);
  if (k <= 256) return route_typed<T, 64, 4>(s, ld, a, lda, n, k, t, norm, idx, w, hist, st);
  if (k <= 512) return route_typed<T, 64, 8>(s, ld, a, lda, n, k, t, norm, idx, w, hist, st);
  if (k <= 1024) return route_typed<T, 64, 16>(s, ld, a, lda, n, k, t, norm, idx, w, hist, st);
  if (k <= 2048) return route_typed<T, 64, 32>(s, ld, a, lda, n, k, t, norm, idx, w, hist, st);
  return route_typed<T, 64, 64>(s, ld, a, lda, n, k, t, norm, idx, w, hist, st);
}

// ---- gradient of the scores ---------------------------------------------------------------------------------------------
// With c = sum_s w_s dw_s: dS = p (dw - c) on the chosen clusters (dw = 0 elsewhere), p the softmax weight over the chosen or
// over all allowed clusters, and 0 where p is.  For weights over the chosen p = w there and nothing else is read.
template <typename T, int LANES, int VPL, bool WIDE>
__global__ __launch_bounds__(kThreads) void route_backward_kernel(const T* __restrict__ scores, int64_t ld,
                                                                  const uint8_t* __restrict__ allowed, int64_t lda, int64_t n, int k,
                                                                  int t, int normalize, const int32_t* __restrict__ idx,
                                                                  const float* __restrict__ weight,
                                                                  const float* __restrict__ dweight, T* __restrict__ dscores,
                                                                  int64_t ldd) {
  constexpr int ROWS = kThreads / LANES;
  const int lane = threadIdx.x & (LANES - 1);
  const int first = lane * VPL;
  const int shift = (threadIdx.x & (kWave - 1)) & ~(LANES - 1);
  const int64_t i = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES;
  if (i >= n) return;
  int32_t at = -1;
  float w = 0.0f, dw = 0.0f;
  if (lane < t) {
    at = idx[i * t + lane];
    if (at >= 0) {
      w = weight[i * t + lane];
      dw = dweight[i * t + lane];
    }
  }
  const float c = group_sum<16>(w * dw);  // t <= 16: the sum over the first 16 lanes
  const float mean = __shfl(c, shift);
  float g[VPL];
  if (normalize) {
#pragma unroll
    for (int u = 0; u < VPL; ++u) g[u] = 0.0f;
    const float mine = w * (dw - mean);
    for (int s = 0; s < t; ++s) {
      const int j = __shfl(at, shift + s) - first;
      const float x = __shfl(mine, shift + s);
#pragma unroll
      for (int u = 0; u < VPL; ++u) g[u] = j == u ? x : g[u];
    }
  } else {
    float v[VPL];
    load_scores<T, VPL, WIDE>(scores + i * ld, allowed ? allowed + i * lda : nullptr, first, k, v);
    float best = v[0];
#pragma unroll
    for (int u = 1; u < VPL; ++u) best = fmaxf(best, v[u]);
    best = group_max<LANES>(best);
    const float top = best > kNone ? best : 0.0f;
    float sum = 0.0f;
#pragma unroll
    for (int u = 0; u < VPL; ++u) {
      v[u] = expf(v[u] - top);
      sum += v[u];
      g[u] = -mean;
    }
    sum = group_sum<LANES>(sum);
    for (int s = 0; s < t; ++s) {
      const int j = __shfl(at, shift + s) - first;
      const float x = __shfl(dw, shift + s) - mean;
#pragma unroll
      for (int u = 0; u < VPL; ++u) g[u] = j == u ? x : g[u];
    }
#pragma unroll
    for (int u = 0; u < VPL; ++u) g[u] = v[u] != 0.0f ? v[u] / sum * g[u] : 0.0f;
  }
  constexpr int E = WIDE ? (VPL * (int)sizeof(T) < 16 ? VPL : 16 / (int)sizeof(T)) : 1;
  typedef T Part __attribute__((ext_vector_type(E)));
  T* out = dscores + i * ldd;
#pragma unroll
  for (int u = 0; u < VPL; u += E) {
    if (first + u < k) {
      if constexpr (E == 1) {
        out[first + u] = static_cast<T>(g[u]);
      } else {
        Part p;
#pragma unroll
        for (int e = 0; e < E; ++e) p[e] = static_cast<T>(g[u + e]);
        *reinterpret_cast<Part*>(out + first + u) = p;
      }
    }
  }
}

template <typename T, int LANES, int VPL>
hipError_t route_backward_typed(const T* scores, int64_t ld, const uint8_t* allowed, int64_t lda, int64_t n, int k, int t,
                                bool normalize, const int32_t* idx, const float* weight, const float* dweight, T* ds,
                                int64_t ldd, hipStream_t st) {
  constexpr int E = VPL * (int)sizeof(T) < 16 ? VPL : 16 / (int)sizeof(T);
  const bool wide = k % E == 0 && ld % E == 0 && ldd % E == 0 && reinterpret_cast<uintptr_t>(scores) % (E * sizeof(T)) == 0 &&
                    reinterpret_cast<uintptr_t>(ds) % (E * sizeof(T)) == 0 &&
                    (!allowed || (lda % E == 0 && reinterpret_cast<uintptr_t>(allowed) % E == 0));
  const int64_t blocks = (n + kThreads / LANES - 1) / (kThreads / LANES);
  if (wide)
    route_backward_kernel<T, LANES, VPL, true><<<(uint32_t)blocks, kThreads, 0, st>>>(scores, ld, allowed, lda, n, k, t, normalize,
                                                                                     idx, weight, dweight, ds, ldd);
  else
    route_backward_kernel<T, LANES, VPL, false><<<(uint32_t)blocks, kThreads, 0, st>>>(scores, ld, allowed, lda, n, k, t,
                                                                                      normalize, idx, weight, dweight, ds, ldd);
  return hipGetLastError();
}

template <typename T>
hipError_t route_backward_sized(const T* s, int64_t ld, const uint8_t* a, int64_t lda, int64_t n, int k, int t, bool norm,
                                const int32_t* idx, const float* w, const float* dw, T* ds, int64_t ldd, hipStream_t st) {
  if (k <= 16) return route_backward_typed<T, 16, 1>(s, ld, a, lda, n, k, t, norm, idx, w, dw, ds, ldd, st);
  if (k <= 32) return route_backward_typed<T, 16, 2>(s, ld, a, lda, n, k, t, norm, idx, w, dw, ds, ldd, st);
  if (k <= 64) return route_backward_typed<T, 16, 4>(s, ld, a, lda, n, k, t, norm, idx, w, dw, ds, ldd, st);
  if (k <= 128) return route_backward_typed<T, 16, 8>(s, ld, a, lda, n, k, t, norm, idx, w, dw, ds, ldd, st);
  if (k <= 256) return route_backward_typed<T, 64, 4>(s, ld, a, lda, n, k, t, norm, idx, w, dw, ds, ldd, st);
  if (k <= 512) return route_backward_typed<T, 64, 8>(s, ld, a, lda, n, k, t, norm, idx, w, dw, ds, ldd, st);
  if (k <= 1024) return route_backward_typed<T, 64, 16>(s, ld, a, lda, n, k, t, norm, idx, w, dw, ds, ldd, st);
  if (k <= 2048) return route_backward_typed<T, 64, 32>(s, ld, a, lda, n, k, t, norm, idx, w, dw, ds, ldd, st);
  return route_backward_typed<T, 64, 64>(s, ld, a, lda, n, k, t, norm, idx, w, dw, ds, ldd, st);
}

// ---- weighted sum -------------------------------------------------------------------------------------------------------
// E values of a row at once: 16 bytes where the rows lie so, else one.
template <typename T, int E>
__device__ __forceinline__ void load_part(const T* p, float (&v)[E]) {
  if constexpr (E == 1) {
    v[0] = static_cast<float>(*p);
  } else {
    typedef T Part __attribute__((ext_vector_type(E)));
    const Part q = *reinterpret_cast<const Part*>(p);
#pragma unroll
    for (int u = 0; u < E; ++u) v[u] = static_cast<float>(q[u]);
  }
}
template <typename T, int E>
__device__ __forceinline__ void store_part(T* p, const float (&v)[E]) {
  if constexpr (E == 1) {
    *p = static_cast<T>(v[0]);
  } else {
    typedef T Part __attribute__((ext_vector_type(E)));
    Part q;
#pragma unroll
    for (int u = 0; u < E; ++u) q[u] = static_cast<T>(v[u]);
    *reinterpret_cast<Part*>(p) = q;
  }
}

// out_i = sum_s w_is z_place(i,s), added in the order of s, one thread an E of them.
template <typename T, int E>
__global__ __launch_bounds__(kThreads) void combine_kernel(const T* __restrict__ z, int64_t ldz, int64_t rows,
                                                           const int32_t* __restrict__ place, const float* __restrict__ weight,
                                                           int64_t n, int t, int parts, T* __restrict__ out, int64_t ldo) {
  const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t i = at / parts;
  if (i >= n) return;
  const int64_t j = (at - i * parts) * E;
  float sum[E];
#pragma unroll
  for (int u = 0; u < E; ++u) sum[u] = 0.0f;
  for (int s = 0; s < t; ++s) {
    const int32_t p = place[i * t + s];
    if (p < 0 || p >= rows) continue;
    const float w = weight ? weight[i * t + s] : 1.0f;
    float v[E];
    load_part<T, E>(z + p * ldz + j, v);
#pragma unroll
    for (int u = 0; u < E; ++u) sum[u] += w * v[u];
  }
  store_part<T, E>(out + i * ldo + j, sum);
}

// One workgroup a row: dz_p = w dout_i and dw = <dout_i, z_p> for its t places, and zeros into rows of dz where nothing has its
// place.
template <typename T, int E>
__global__ __launch_bounds__(kThreads) void combine_backward_kernel(const T* __restrict__ dout, int64_t ldo, const T* __restrict__ z,
                                                                    int64_t ldz, int64_t rows, const int32_t* __restrict__ place,
                                                                    const float* __restrict__ weight,
                                                                    const int32_t* __restrict__ order, int64_t n, int t, int d,
                                                                    T* __restrict__ dz, int64_t lddz, float* __restrict__ dweight) {
  __shared__ float part[kThreads / kWave];
  const int64_t i = blockIdx.x;
  for (int s = 0; s < t && i < n; ++s) {
    const int32_t p = place[i * t + s];
    float dot = 0.0f;
    if (p >= 0 && p < rows) {
      const float w = weight ? weight[i * t + s] : 1.0f;
      for (int j = threadIdx.x * E; j < d; j += kThreads * E) {
        float g[E], v[E], o[E];
        load_part<T, E>(dout + i * ldo + j, g);
#pragma unroll
        for (int u = 0; u < E; ++u) o[u] = w * g[u];
        store_part<T, E>(dz + p * lddz + j, o);
        if (dweight) {
          load_part<T, E>(z + p * ldz + j, v);
#pragma unroll
          for (int u = 0; u < E; ++u) dot += g[u] * v[u];
        }
      }
    }
    if (dweight) {
      dot = group_sum<kWave>(dot);
      if ((threadIdx.x & (kWave - 1)) == 0) part[threadIdx.x / kWave] = dot;
      __syncthreads();
      if (threadIdx.x == 0) {
        float sum = 0.0f;
        for (int q = 0; q < kThreads / kWave; ++q) sum += part[q];
        dweight[i * t + s] = sum;
      }
      __syncthreads();
    }
  }
  for (int64_t p = i; p < rows; p += gridDim.x) {
    if (order[p] >= 0) continue;
    float o[E];
#pragma unroll
    for (int u = 0; u < E; ++u) o[u] = 0.0f;
    for (int j = threadIdx.x * E; j < d; j += kThreads * E) store_part<T, E>(dz + p * lddz + j, o);
  }
}

template <typename T>
bool wide_rows(const void* p, int64_t ld) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % (16 / (int64_t)sizeof(T)) == 0;
}

template <typename T>
hipError_t combine_typed(const T* z, int64_t ldz, int64_t rows, const int32_t* place, const float* weight, int64_t n, int t, int d,
                         T* out, int64_t ldo, hipStream_t st) {
  constexpr int E = 16 / (int)sizeof(T);
  const bool wide = d % E == 0 && wide_rows<T>(z, ldz) && wide_rows<T>(out, ldo);
  const int parts = wide ? d / E : d;
  const int64_t blocks = (n * parts + kThreads - 1) / kThreads;
  if (wide)
    combine_kernel<T, E><<<(uint32_t)blocks, kThreads, 0, st>>>(z, ldz, rows, place, weight, n, t, parts, out, ldo);
  else
    combine_kernel<T, 1><<<(uint32_t)blocks, kThreads, 0, st>>>(z, ldz, rows, place, weight, n, t, parts, out, ldo);
  return hipGetLastError();
}

template <typename T>
hipError_t combine_backward_typed(const T* dout, int64_t ldo, const T* z, int64_t ldz, int64_t rows, const int32_t* place,
                                  const float* weight, const int32_t* order, int64_t n, int t, int d, T* dz, int64_t lddz,
                                  float* dweight, hipStream_t st) {
  constexpr int E = 16 / (int)sizeof(T);
  const uint32_t blocks = (uint32_t)(n > 0 ? n : 1);
  const bool wide = d % E == 0 && wide_rows<T>(dout, ldo) && wide_rows<T>(dz, lddz) && (!dweight || wide_rows<T>(z, ldz));
  if (wide)
    combine_backward_kernel<T, E><<<blocks, kThreads, 0, st>>>(dout, ldo, z, ldz, rows, place, weight, order, n, t, d, dz, lddz,
                                                               dweight);
  else
    combine_backward_kernel<T, 1><<<blocks, kThreads, 0, st>>>(dout, ldo, z, ldz, rows, place, weight, order, n, t, d, dz, lddz,
                                                               dweight);
  return hipGetLastError();
}

}  // namespace

size_t route_workspace(int64_t n, int k, int t) {
  (void)t;
  if (n == 0) return 0;
  return sizeof(int32_t) * ((size_t)route_blocks(n, k) * k + k);
}

__global__ __launch_bounds__(kThreads) void zero_words_kernel(int32_t* p, int count) {
  for (int c = threadIdx.x; c < count; c += kThreads) p[c] = 0;
}

hipError_t launch_route(const void* scores, int dtype, int64_t ld, const uint8_t* allowed, int64_t lda, int64_t n, int k, int t,
                        bool normalize, int32_t* idx, float* weight, int32_t* offsets, int32_t* order, int32_t* place,
                        void* work, hipStream_t st) {
  if (n == 0) {
    zero_words_kernel<<<1, kThreads, 0, st>>>(offsets, k + 1);
    return hipGetLastError();
  }
  const int blocks = route_blocks(n, k), chunk = route_chunk(n, k);
  int32_t* hist = static_cast<int32_t*>(work);
  int32_t* totals = hist + (size_t)blocks * k;
  hipError_t e;
  if (dtype == kF32)
    e = route_sized(static_cast<const float*>(scores), ld, allowed, lda, n, k, t, normalize, idx, weight, hist, st);
  else if (dtype == kBF16)
    e = route_sized(static_cast<const __bf16*>(scores), ld, allowed, lda, n, k, t, normalize, idx, weight, hist, st);
  else
    e = route_sized(static_cast<const _Float16*>(scores), ld, allowed, lda, n, k, t, normalize, idx, weight, hist, st);
  if (e != hipSuccess) return e;
  route_scan_kernel<<<(k + kThreads - 1) / kThreads, kThreads, 0, st>>>(hist, blocks, k, totals);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  route_place_kernel<<<blocks, kWave, sizeof(int32_t) * k, st>>>(idx, n, k, t, chunk, hist, totals, offsets, order, place);
  return hipGetLastError();
}

hipError_t launch_route_backward(const void* scores, int dtype, int64_t ld, const uint8_t* allowed, int64_t lda, int64_t n,
                                 int k, int t, bool normalize, const int32_t* idx, const float* weight, const float* dweight,
                                 void* dscores, int64_t ldd, hipStream_t st) {
  if (n == 0) return hipSuccess;
  if (dtype == kF32)
    return route_backward_sized(static_cast<const float*>(scores), ld, allowed, lda, n, k, t, normalize, idx, weight, dweight,
                                static_cast<float*>(dscores), ldd, st);
  if (dtype == kBF16)
    return route_backward_sized(static_cast<const __bf16*>(scores), ld, allowed, lda, n, k, t, normalize, idx, weight, dweight,
                                static_cast<__bf16*>(dscores), ldd, st);
  return route_backward_sized(static_cast<const _Float16*>(scores), ld, allowed, lda, n, k, t, normalize, idx, weight, dweight,
                              static_cast<_Float16*>(dscores), ldd, st);
}

hipError_t launch_group_combine(const void* z, int dtype, int64_t ldz, int64_t rows, const int32_t* place, const float* weight,
                                int64_t n, int t, int d, void* out, int64_t ldo, hipStream_t st) {
  if (n == 0) return hipSuccess;
  if (dtype == kF32)
    return combine_typed(static_cast<const float*>(z), ldz, rows, place, weight, n, t, d, static_cast<float*>(out), ldo, st);
  if (dtype == kBF16)
    return combine_typed(static_cast<const __bf16*>(z), ldz, rows, place, weight, n, t, d, static_cast<__bf16*>(out), ldo, st);
  return combine_typed(static_cast<const _Float16*>(z), ldz, rows, place, weight, n, t, d, static_cast<_Float16*>(out), ldo, st);
}

hipError_t launch_group_combine_backward(const void* dout, int dtype, int64_t ldo, const void* z, int64_t ldz, int64_t rows,
                                         const int32_t* place, const float* weight, const int32_t* order, int64_t n, int t,
                                         int d, void* dz, int64_t lddz, float* dweight, hipStream_t st) {
  if (n == 0 && rows == 0) return hipSuccess;
  if (dtype == kF32)
    return combine_backward_typed(static_cast<const float*>(dout), ldo, static_cast<const float*>(z), ldz, rows, place, weight,
                                  order, n, t, d, static_cast<float*>(dz), lddz, dweight, st);
  if (dtype == kBF16)
    return combine_backward_typed(static_cast<const __bf16*>(dout), ldo, static_cast<const __bf16*>(z), ldz, rows, place, weight,
                                  order, n, t, d, static_cast<__bf16*>(dz), lddz, dweight, st);
  return combine_backward_typed(static_cast<const _Float16*>(dout), ldo, static_cast<const _Float16*>(z), ldz, rows, place,
                                weight, order, n, t, d, static_cast<_Float16*>(dz), lddz, dweight, st);
}

}  // namespace sceig
