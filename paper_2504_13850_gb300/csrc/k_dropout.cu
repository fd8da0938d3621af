// Dropout from a counter-based generator, with the residual add, and its
// gradient: y = residual + keep(x) and dx = keep(dy).  No mask is stored; both
// directions draw the same bits again.
//
// Elements 8 g .. 8 g + 7 of the row-major matrix take the eight 16-bit
// halves (low half first) of Philox4x32-10 (Salmon, Moraes, Dror, Shaw:
// "Parallel random numbers: as easy as 1, 2, 3", SC 2011) with counter
// (g, call) and key seed.  An element is kept when its half is at least
// T = round(65536 p), so the drop probability is T / 65536 exactly, and is
// then scaled by 65536 / (65536 - T).  16 bits per element let one generator
// call serve one 16-byte vector of bf16, which keeps the integer work below
// the memory time.  A dropped element is replaced by zero, not multiplied, so
// an infinity or NaN in it does not spread.
#include "fo_common.cuh"
#include "../../include/fedoptima.h"

#include <cmath>
#include <string>

namespace fo {
int report_error(int code, const std::string& msg);

namespace {

struct DropParams {
  const void *x, *r;
  void* y;
  int64_t groups, n, cols, ldx, ldr, ldy;
  uint32_t key[20];        // both key words of each of the ten rounds
  uint32_t c2, c3, drop;
  float scale;
};

__device__ __forceinline__ uint4 philox(uint64_t g, const DropParams& p) {
  uint32_t c0 = uint32_t(g), c1 = uint32_t(g >> 32), c2 = p.c2, c3 = p.c3;
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = uint64_t(c0) * 0xD2511F53u, b = uint64_t(c2) * 0xCD9E8D57u;
    const uint32_t n0 = uint32_t(b >> 32) ^ c1 ^ p.key[2 * i], n2 = uint32_t(a >> 32) ^ c3 ^ p.key[2 * i + 1];
    c1 = uint32_t(b);
    c3 = uint32_t(a);
    c0 = n0;
    c2 = n2;
  }
  return make_uint4(c0, c1, c2, c3);
}

__device__ __forceinline__ float kept(float v, uint32_t word, int half, const DropParams& p) {
  const uint32_t u = half ? word >> 16 : word & 0xffffu;
  return u >= p.drop ? v * p.scale : 0.f;
}
// The same where p.drop < 65536, with floor = p.drop << 16: the half in the
// upper 16 bits compares as it stands.
__device__ __forceinline__ float kept_fast(float v, uint32_t word, int half, uint32_t floor, const DropParams& p) {
  return (half ? word : word << 16) >= floor ? v * p.scale : 0.f;
}

template <typename T> struct Vec8;
template <> struct Vec8<bf16> {
  uint4 a;
  __device__ __forceinline__ void load(const bf16* s) { a = *reinterpret_cast<const uint4*>(s); }
  __device__ __forceinline__ void store(bf16* d) const { *reinterpret_cast<uint4*>(d) = a; }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(w[e] << 16);
      v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
      w[e] = *reinterpret_cast<const uint32_t*>(&h);
    }
    a = make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <> struct Vec8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* s) {
    a = reinterpret_cast<const float4*>(s)[0];
    b = reinterpret_cast<const float4*>(s)[1];
  }
  __device__ __forceinline__ void store(float* d) const {
    reinterpret_cast<float4*>(d)[0] = a;
    reinterpret_cast<float4*>(d)[1] = b;
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
    a = make_float4(v[0], v[1], v[2], v[3]);
    b = make_float4(v[4], v[5], v[6], v[7]);
  }
};

// Rows of whole groups, 16-byte aligned (or one contiguous row: cols = n).
// Each thread has the vectors of U groups in flight while it draws their bits.
// One group: eight blocks, the whole grid, stay on an SM (at six, with more
// registers, the gradient of 134 M bf16 took 107 us instead of 89).
template <typename T, bool RES, int U>
__global__ void __launch_bounds__(256, U == 1 ? 8 : 2) dropout_vec_k(const __grid_constant__ DropParams p) {
  pdl_wait();
  pdl_trigger();
  const T *x = static_cast<const T*>(p.x), *r = static_cast<const T*>(p.r);
  T* y = static_cast<T*>(p.y);
  const int64_t step = int64_t(gridDim.x) * blockDim.x, whole = p.n / 8;
  const uint32_t floor = p.drop << 16;
  for (int64_t g0 = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; g0 < whole; g0 += U * step) {
    Vec8<T> a[U], c[U];
    T* out[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t g = g0 + u * step;
      if (g >= whole) break;
      const int64_t e = 8 * g, row = p.cols == p.n ? 0 : e / p.cols, col = e - row * p.cols;
      a[u].load(x + row * p.ldx + col);
      if (RES) c[u].load(r + row * p.ldr + col);
      out[u] = y + row * p.ldy + col;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t g = g0 + u * step;
      if (g >= whole) break;
      const uint4 b = philox(uint64_t(g), p);
      const uint32_t w[4] = {b.x, b.y, b.z, b.w};
      float v[8], z[8];
      a[u].get(v);
      if (RES) c[u].get(z);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        v[k] = kept_fast(v[k], w[k >> 1], k & 1, floor, p);
        if (RES) v[k] += z[k];
      }
      a[u].set(v);
      a[u].store(out[u]);
    }
  }
  // the last, partial group (only one contiguous row has one)
  if (p.n % 8 && blockIdx.x == 0 && threadIdx.x == 0) {
    const uint4 b = philox(uint64_t(whole), p);
    const uint32_t w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int k = 0; k < 7; ++k) {
      const int64_t e = 8 * whole + k;
      if (e >= p.n) break;
      float v = kept(to_f(x[e]), w[k >> 1], k & 1, p);
      if (RES) v += to_f(r[e]);
      y[e] = from_f<T>(v);
    }
  }
}

// Any strides and widths.
template <typename T, bool RES>
__global__ void __launch_bounds__(256) dropout_any_k(const __grid_constant__ DropParams p) {
  pdl_wait();
  pdl_trigger();
  const T *x = static_cast<const T*>(p.x), *r = static_cast<const T*>(p.r);
  T* y = static_cast<T*>(p.y);
  const int64_t step = int64_t(gridDim.x) * blockDim.x;
  for (int64_t g = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; g < p.groups; g += step) {
    const uint4 u = philox(uint64_t(g), p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    int64_t row = 8 * g / p.cols, col = 8 * g - row * p.cols;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (8 * g + k >= p.n) break;
      float v = kept(to_f(x[row * p.ldx + col]), w[k >> 1], k & 1, p);
      if (RES) v += to_f(r[row * p.ldr + col]);
      y[row * p.ldy + col] = from_f<T>(v);
      if (++col == p.cols) {
        col = 0;
        ++row;
      }
    }
  }
}

template <typename T>
cudaError_t dropout(DropParams p, cudaStream_t st) {
  const int64_t rows = p.n / p.cols;
  if (rows == 1 || (p.ldx == p.cols && p.ldy == p.cols && (!p.r || p.ldr == p.cols))) {
    p.cols = p.n;      // one contiguous row
    p.ldx = p.ldy = p.ldr = 0;
  }
  auto wide = [](const void* q) { return reinterpret_cast<uintptr_t>(q) % 16 == 0; };
  const int64_t per = 16 / sizeof(T);
  const bool vec = p.drop < 65536u && wide(p.x) && wide(p.y) && (!p.r || wide(p.r)) &&
                   (p.cols == p.n || (p.cols % 8 == 0 && p.ldx % per == 0 && p.ldy % per == 0 &&
                                      (!p.r || p.ldr % per == 0)));
  const int full = elementwise_blocks(INT64_MAX / 2, 256);        // eight blocks per SM
  // fp32 is bound by memory and wants two groups in flight per thread once
  // there are enough (134 M elements: 6.8 TB/s against 5.9); bf16, with twice
  // the elements per byte, is bound by the generator and wants the occupancy
  // of one
  auto go = [&](auto kernel, int u) {
    const int64_t want = (p.groups + 256 * u - 1) / (256 * u);
    return launch_k(kernel, dim3(unsigned(want < full ? want : full)), dim3(256), 0, st, p);
  };
  if (!vec) return go(p.r ? dropout_any_k<T, true> : dropout_any_k<T, false>, 1);
  if (sizeof(T) == 4 && p.groups >= int64_t(full) * 256)
    return go(p.r ? dropout_vec_k<T, true, 2> : dropout_vec_k<T, false, 2>, 2);
  return go(p.r ? dropout_vec_k<T, true, 1> : dropout_vec_k<T, false, 1>, 1);
}

}  // namespace
}  // namespace fo

extern "C" int fo_dropout_add(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, void* y,
                              int64_t y_stride, int dtype, int64_t rows, int64_t cols, double p, uint64_t seed,
                              uint64_t call, void* stream) {
  using namespace fo;
  if (dtype != FO_DTYPE_F32 && dtype != FO_DTYPE_BF16) return report_error(FO_ERR_ARG, "dropout: unknown dtype");
  if (rows < 0 || cols < 0 || (cols > 0 && rows > INT64_MAX / 8 / cols))
    return report_error(FO_ERR_ARG, "dropout: rows or cols out of range");
  if (!(p >= 0.0 && p <= 1.0)) return report_error(FO_ERR_ARG, "dropout: p must be in [0, 1]");
  if (rows == 0 || cols == 0) return FO_OK;
  const size_t size = dtype == FO_DTYPE_F32 ? 4 : 2;
  auto odd = [size](const void* q) { return reinterpret_cast<uintptr_t>(q) % size != 0; };
  if (!x || !y || odd(x) || odd(y) || (residual && odd(residual)))
    return report_error(FO_ERR_ARG, "dropout: null or misaligned pointer");
  if (rows > 1 && (x_stride < 0 || y_stride < cols || (residual && residual_stride < 0)))
    return report_error(FO_ERR_ARG, "dropout: bad row stride");
  DropParams d;
  d.x = x;
  d.r = residual;
  d.y = y;
  d.n = rows * cols;
  d.groups = (d.n + 7) / 8;
  d.cols = cols;
  d.ldx = x_stride;
  d.ldr = residual_stride;
  d.ldy = y_stride;
  for (uint32_t i = 0; i < 10; ++i) {
    d.key[2 * i] = uint32_t(seed) + i * 0x9E3779B9u;
    d.key[2 * i + 1] = uint32_t(seed >> 32) + i * 0xBB67AE85u;
  }
  d.c2 = uint32_t(call);
  d.c3 = uint32_t(call >> 32);
  d.drop = uint32_t(std::nearbyint(65536.0 * p));
  d.scale = d.drop < 65536u ? float(65536.0 / (65536.0 - d.drop)) : 0.f;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == FO_DTYPE_F32 ? dropout<float>(d, st) : dropout<bf16>(d, st);
  return e == cudaSuccess ? FO_OK : report_error(FO_ERR_CUDA, cudaGetErrorString(e));
}
