// Root-mean-square norm of a residual's addition, its gradient, and its output
// as 8-bit floats with shared scales.
//
//   s = x + residual (rounded to the tensors' type);  r = (mean s^2 + eps)^(-1/2);  y = s r w
//   dx = r (w dy - s r^2 mean(w dy s)) + ds;          dw = sum over rows of dy s r
//
// The gradient is taken as r (w dy - z mean(w dy z)) + ds with z = s r: of r^2 and r^3
// either leaves fp32 where r alone and the result do not.
//
// A row's elements stay in registers between the sum of squares and the
// output, so that each tensor passes once: forward x, residual in, s, y out;
// backward dy, ds, s in, dx out.  Both are bound by HBM for large inputs and by
// the latency of a launch and one row's way through a warp or block for small.
#include "fo_vec8.cuh"
#include "../../include/fedoptima.h"

#include <cuda_fp8.h>
#include <atomic>
#include <string>

namespace fo {
int report_error(int code, const std::string& msg);

namespace {

constexpr int kMaxDevices = 64;

struct NormParams {
  const void *x, *r, *w;
  void *s, *y;
  uint8_t *q, *scales;
  float* rstd;
  int64_t ldx, ldr, lds, ldy;
  int rows, cols;
  float eps, inv_cols, inv_rest;       // 1 / cols, and what its rounding left
};
struct NormGradParams {
  const void *dy, *ds, *s, *w;
  const float* rstd;
  void* dx;
  float* part;             // [blocks][cols]
  int64_t lddy, ldds, lds, lddx;
  int rows, cols;
  float inv_cols;
};

// Which elements a thread of a row's G threads holds: chunk j's eight stand
// side by side (VEC), or G apart, so that the threads' accesses do.
template <bool VEC>
__device__ __forceinline__ int column(int j, int e, int t, int G) {
  return VEC ? (j * G + t) * 8 + e : (j * 8 + e) * G + t;
}
template <typename T, bool VEC, int NV>
__device__ __forceinline__ void load_row(const T* p, int cols, int t, int G, float (&v)[8 * NV]) {
  if constexpr (VEC) {
    Raw8<T> raw[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = column<true>(j, 0, t, G);
      if (c < cols) raw[j].load(p + c);
      else raw[j].zero();
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) raw[j].get(v + 8 * j);
  } else {
#pragma unroll
    for (int i = 0; i < 8 * NV; ++i) {
      const int c = column<false>(i / 8, i % 8, t, G);
      v[i] = c < cols ? to_f(p[c]) : 0.f;
    }
  }
}
template <typename T, bool VEC, int NV>
__device__ __forceinline__ void store_row(T* p, int cols, int t, int G, const float (&v)[8 * NV]) {
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if constexpr (VEC) {
      const int c = column<true>(j, 0, t, G);
      if (c < cols) store8(p + c, v + 8 * j);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = column<false>(j, e, t, G);
        if (c < cols) p[c] = from_f<T>(v[8 * j + e]);
      }
    }
  }
}

// The shared exponent of a block of 32 whose largest magnitude has these bits:
// the smallest e in -127 .. 127 with max / 2^e <= 448 = 1.75 * 2^8, as e + 127;
// 255 where the block holds an infinity or NaN.
__device__ __forceinline__ int block_exponent(uint32_t top) {
  if (top >= 0x7f800000u) return 255;
  const int e = int(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);   // biased by 127
  return max(e, 0);
}
__device__ __forceinline__ float up_by(int biased) {   // 2^-(biased - 127)
  return __uint_as_float(uint32_t(254 - min(biased, 253)) << 23);
}
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// The 8-bit form rounds y where its neighbours are 2^-4 apart, and an error of fp32's
// size on the way would now and then round it to the other side (two or three of the
// 33 million elements of 16384 x 2048).  For it y is rounded once, and the joined sum
// of squares and r are held as two numbers, the second what rounding left of the first
// (the products and sums whose rounding is asked for are not to be contracted): 45
// instead of 41 us.  The threads' and warps' own sums stay single, their errors are
// many and of either sign; with them in two numbers it takes 59 us.
struct Two {
  float hi, lo;
  __device__ __forceinline__ void add(float x) {
    const float s = __fadd_rn(hi, x), b = __fsub_rn(s, hi);
    lo += __fsub_rn(hi, __fsub_rn(s, b)) + __fsub_rn(x, b);
    hi = s;
  }
  __device__ __forceinline__ void over_warp() {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      const float h = __shfl_xor_sync(0xffffffffu, hi, o), l = __shfl_xor_sync(0xffffffffu, lo, o);
      lo += l;             // the same in both lanes, as what add() adds is
      add(h);
    }
  }
  __device__ __forceinline__ void over_block(float* box) {
    const float mine = warp_sum(hi + lo);
    if (threadIdx.x % 32 == 0) box[threadIdx.x / 32] = mine;
    __syncthreads();
    hi = box[0];
    lo = 0.f;
    // not unrolled: 48 us
#pragma unroll 1
    for (unsigned w = 1; w < blockDim.x / 32; ++w) add(box[w]);
  }
};
__device__ __forceinline__ float finite_or_zero(float x) { return fabsf(x) < INFINITY ? x : 0.f; }
// (sum / cols + eps)^(-1/2)
__device__ __forceinline__ Two root_of(Two sum, float inv_cols, float inv_rest, float eps) {
  sum.lo = finite_or_zero(sum.lo);       // beside an infinity
  Two m = {__fmul_rn(sum.hi, inv_cols), 0.f};
  m.lo = fmaf(sum.hi, inv_cols, -m.hi) + fmaf(sum.lo, inv_cols, sum.hi * inv_rest);
  m.add(eps);
  const float r = __frsqrt_rn(m.hi), q = __fmul_rn(r, r);
  const float off = fmaf(-m.hi, q, 1.f) - fmaf(m.hi, fmaf(r, r, -q), m.lo * q);
  return {r, finite_or_zero(0.5f * r * off)};
}
// Two products or sums in one instruction.
__device__ __forceinline__ uint64_t pair_of(float a, float b) {
  uint64_t p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(a), "f"(b));
  return p;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t p;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(p) : "l"(a), "l"(b));
  return p;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t p;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(p) : "l"(a), "l"(b), "l"(c));
  return p;
}
// v r w of two elements, rounded once: v r as h + l.  An infinite weight gives NaN.
__device__ __forceinline__ void scale_pair(float* v, const Two& r, const float* w) {
  const uint64_t x = pair_of(v[0], v[1]), m = pair_of(w[0], w[1]), hi = pair_of(r.hi, r.hi);
  const uint64_t h = mul2(x, hi), minus = mul2(x, pair_of(-r.hi, -r.hi));
  const uint64_t l = fma2(x, pair_of(r.lo, r.lo), fma2(x, hi, minus)), y = fma2(h, m, mul2(l, m));
  asm("mov.b64 {%0, %1}, %2;" : "=f"(v[0]), "=f"(v[1]) : "l"(y));
}
__device__ __forceinline__ float scaled(float v, const Two& r, float w) {
  float x[2] = {v, 0.f};
  const float m[2] = {w, 0.f};
  scale_pair(x, r, m);
  return x[0];
}

// y of one row as 8-bit floats.  The 32 columns of a block are four
// neighbouring lanes' chunk (VEC) or one element of each lane of a warp.
template <bool VEC, int NV>
__device__ __forceinline__ void store_eight(const NormParams& p, int row, int t, int G, const float (&v)[8 * NV]) {
  uint8_t* q = p.q + int64_t(row) * p.cols;
  uint8_t* scales = p.scales + int64_t(row) * ((p.cols + 31) / 32);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if constexpr (VEC) {
      const int c = column<true>(j, 0, t, G);
      uint32_t top = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, magnitude(v[8 * j + e]));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int b = block_exponent(top);
      const float up = up_by(b);
      uint32_t w[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float* u = v + 8 * j + 4 * h;
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(u[0] * up, u[1] * up), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(u[2] * up, u[3] * up), __NV_SATFINITE, __NV_E4M3);
        w[h] = lo | hi << 16;
      }
      if (c < p.cols) {
        *reinterpret_cast<uint2*>(q + c) = make_uint2(w[0], w[1]);
        if (t % 4 == 0) scales[c / 32] = uint8_t(b);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = column<false>(j, e, t, G);
        const int b = block_exponent(__reduce_max_sync(0xffffffffu, magnitude(v[8 * j + e])));
        if (c < p.cols) {
          q[c] = __nv_cvt_float_to_fp8(v[8 * j + e] * up_by(b), __NV_SATFINITE, __NV_E4M3);
          if (t % 32 == 0) scales[c / 32] = uint8_t(b);
        }
      }
    }
  }
}

// One row per warp (WARP) or per block; 8 NV elements per thread.
template <typename T, typename W, int NV, bool VEC, bool WARP, int THREADS, bool EIGHT>
__global__ void __launch_bounds__(THREADS) norm_fwd_k(const __grid_constant__ NormParams p) {
  __shared__ float box[32];
  pdl_wait();
  pdl_trigger();
  const int G = WARP ? 32 : int(blockDim.x), t = int(threadIdx.x) % G;
  const int row = WARP ? int(blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32) : int(blockIdx.x);
  if (row >= p.rows) return;        // whole warps or blocks
  float v[8 * NV];
  load_row<T, VEC, NV>(static_cast<const T*>(p.x) + row * p.ldx, p.cols, t, G, v);
  if (p.r) {
    float z[8 * NV];
    load_row<T, VEC, NV>(static_cast<const T*>(p.r) + row * p.ldr, p.cols, t, G, z);
#pragma unroll
    for (int i = 0; i < 8 * NV; ++i) v[i] = to_f(from_f<T>(v[i] + z[i]));
  }
  if (p.s) store_row<T, VEC, NV>(static_cast<T*>(p.s) + row * p.lds, p.cols, t, G, v);
  float w[8 * NV];
  if constexpr (EIGHT) {
    float a[4] = {};
#pragma unroll
    for (int i = 0; i < 8 * NV; ++i) a[i % 4] = fmaf(v[i], v[i], a[i % 4]);
    Two sum = {(a[0] + a[1]) + (a[2] + a[3]), 0.f};
    if (WARP) sum.over_warp();
    else sum.over_block(box);
    const Two r = root_of(sum, p.inv_cols, p.inv_rest, p.eps);
    if (p.rstd && t == 0) p.rstd[row] = r.hi;
    load_row<W, VEC, NV>(static_cast<const W*>(p.w), p.cols, t, G, w);
#pragma unroll
    for (int i = 0; i < 8 * NV; i += 2) scale_pair(v + i, r, w + i);
  } else {
    float a = 0.f;
#pragma unroll
    for (int i = 0; i < 8 * NV; ++i) a = fmaf(v[i], v[i], a);
    a = WARP ? warp_sum(a) : block_sum(a, box);
    const float r = __frsqrt_rn(fmaf(a, p.inv_cols, p.eps));
    if (p.rstd && t == 0) p.rstd[row] = r;
    load_row<W, VEC, NV>(static_cast<const W*>(p.w), p.cols, t, G, w);
#pragma unroll
    for (int i = 0; i < 8 * NV; ++i) v[i] = v[i] * r * w[i];
  }
  if (p.y) store_row<T, VEC, NV>(static_cast<T*>(p.y) + row * p.ldy, p.cols, t, G, v);
  if constexpr (EIGHT) store_eight<VEC, NV>(p, row, t, G, v);
}

// Rows wider than the registers of a block: two passes over each row.
template <typename T, typename W>
__global__ void __launch_bounds__(1024) norm_fwd_wide_k(const __grid_constant__ NormParams p) {
  __shared__ float box[32];
  pdl_wait();
  pdl_trigger();
  const int row = int(blockIdx.x), t = int(threadIdx.x), G = int(blockDim.x);
  const T *x = static_cast<const T*>(p.x) + row * p.ldx, *res = static_cast<const T*>(p.r);
  if (res) res += row * p.ldr;
  T *s = static_cast<T*>(p.s), *y = static_cast<T*>(p.y);
  if (s) s += row * p.lds;
  if (y) y += row * p.ldy;
  Two sum = {};
  for (int c = t; c < p.cols; c += G) {
    float v = to_f(x[c]);
    if (res) v = to_f(from_f<T>(v + to_f(res[c])));
    if (s) s[c] = from_f<T>(v);
    sum.add(v * v);
  }
  sum.over_block(box);
  const Two r = root_of(sum, p.inv_cols, p.inv_rest, p.eps);
  if (p.rstd && t == 0) p.rstd[row] = r.hi;
  const T* from = s ? s : x;        // each thread reads what it wrote
  const int blocks = (p.cols + 31) / 32;
  for (int c = t; c < 32 * blocks; c += G) {     // whole warps
    float v = 0.f;
    if (c < p.cols) {
      const float z = to_f(from[c]), w = to_f(static_cast<const W*>(p.w)[c]);
      v = p.q ? scaled(z, r, w) : z * r.hi * w;       // an infinite weight stays one where y alone is wanted
    }
    if (y && c < p.cols) y[c] = from_f<T>(v);
    if (p.q) {
      const int b = block_exponent(__reduce_max_sync(0xffffffffu, magnitude(v)));
      if (c < p.cols) {
        p.q[int64_t(row) * p.cols + c] = __nv_cvt_float_to_fp8(v * up_by(b), __NV_SATFINITE, __NV_E4M3);
        if (c % 32 == 0) p.scales[int64_t(row) * blocks + c / 32] = uint8_t(b);
      }
    }
  }
}

// Rows on their way into shared memory: each thread copies what it will read
// itself, so its own copies are all it waits for.  STAGES rows are in flight.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
template <typename T, int NV>
struct RowRing {
  static constexpr int kPlanes = 3 * NV * int(sizeof(T)) / 2;      // 16 bytes of each thread: dy, s, ds
  uint32_t at, stage;                  // this thread's first plane; bytes of a stage
  __device__ __forceinline__ RowRing(const void* smem, int threads)
      : at(uint32_t(__cvta_generic_to_shared(smem)) + threadIdx.x * 16), stage(kPlanes * threads * 16) {}
  // Tensor `which` of a row into stage n.
  __device__ __forceinline__ void copy(int n, int which, const T* row, int cols, int t, int G, int threads) const {
    constexpr int kParts = int(sizeof(T)) / 2;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = column<true>(j, 0, t, G);
      if (c < cols)
#pragma unroll
        for (int h = 0; h < kParts; ++h)
          copy16(at + n * stage + ((which * NV + j) * kParts + h) * threads * 16, reinterpret_cast<const char*>(row + c) + 16 * h);
    }
  }
  __device__ __forceinline__ void get(int n, int which, int cols, int t, int G, int threads, float (&v)[8 * NV]) const {
    constexpr int kParts = int(sizeof(T)) / 2;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      uint4 w[kParts];
#pragma unroll
      for (int h = 0; h < kParts; ++h) {
        w[h] = make_uint4(0u, 0u, 0u, 0u);
        if (column<true>(j, 0, t, G) < cols)
          asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                       : "=r"(w[h].x), "=r"(w[h].y), "=r"(w[h].z), "=r"(w[h].w)
                       : "r"(at + n * stage + ((which * NV + j) * kParts + h) * threads * 16)
                       : "memory");
      }
      if constexpr (kParts == 1) {
        unpack8(w[0], v + 8 * j);
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          v[8 * j + 4 * h] = __uint_as_float(w[h].x);
          v[8 * j + 4 * h + 1] = __uint_as_float(w[h].y);
          v[8 * j + 4 * h + 2] = __uint_as_float(w[h].z);
          v[8 * j + 4 * h + 3] = __uint_as_float(w[h].w);
        }
      }
    }
  }
};

// Each warp or block takes neighbouring rows and holds its part of dw until the
// end.  With 16-byte rows (VEC) the next STAGES - 1 rows are being copied while
// one is worked on: a row's sum stands between its loads and its stores, and
// without them a block waits for memory once per row (32768 x 4096 bf16: 345 us
// without, 208 with them, 161 with neighbouring rows: 6.7 TB/s).
template <typename T, typename W, int NV, bool VEC, bool WARP, int THREADS, int STAGES>
__global__ void __launch_bounds__(THREADS) norm_bwd_k(const __grid_constant__ NormGradParams p) {
  extern __shared__ __align__(16) char smem[];         // rows in flight; WARP, at the end: dw of [warps][cols]
  __shared__ float box[2][32];
  pdl_wait();
  pdl_trigger();
  const int G = WARP ? 32 : int(blockDim.x), t = int(threadIdx.x) % G;
  const int warp = int(threadIdx.x) / 32, per = WARP ? int(blockDim.x) / 32 : 1;
  // neighbouring rows: blocks that took every n-th one read 5.2 TB/s instead of 6.7
  const int64_t groups = int64_t(gridDim.x) * per, share = (p.rows + groups - 1) / groups;
  const int64_t first = (int64_t(blockIdx.x) * per + (WARP ? warp : 0)) * share, end = min(int64_t(p.rows), first + share);
  const T *dy = static_cast<const T*>(p.dy), *sum = static_cast<const T*>(p.s), *ds = static_cast<const T*>(p.ds);
  const RowRing<T, NV> ring(smem, THREADS);
  auto fetch = [&](int64_t row, int n) {
    if (row < end) {
      ring.copy(n, 0, dy + row * p.lddy, p.cols, t, G, THREADS);
      ring.copy(n, 1, sum + row * p.lds, p.cols, t, G, THREADS);
      if (ds) ring.copy(n, 2, ds + row * p.ldds, p.cols, t, G, THREADS);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  if constexpr (VEC)
#pragma unroll
    for (int n = 0; n < STAGES - 1; ++n) fetch(first + n, n);
  float w[8 * NV], dw[8 * NV];
  load_row<W, VEC, NV>(static_cast<const W*>(p.w), p.cols, t, G, w);
#pragma unroll
  for (int i = 0; i < 8 * NV; ++i) dw[i] = 0.f;
  int turn = 0, n = 0;
  for (int64_t row = first; row < end; ++row) {
    float g[8 * NV], s[8 * NV], d[8 * NV];
    const float r = p.rstd[row];
    if constexpr (VEC) {
      fetch(row + (STAGES - 1), n == 0 ? STAGES - 1 : n - 1);
      asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
      ring.get(n, 0, p.cols, t, G, THREADS, g);
      ring.get(n, 1, p.cols, t, G, THREADS, s);
    } else {
      load_row<T, VEC, NV>(dy + row * p.lddy, p.cols, t, G, g);
      load_row<T, VEC, NV>(sum + row * p.lds, p.cols, t, G, s);
      if (ds) load_row<T, VEC, NV>(ds + row * p.ldds, p.cols, t, G, d);
    }
    float a = 0.f;
#pragma unroll
    for (int i = 0; i < 8 * NV; ++i) {
      s[i] *= r;
      dw[i] = fmaf(g[i], s[i], dw[i]);
      g[i] *= w[i];
      a = fmaf(g[i], s[i], a);
    }
    a = WARP ? warp_sum(a) : block_sum(a, box[turn]);
    turn ^= 1;
    const float k = -a * p.inv_cols;
    if (VEC && ds) ring.get(n, 2, p.cols, t, G, THREADS, d);
#pragma unroll
    for (int i = 0; i < 8 * NV; ++i) {
      g[i] = fmaf(s[i], k, g[i]);
      g[i] = ds ? fmaf(g[i], r, d[i]) : g[i] * r;
    }
    store_row<T, VEC, NV>(static_cast<T*>(p.dx) + row * p.lddx, p.cols, t, G, g);
    n = n + 1 == STAGES ? 0 : n + 1;
  }
  float* out = p.part + int64_t(blockIdx.x) * p.cols;
  if constexpr (!WARP) {
    store_row<float, VEC, NV>(out, p.cols, t, G, dw);
  } else {
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
    float* dw_box = reinterpret_cast<float*>(smem);
    store_row<float, VEC, NV>(dw_box + warp * p.cols, p.cols, t, G, dw);
    __syncthreads();
    for (int c = threadIdx.x; c < p.cols; c += blockDim.x) {
      float a = 0.f;
      for (int n = 0; n < per; ++n) a += dw_box[n * p.cols + c];
      out[c] = a;
    }
  }
}
template <typename T, typename W>
__global__ void __launch_bounds__(1024) norm_bwd_wide_k(const __grid_constant__ NormGradParams p) {
  __shared__ float box[2][32];
  pdl_wait();
  pdl_trigger();
  const int t = int(threadIdx.x), G = int(blockDim.x);
  const W* w = static_cast<const W*>(p.w);
  float* out = p.part + int64_t(blockIdx.x) * p.cols;
  for (int c = t; c < p.cols; c += G) out[c] = 0.f;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const T *dy = static_cast<const T*>(p.dy) + row * p.lddy, *s = static_cast<const T*>(p.s) + row * p.lds;
    const T* ds = p.ds ? static_cast<const T*>(p.ds) + row * p.ldds : nullptr;
    T* dx = static_cast<T*>(p.dx) + row * p.lddx;
    const float r = p.rstd[row];
    float a = 0.f;
    for (int c = t; c < p.cols; c += G) {
      const float g = to_f(dy[c]), z = to_f(s[c]) * r;
      out[c] = fmaf(g, z, out[c]);
      a = fmaf(g * to_f(w[c]), z, a);
    }
    const float k = -block_sum(a, box[turn]) * p.inv_cols;
    turn ^= 1;
    for (int c = t; c < p.cols; c += G) {
      const float g = fmaf(to_f(s[c]) * r, k, to_f(dy[c]) * to_f(w[c]));
      dx[c] = from_f<T>(ds ? fmaf(g, r, to_f(ds[c])) : g * r);
    }
  }
}
// dw: 32 columns per block, whose 32 warps' sums of the parts are added in order.
template <typename W>
__global__ void __launch_bounds__(1024) norm_dw_k(const float* part, W* dw, int parts, int cols) {
  __shared__ float box[32][33];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x % 32, n = int(threadIdx.x) / 32, c = int(blockIdx.x) * 32 + lane;
  float a = 0.f;
  if (c < cols)
#pragma unroll 8
    for (int i = n; i < parts; i += 32) a += part[int64_t(i) * cols + c];
  box[n][lane] = a;
  __syncthreads();
  // warp n takes column n of the block
  a = warp_sum(box[lane][n]);
  if (lane == 0 && int(blockIdx.x) * 32 + n < cols) dw[blockIdx.x * 32 + n] = from_f<W>(a);
}

// 2^(scale - 127); a NaN for 255.
__device__ __forceinline__ float scale_of(int b) {
  // 2^-127 is half of the smallest normal number
  return b == 255 ? __uint_as_float(0x7fc00000u) : b == 0 ? __uint_as_float(0x400000u) : __uint_as_float(uint32_t(b) << 23);
}
__device__ __forceinline__ float2 decode_pair(uint32_t two, float up) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(__nv_fp8x2_storage_t(two), __NV_E4M3);     // exact
  const float2 f = __half22float2(__half2(h));
  return make_float2(f.x * up, f.y * up);
}

// The scale times the 8-bit floats.  A thread's U vectors of eight are loaded
// before the first is used (16384 x 2048: 20.5 us with one, 5.0 TB/s).
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) decode_k(const uint8_t* q, const uint8_t* scales, T* y, int64_t ldy, int64_t items,
                                                int cols) {
  pdl_wait();
  pdl_trigger();
  constexpr int U = VEC ? 4 : 1;
  const int per = VEC ? cols / 8 : cols, blocks = (cols + 31) / 32;
  const int64_t step = int64_t(gridDim.x) * blockDim.x;
  for (int64_t i0 = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; i0 < items; i0 += U * step) {
    if constexpr (VEC) {
      uint2 w[U];
      int b[U];
      T* to[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t i = i0 + u * step;
        to[u] = nullptr;
        if (i >= items) continue;
        const int64_t row = i / per;
        const int c = int(i - row * per) * 8;
        w[u] = *reinterpret_cast<const uint2*>(q + row * cols + c);
        b[u] = scales[row * blocks + c / 32];
        to[u] = y + row * ldy + c;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (!to[u]) continue;
        const float up = scale_of(b[u]);
        float v[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 f = decode_pair((e < 2 ? w[u].x : w[u].y) >> (16 * (e % 2)) & 0xffffu, up);
          v[2 * e] = f.x;
          v[2 * e + 1] = f.y;
        }
        store8(to[u], v);
      }
    } else {
      const int64_t row = i0 / per;
      const int c = int(i0 - row * per);
      y[row * ldy + c] = from_f<T>(decode_pair(q[row * cols + c], scale_of(scales[row * blocks + c / 32])).x);
    }
  }
}

// Threads of a row: a warp up to 1024 columns, above a block with up to 16
// elements per thread.
struct RowShape {
  bool warp;
  int threads;
};
RowShape row_shape(int cols) {
  if (cols <= 1024) return {true, 256};
  if (cols <= 16384) return {false, (cols + 16 * 32 - 1) / (16 * 32) * 32};
  return {false, 1024};
}
// Blocks of a gradient: two per SM, or one whose rows in flight fill its shared
// memory (fewer where there are fewer rows).  fp32 rows of 513 to 1024 columns fill
// it too, and their 304 blocks take two turns.
int grad_blocks(int64_t rows, int cols) {
  const RowShape a = row_shape(cols);
  const int64_t per = a.warp ? a.threads / 32 : 1, want = (rows + per - 1) / per;
  const int most = cols <= 4096 ? 2 * 152 : 152;
  return want < most ? int(want) : most;
}

template <typename T, typename W, bool VEC, bool EIGHT>
cudaError_t forward_rows(const NormParams& p, cudaStream_t st) {
  const RowShape a = row_shape(p.cols);
  const int per = a.warp ? a.threads / 32 : 1;
  const dim3 grid(unsigned((int64_t(p.rows) + per - 1) / per)), block(unsigned(a.threads));
  auto k = p.cols <= 256     ? norm_fwd_k<T, W, 1, VEC, true, 256, EIGHT>
           : p.cols <= 512   ? norm_fwd_k<T, W, 2, VEC, true, 256, EIGHT>
           : p.cols <= 1024  ? norm_fwd_k<T, W, 4, VEC, true, 256, EIGHT>
           : p.cols <= 4096  ? norm_fwd_k<T, W, 2, VEC, false, 256, EIGHT>
           : p.cols <= 8192  ? norm_fwd_k<T, W, 2, VEC, false, 512, EIGHT>
           : p.cols <= 16384 ? norm_fwd_k<T, W, 2, VEC, false, 1024, EIGHT>
                             : norm_fwd_wide_k<T, W>;
  return launch_k(k, grid, block, 0, st, p);
}
template <typename T, typename W, bool VEC>
cudaError_t forward(const NormParams& p, cudaStream_t st) {
  return p.q ? forward_rows<T, W, VEC, true>(p, st) : forward_rows<T, W, VEC, false>(p, st);
}
// The gradient's kernel, launched with its shared memory.
template <typename T, typename W, int NV, bool VEC, bool WARP, int THREADS, int STAGES>
cudaError_t backward_rows(const NormGradParams& p, int blocks, cudaStream_t st) {
  auto k = norm_bwd_k<T, W, NV, VEC, WARP, THREADS, STAGES>;
  const size_t ring = VEC ? size_t(STAGES) * RowRing<T, NV>::kPlanes * THREADS * 16 : 0;
  const size_t box = WARP ? size_t(THREADS / 32) * p.cols * sizeof(float) : 0, smem = ring > box ? ring : box;
  static std::atomic<bool> allowed[kMaxDevices];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && smem > 47 * 1024 && !(dev < kMaxDevices && allowed[dev])) {
    e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem));
    if (e == cudaSuccess && dev < kMaxDevices) allowed[dev] = true;
  }
  if (e != cudaSuccess) return e;
  return launch_k(k, dim3(unsigned(blocks)), dim3(THREADS), smem, st, p);
}
template <typename T, typename W, bool VEC>
cudaError_t backward(const NormGradParams& p, void* dw, cudaStream_t st) {
  const int blocks = grad_blocks(p.rows, p.cols);
  constexpr int K = sizeof(T) == 2 ? 4 : 2;       // rows in flight: 96 KB per block of 256 threads
  cudaError_t e;
  if (p.cols <= 256) e = backward_rows<T, W, 1, VEC, true, 256, K>(p, blocks, st);
  else if (p.cols <= 512) e = backward_rows<T, W, 2, VEC, true, 256, K>(p, blocks, st);
  else if (p.cols <= 1024) e = backward_rows<T, W, 4, VEC, true, 256, 2>(p, blocks, st);
  else if (p.cols <= 4096) e = backward_rows<T, W, 2, VEC, false, 256, K>(p, blocks, st);
  else if (p.cols <= 8192) e = backward_rows<T, W, 2, VEC, false, 512, K>(p, blocks, st);
  else if (p.cols <= 16384) e = backward_rows<T, W, 2, VEC, false, 1024, K / 2>(p, blocks, st);
  else e = launch_k(norm_bwd_wide_k<T, W>, dim3(unsigned(blocks)), dim3(1024), 0, st, p);
  if (e != cudaSuccess) return e;
  return launch_k(norm_dw_k<W>, dim3(unsigned((p.cols + 31) / 32)), dim3(1024), 0, st, (const float*)p.part,
                  static_cast<W*>(dw), blocks, p.cols);
}

int bad(const char* why) { return report_error(FO_ERR_ARG, std::string("norm: ") + why); }
int done(cudaError_t e) { return e == cudaSuccess ? FO_OK : report_error(FO_ERR_CUDA, cudaGetErrorString(e)); }

int check_sizes(int dtype, int64_t rows, int64_t cols) {
  if (dtype != FO_DTYPE_F32 && dtype != FO_DTYPE_BF16) return bad("unknown dtype");
  if (rows < 0 || rows >= int64_t(1) << 31 || cols < 1 || cols > int64_t(1) << 20)
    return bad("rows below 2^31 and 1 to 2^20 columns");
  return FO_OK;
}
// A tensor that is there: its address, and its row stride where it matters.
int check_rows(const void* t, int64_t stride, int dtype, int64_t rows, int64_t cols, bool output, const char* name) {
  const size_t size = dtype == FO_DTYPE_F32 ? 4 : 2;
  if (!t || reinterpret_cast<uintptr_t>(t) % size) return bad((std::string(name) + " is null or misaligned").c_str());
  if (rows > 1 && (stride < (output ? cols : 0) || stride > INT64_MAX / 8 / rows))
    return bad((std::string("bad row stride of ") + name).c_str());
  return FO_OK;
}
bool wide_rows(const void* t, int64_t stride, int dtype, int64_t rows) {
  return aligned16(t) && (rows <= 1 || stride % (dtype == FO_DTYPE_F32 ? 4 : 8) == 0);
}

}  // namespace
}  // namespace fo

using namespace fo;

extern "C" {

int fo_rms_norm(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, const void* weight,
                int weight_dtype, void* sum, int64_t sum_stride, void* y, int64_t y_stride, uint8_t* q, uint8_t* scales,
                float* rstd, int dtype, int64_t rows, int64_t cols, double eps, void* stream) {
  int rc = check_sizes(dtype, rows, cols);
  if (rc) return rc;
  if (weight_dtype != FO_DTYPE_F32 && weight_dtype != dtype) return bad("the weight is fp32 or of the tensors' type");
  if (!(eps >= 0.0 && eps <= 1e30)) return bad("eps out of range");
  if (rows == 0) return FO_OK;
  if (!y && !q) return bad("neither y nor q is wanted");
  if (!q != !scales) return bad("q and scales go together");
  if ((rc = check_rows(x, x_stride, dtype, rows, cols, false, "x")) ||
      (residual && (rc = check_rows(residual, residual_stride, dtype, rows, cols, false, "residual"))) ||
      (rc = check_rows(weight, 0, weight_dtype, 1, cols, false, "weight")) ||
      (sum && (rc = check_rows(sum, sum_stride, dtype, rows, cols, true, "sum"))) ||
      (y && (rc = check_rows(y, y_stride, dtype, rows, cols, true, "y"))))
    return rc;
  if (reinterpret_cast<uintptr_t>(rstd) % 4) return bad("rstd is misaligned");
  if (y && y == sum) return bad("y and sum are one tensor");
  if (residual && !sum) return bad("a residual's addition has a sum to write");
  NormParams p;
  p.x = x;
  p.r = residual;
  p.w = weight;
  p.s = sum;
  p.y = y;
  p.q = q;
  p.scales = scales;
  p.rstd = rstd;
  p.ldx = x_stride;
  p.ldr = residual_stride;
  p.lds = sum_stride;
  p.ldy = y_stride;
  p.rows = int(rows);
  p.cols = int(cols);
  p.eps = float(eps);
  p.inv_cols = float(1.0 / double(cols));
  p.inv_rest = float(1.0 / double(cols) - double(p.inv_cols));
  const bool vec = cols % 8 == 0 && wide_rows(x, x_stride, dtype, rows) && aligned16(weight) &&
                   (!residual || wide_rows(residual, residual_stride, dtype, rows)) &&
                   (!sum || wide_rows(sum, sum_stride, dtype, rows)) && (!y || wide_rows(y, y_stride, dtype, rows)) &&
                   reinterpret_cast<uintptr_t>(q) % 8 == 0;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == FO_DTYPE_F32) return done(vec ? forward<float, float, true>(p, st) : forward<float, float, false>(p, st));
  if (weight_dtype == FO_DTYPE_F32) return done(vec ? forward<bf16, float, true>(p, st) : forward<bf16, float, false>(p, st));
  return done(vec ? forward<bf16, bf16, true>(p, st) : forward<bf16, bf16, false>(p, st));
}

int64_t fo_rms_norm_workspace(int64_t rows, int64_t cols) {
  if (check_sizes(FO_DTYPE_F32, rows, cols)) return -1;
  return rows == 0 ? 0 : int64_t(grad_blocks(rows, int(cols))) * cols * 4;
}

int fo_rms_norm_grad(const void* dy, int64_t dy_stride, const void* ds, int64_t ds_stride, const void* s, int64_t s_stride,
                     const void* weight, int weight_dtype, const float* rstd, void* dx, int64_t dx_stride, void* dweight,
                     int dtype, int64_t rows, int64_t cols, void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check_sizes(dtype, rows, cols);
  if (rc) return rc;
  if (weight_dtype != FO_DTYPE_F32 && weight_dtype != dtype) return bad("the weight is fp32 or of the tensors' type");
  const size_t wsize = weight_dtype == FO_DTYPE_F32 ? 4 : 2;
  if (!dweight || reinterpret_cast<uintptr_t>(dweight) % wsize) return bad("dweight is null or misaligned");
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (rows == 0) return done(cudaMemsetAsync(dweight, 0, size_t(cols) * wsize, st));
  if ((rc = check_rows(dy, dy_stride, dtype, rows, cols, false, "dy")) ||
      (ds && (rc = check_rows(ds, ds_stride, dtype, rows, cols, false, "ds"))) ||
      (rc = check_rows(s, s_stride, dtype, rows, cols, false, "s")) ||
      (rc = check_rows(weight, 0, weight_dtype, 1, cols, false, "weight")) ||
      (rc = check_rows(dx, dx_stride, dtype, rows, cols, true, "dx")))
    return rc;
  if (!rstd || reinterpret_cast<uintptr_t>(rstd) % 4) return bad("rstd is null or misaligned");
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 || workspace_bytes < fo_rms_norm_workspace(rows, cols))
    return bad("the workspace is missing, misaligned or too small");
  NormGradParams p;
  p.dy = dy;
  p.ds = ds;
  p.s = s;
  p.w = weight;
  p.rstd = rstd;
  p.dx = dx;
  p.part = static_cast<float*>(workspace);
  p.lddy = dy_stride;
  p.ldds = ds_stride;
  p.lds = s_stride;
  p.lddx = dx_stride;
  p.rows = int(rows);
  p.cols = int(cols);
  p.inv_cols = float(1.0 / double(cols));
  const bool vec = cols % 8 == 0 && wide_rows(dy, dy_stride, dtype, rows) && wide_rows(s, s_stride, dtype, rows) &&
                   wide_rows(dx, dx_stride, dtype, rows) && aligned16(weight) && (!ds || wide_rows(ds, ds_stride, dtype, rows));
  if (dtype == FO_DTYPE_F32) return done(vec ? backward<float, float, true>(p, dweight, st) : backward<float, float, false>(p, dweight, st));
  if (weight_dtype == FO_DTYPE_F32) return done(vec ? backward<bf16, float, true>(p, dweight, st) : backward<bf16, float, false>(p, dweight, st));
  return done(vec ? backward<bf16, bf16, true>(p, dweight, st) : backward<bf16, bf16, false>(p, dweight, st));
}

int fo_decode_8bit(const uint8_t* q, const uint8_t* scales, void* y, int64_t y_stride, int dtype, int64_t rows, int64_t cols,
                   void* stream) {
  int rc = check_sizes(dtype, rows, cols);
  if (rc || rows == 0) return rc;
  if (!q || !scales) return bad("q or scales is null");
  if ((rc = check_rows(y, y_stride, dtype, rows, cols, true, "y"))) return rc;
  const bool vec = cols % 8 == 0 && reinterpret_cast<uintptr_t>(q) % 8 == 0 && wide_rows(y, y_stride, dtype, rows);
  const int64_t items = rows * (vec ? cols / 8 : cols);
  const dim3 grid(unsigned(elementwise_blocks(items, 256)));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == FO_DTYPE_F32)
    return done(launch_k(vec ? decode_k<float, true> : decode_k<float, false>, grid, dim3(256), 0, st, q, scales,
                         static_cast<float*>(y), y_stride, items, int(cols)));
  return done(launch_k(vec ? decode_k<bf16, true> : decode_k<bf16, false>, grid, dim3(256), 0, st, q, scales,
                       static_cast<bf16*>(y), y_stride, items, int(cols)));
}

}  // extern "C"
