// Pieces shared by the tensor-core kernels of scored attention
// (k_scored_fwd.cu, k_scored_bwd.cu): bounded waits, the list of blocks a tile
// walks, tensor maps and fast exponentials.
#pragma once
#include "fo_common.cuh"
#include "fo_ptx.cuh"
#include "fo_scored.h"
#include "fo_tc.h"

#include <cuda_fp16.h>

namespace fo {
namespace {

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Pairs of fp32 in one instruction (two independent roundings).
struct F2 {
  uint64_t v;
};
__device__ __forceinline__ F2 f2(float a, float b) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ F2 f2u(uint32_t a, uint32_t b) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ void split(F2 p, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p.v));
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
// Two pairs from shared memory (16-byte aligned).
__device__ __forceinline__ void ld_pairs(uint32_t addr, F2& a, F2& b) {
  asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(a.v), "=l"(b.v) : "r"(addr) : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// x <- x + y for two neighbours of a register array of fp32 bits.
__device__ __forceinline__ void add_to(uint32_t& a, uint32_t& b, F2 y) {
  float u, v;
  split(add2(f2u(a, b), y), u, v);
  a = __float_as_uint(u);
  b = __float_as_uint(v);
}
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// tcgen05.mma and its commit, issued by one elected lane of a converged warp:
// both operands in shared memory, or A in tensor memory (lane = row, each
// 32-bit column two consecutive K elements, so 16 elements of K are 8
// columns).  elect.sync stands beside each product, which tells the compiler
// that one lane issues: from a branch on the lane index every product took 170
// cycles whatever its size, and under a predicate computed once 90.
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.b32 p, %4, 0;\n elect.sync _|q, 0xffffffff;\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(acc)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.b32 p, %4, 0;\n elect.sync _|q, 0xffffffff;\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(acc)
      : "memory");
}
__device__ __forceinline__ void commit_to(uint64_t* bar) {
  asm volatile(
      "{\n .reg .pred q;\n elect.sync _|q, 0xffffffff;\n"
      " @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(smem_u32(bar))
      : "memory");
}

// A K- or MN-major operand descriptor whose high word is a constant, so that
// moving it by `off` bytes within shared memory is a 32-bit addition.
// (In a cluster the upper bits of a shared-memory address hold the block's
// rank, which is no part of a descriptor.)
template <uint32_t LBO>
struct Operand {
  uint32_t lo;
  __device__ __forceinline__ explicit Operand(uint32_t addr) : lo((addr & 0x3ffff) >> 4 | (LBO >> 4) << 16) {}
  __device__ __forceinline__ uint64_t at(uint32_t off) const {
    constexpr uint32_t hi = (1024u >> 4) | (1u << 14) | (2u << 29);      // stride 1024, version 1, 128-byte swizzle
    return uint64_t(lo + (off >> 4)) | uint64_t(hi) << 32;
  }
};

// What a kernel's waits that gave up leave on a device: the last one's code and
// how many threads did.  The count only grows: each host thread holds what it
// has been told of.
struct GaveUp {
  int code;
  unsigned count;
};
// The code of a wait that gave up since this thread last asked (`told`), or 0.
template <typename Symbol>
cudaError_t gave_up_since(const Symbol& symbol, unsigned* told, int* code) {
  GaveUp now;
  const cudaError_t e = cudaMemcpyFromSymbol(&now, symbol, sizeof(now));
  *code = 0;
  if (e != cudaSuccess || now.count == *told) return e;
  *told = now.count;
  *code = now.code;
  return e;
}

// A role's waits: after one has given up (about two seconds) the rest return
// at once, so the kernel ends soon and says so in `err`.
struct Waits {
  GaveUp* err;
  uint64_t limit;
  bool dead = false;
  __device__ __forceinline__ explicit Waits(GaveUp* e, uint64_t ns = kWaitLimit) : err(e), limit(ns) {}
  __device__ __forceinline__ void give_up(int code) {
    atomicExch(&err->code, code);
    atomicAdd(&err->count, 1u);
    dead = true;
  }
  __device__ __forceinline__ void on(uint64_t* bar, uint32_t parity, int code) {
    if (dead || mbar_wait(bar, parity, limit)) return;
    give_up(code);
  }
  // The same for the lanes of a warp of arithmetic, converged afterwards.
  __device__ __forceinline__ void on_lanes(uint64_t* bar, uint32_t parity, int code) {
    on(bar, parity, code);
    __syncwarp();
  }
  // The same for a whole converged warp, whose lanes agree on the outcome.
  __device__ __forceinline__ void on_warp(uint64_t* bar, uint32_t parity, int code) {
    if (dead || __all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return;
    const uint64_t t0 = global_ns();
    while (true) {
      for (int i = 0; i < 64; ++i)
        if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return;
      if (__any_sync(0xffffffffu, global_ns() - t0 > limit)) break;
    }
    give_up(code);
  }
};

// One arrival for a warp whose lanes have all written what it announces.
__device__ __forceinline__ void arrive_warp(uint64_t* bar) {
  __syncwarp();
  if (threadIdx.x % 32 == 0) mbar_arrive(bar);
}

// Walks the blocks set in either of two bitmaps in shared memory, in ascending
// order; on[k] tells whether map k has the current one.
struct Bits {
  const uint32_t *a, *b;
  int words, w;
  uint32_t wa, wb, left;
  bool on[2];
  __device__ __forceinline__ Bits(const uint32_t* a_, const uint32_t* b_, int words_)
      : a(a_), b(b_), words(words_), w(0), wa(a_[0]), wb(b_[0]), left(wa | wb) {}
  // The next block, or -1.
  __device__ __forceinline__ int next() {
    while (!left) {
      if (++w >= words) return -1;
      wa = a[w];
      wb = b[w];
      left = wa | wb;
    }
    const int bit = __ffs(int(left)) - 1;
    left &= left - 1;
    on[0] = (wa >> bit) & 1u;
    on[1] = (wb >> bit) & 1u;
    return 32 * w + bit;
  }
};
// The same for one bitmap, with few registers for the warps of arithmetic.
struct BitList {
  uint32_t map;             // shared-memory address
  int words, w;
  uint32_t left;
  __device__ __forceinline__ static uint32_t word(uint32_t map, int w) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(map + 4 * w));
    return v;
  }
  __device__ __forceinline__ BitList(const uint32_t* m, int words_) : map(smem_u32(m)), words(words_), w(0) {
    left = word(map, 0);
  }
  __device__ __forceinline__ int next() {
    while (!left) {
      if (++w >= words) return -1;
      left = word(map, w);
    }
    const int bit = __ffs(int(left)) - 1;
    left &= left - 1;
    return 32 * w + bit;
  }
};
__device__ __forceinline__ bool bit_of(const uint32_t* map, int i) { return (map[i >> 5] >> (i & 31)) & 1u; }
__device__ __forceinline__ bool any_bit(const uint32_t* map, int words) {
  uint32_t o = 0;
  for (int w = 0; w < words; ++w) o |= map[w];
  return o != 0;
}

// A position in a ring of N stages that moves S at a time, and the parity of
// its barrier's phase.
template <int N, int S = 1>
struct Ring {
  int at, phase;
  __device__ __forceinline__ explicit Ring(int first = 0) : at(first), phase(0) {}
  __device__ __forceinline__ void step() {
    at += S;
    if (at >= N) at -= N, phase ^= 1;
  }
};

// Bias kinds and caps, compile-time in the kernels.
enum { kBiasNone = 0, kBiasSlope = 1, kBiasTable = 2 };
enum { kCapNone = 0, kCapPlain = 1, kCapLarge = 2 };

// The table's biases by distance, extended by kExt on both sides with the
// outermost values: a patch of up to 32 x 64 scores that is not entirely
// beyond the reach then reads it directly.
constexpr int kExt = 96;
constexpr int kBiasFloats = 2 * kMaxReach + 2 * kExt + 4;
__device__ __forceinline__ void load_bias(float* bias, const ScoredParams& p, int h, float inv_unit, int tid, int n) {
  const bf16* t = static_cast<const bf16*>(p.table) + int64_t(h) * p.buckets;
  for (int e = tid; e < 2 * p.reach + 1 + 2 * kExt; e += n)
    bias[e] = bias_of(__bfloat162float(t[p.map[min(max(e - kExt, 0), 2 * p.reach)]])) * inv_unit;
}

// N scores (fp32 bits) of one query row, keys j0 .. j0 + N - 1 -> score units:
// the cap (KEEP: ch receives kChainUp times its derivative 1 - tanh^2 as pairs
// of fp16, a factor of a product that is itself rounded to bf16; times kChainUp
// it keeps its 11 bits down to 2e-9, the derivative at ten times the cap) and
// the bias.
// DIR is +1 when the columns are keys and -1 when they are queries (the row
// then is the key); d = distance of column 0, lo and hi the bounds of the
// warp's distances.
// Two forms of tanh y: 1 - 2 q with q = 1 / (1 + e^2y), whose derivative is
// 4 q (1 - q), and up to |y| = kSeriesEnd the Taylor series to y^11 (the next
// term is below 6e-8 of the sum there).  The first has an absolute error of
// about 1.7e-7 (q to 2 units in the last place), so a score is off by 1.7e-7
// of the cap however small it is: up to caps of kPlainCap 1.1e-5, which P's
// rounding to bf16 hides 300 times over.  Above it (kCapLarge) each score takes
// the form that is exact for it, the same one forward and backward; as a branch
// at run time instead of a kernel of its own it cost the backward pass of 4 x
// 2048 tokens, 16 heads of 128 on 4, 6% (274 -> 292 us) at a cap of 50.
// In the forward pass a warp whose patch has only |y| up to kSeriesEnd, as
// scores well below the cap have, takes the series alone, which needs no
// special-function operation against two per score: scoring 2 x 4095 tokens,
// 16 heads of 128, with a prefix took 203 us against 223.  The backward pass,
// whose special-function unit is less busy, ran 3% slower with it.
constexpr float kSeriesEnd = 0.4f, kPlainCap = 64.f, kChainUp = 32768.f;
struct Shape {
  float cap, cap_in, y_in;      // the cap; scale to 2 y log2(e) and to y
  float slope;                  // negated, in score units
  const float* bias;
  int reach;
};
__device__ __forceinline__ F2 tanh_series(F2 y) {
  const F2 z = mul2(y, y);
  F2 t = fma2(z, f2(-1382.f / 155925.f, -1382.f / 155925.f), f2(62.f / 2835.f, 62.f / 2835.f));
  t = fma2(z, t, f2(-17.f / 315.f, -17.f / 315.f));
  t = fma2(z, t, f2(2.f / 15.f, 2.f / 15.f));
  t = fma2(z, t, f2(-1.f / 3.f, -1.f / 3.f));
  return fma2(mul2(z, t), y, y);
}
template <int N, int BIAS, int CAP, int DIR, bool KEEP>
__device__ __forceinline__ void shape_scores(uint32_t (&r)[N], uint32_t* ch, const Shape& a, int d, int lo, int hi) {
  if (CAP) {
    const F2 one = f2(1.f, 1.f), cap = f2(a.cap, a.cap), in = f2(a.cap_in, a.cap_in), y_in = f2(a.y_in, a.y_in),
             two = f2(-2.f * a.cap, -2.f * a.cap);
    // scores e and e + 1 by the exponential; the second form (and ch)
    auto by_exponential = [&](int e, float& u, float& v) {
      float x, y;
      split(mul2(f2u(r[e], r[e + 1]), in), x, y);
      split(add2(f2(ex2(x), ex2(y)), one), x, y);
      const F2 q = f2(rcp(x), rcp(y));
      if (KEEP) {
        split(mul2(mul2(f2(4.f * kChainUp, 4.f * kChainUp), q), fma2(q, f2(-1.f, -1.f), one)), x, y);
        const __half2 h = __floats2half2_rn(x, y);
        ch[e / 2] = *reinterpret_cast<const uint32_t*>(&h);
      }
      split(fma2(two, q, cap), u, v);
    };
    bool small = false;
    if (!KEEP) {
      float top = 0.f;
#pragma unroll
      for (int e = 0; e < N; e += 2) top = max3(top, fabsf(__uint_as_float(r[e])), fabsf(__uint_as_float(r[e + 1])));
      small = __all_sync(0xffffffffu, top * a.y_in <= kSeriesEnd);
    }
    if (small) {
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        float u, v;
        split(mul2(tanh_series(mul2(f2u(r[e], r[e + 1]), y_in)), cap), u, v);
        r[e] = __float_as_uint(u);
        r[e + 1] = __float_as_uint(v);
      }
    } else if (CAP == kCapPlain) {
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        float u, v;
        by_exponential(e, u, v);
        r[e] = __float_as_uint(u);
        r[e + 1] = __float_as_uint(v);
      }
    } else {
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        float u, v, x, y, s, t;
        by_exponential(e, u, v);
        const F2 at = mul2(f2u(r[e], r[e + 1]), y_in);
        split(at, x, y);
        split(mul2(tanh_series(at), cap), s, t);
        r[e] = __float_as_uint(fabsf(x) <= kSeriesEnd ? s : u);
        r[e + 1] = __float_as_uint(fabsf(y) <= kSeriesEnd ? t : v);
      }
    }
  }
  if (BIAS == kBiasTable) {
    if (lo >= a.reach || hi <= -a.reach) {
      const float c = a.bias[kExt + (lo >= a.reach ? 2 * a.reach : 0)];
#pragma unroll
      for (int e = 0; e < N; e += 2) add_to(r[e], r[e + 1], f2(c, c));
    } else {
      const float* c = a.bias + (d + a.reach + kExt);
#pragma unroll
      for (int e = 0; e < N; e += 2) add_to(r[e], r[e + 1], f2(c[DIR * e], c[DIR * (e + 1)]));
    }
  }
  if (BIAS == kBiasSlope) {
    const float f = float(d);
#pragma unroll
    for (int e = 0; e < N; ++e) r[e] = __float_as_uint(fmaf(a.slope, fabsf(f + float(DIR * e)), __uint_as_float(r[e])));
  }
}
__device__ __forceinline__ Shape shape_of(const ScoredParams& p, int h, float unit, const float* bias) {
  Shape a;
  a.cap = p.cap;
  a.y_in = p.cap > 0.f ? p.scale / p.cap : 0.f;
  a.cap_in = 2.f * kLog2e * a.y_in;
  a.slope = p.slopes ? -p.slopes[h] / unit : 0.f;
  a.bias = bias;
  a.reach = p.reach;
  return a;
}

// Clears the rows of padded tokens of a swizzled tile of `rows` rows and
// `subs` 64-column sub-tiles (a whole warp; a row's swizzled units stay within
// its 128 bytes), so that what they hold meets no product as an operand summed
// over tokens.  doc: the ids of the tile's tokens (-1 past the end, where the
// copy has filled in zeros).
__device__ __forceinline__ void clear_padding(char* tile, int rows, int subs, const int32_t* doc) {
  const int lane = threadIdx.x % 32;
  for (int r = lane; r < rows; r += 32)
    if (doc[r] < 0)
      for (int s = 0; s < subs; ++s)
#pragma unroll
        for (int u = 0; u < 8; ++u) st_shared4(smem_u32(tile) + s * rows * 128 + r * 128 + u * 16, 0u, 0u, 0u, 0u);
  fence_proxy_async_smem();
}

// Calls f.template operator()<BIAS, CAP>() for the bias and cap of p.
template <int CAP, typename Fn>
cudaError_t with_bias(const ScoredParams& p, Fn f) {
  return p.table ? f.template operator()<kBiasTable, CAP>()
                 : p.slopes ? f.template operator()<kBiasSlope, CAP>() : f.template operator()<kBiasNone, CAP>();
}
template <typename Fn>
cudaError_t with_shape(const ScoredParams& p, Fn f) {
  return p.cap > kPlainCap ? with_bias<kCapLarge>(p, f)
                           : p.cap > 0.f ? with_bias<kCapPlain>(p, f) : with_bias<kCapNone>(p, f);
}

// Tensor map of [batch][len][heads][head_dim] as {head_dim, len, heads, batch}
// with boxes of 64 columns x `rows` tokens; head widths that are no multiple
// of 64 are zero-filled by the copy.
inline bool scored_map(CUtensorMap* m, const Strided& t, const ScoredParams& p, int heads, int rows) {
  const uint64_t dims[4] = {uint64_t(p.D), uint64_t(p.L), uint64_t(heads), uint64_t(p.B)};
  // a dimension of one element may carry any stride: give it a valid one
  const int64_t row = (p.D + 7) / 8 * 8;
  const uint64_t strides[3] = {uint64_t(p.L > 1 ? t.sl : row) * 2, uint64_t(heads > 1 ? t.sh : row) * 2,
                               uint64_t(p.B > 1 ? t.sb : row) * 2};
  const uint32_t box[4] = {64, uint32_t(rows), 1, 1};
  return tc_encode(m, t.p, 4, dims, strides, box);
}

}  // namespace
}  // namespace fo
