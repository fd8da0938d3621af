// Orthogonalised updates of weight matrices by Newton-Schulz products, for a
// list of matrices at once, with the momentum before and the parameters' update
// after them.
//
//   X = U / (|U|_F + eps), of U or its transpose so that m <= n;  then `steps` times
//   A = X X^T (m x m);  C = b A + c A A;  X <- a X + C X
//
// A and A A are symmetric: only tiles on and above the diagonal are formed and
// stored, 3 m^2 n + m^3 multiplications and additions per step instead of
// 4 m^2 n + 2 m^3.  An operand whose tile lies below the diagonal is read from
// its mirror image as a matrix with the other major-ness, so nothing is
// transposed in memory.
//
// Operands are fp16, not bf16: singular values stay below about 1.3, so the
// range is known and held in the middle of fp16's by powers of two, and each
// rounding costs 2^-12 instead of 2^-9.  X itself is kept as the sum of two fp16
// numbers (22 bits), and what the product's operands would round most is added
// without them: a X, and for bf16 matrices also the diagonal of C times X, in
// fp32.  The roundings that are left fall on the rest of C, which is small in the
// weak directions that each step multiplies by up to a, and small once the rows
// are orthogonal (errors before the result's rounding: 512 x 512 2.2e-3 with all
// of it in the product, 0.7e-3 without a, 0.5e-3 without the diagonal; 16 x 300
// 2.1, 1.4 and 0.6e-3).  For fp32 matrices, and for bf16 ones that update
// parameters or have a side of up to 16, all operands are such pairs, and each product three (hi lo, lo hi,
// hi hi, in this order; the fourth is below fp32's rounding).  The second number is
// held 2^11 times its size, or it would be subnormal where the first is small: an
// element of X is off by 2^-23 of itself or 2^-46, whichever is more (2^-35 without:
// a row of a 512 x 2048 matrix at 1e-5 of the others was off by 1.9e-3 of itself).
// The tensor cores take the sum of the two mixed products times 2^-11 as they begin
// the third.  Sums are fp32 in tensor memory; because the tensor cores truncate,
// those of pairs are moved to registers and added there, rounded, every 64 terms
// (matrices of width 512 are 7e-7 off, moved every 512 terms they were 7e-6;
// torch's fp32 products 2.3e-6).
//
// X, A and C lie in the workspace as blocks of 64 x 64 elements of 8 KB in the
// image that a 128-byte-swizzled operand has in shared memory, block rows
// fastest: every operand tile is a few contiguous copies without a tensor map,
// whatever the number and sizes of the matrices, and the padding of odd sizes to
// 128 is zeros.
//
// A pair of CTAs (cta_group::2) works on a tile of 256 x 256 or 256 x 128: each
// loads its 128 rows and half of the columns' operand.  A single CTA's tile of
// 128 x 128 loads twice to four times the bytes per product, and 64 bytes per
// clock and SM is what L2 gives: it ran 4096 x 4096 at 1.0 PFLOP/s.
#include "fo_scored_tc.cuh"
#include "fo_vec8.cuh"
#include "../../include/fedoptima.h"

#include <algorithm>
#include <atomic>
#include <cmath>
#include <functional>
#include <new>
#include <string>
#include <vector>

namespace fo {
int report_error(int code, const std::string& msg);

namespace {

__device__ GaveUp g_err;

constexpr int kItems = 32;                    // matrices per launch
constexpr int kBlock = 8192;                  // bytes of a 64 x 64 block
constexpr int kMaxSums = 1024;                // partial sums of squares per matrix
constexpr float kUpX = 1024.f, kUpA = 256.f;  // what X, and A and C, are multiplied by as fp16
constexpr int kLowBits = 11;                  // and the second number of a pair by 2^11 more
constexpr float kUpLow = 1 << kLowBits, kDownLow = 1.f / kUpLow;

struct Item {
  const void* g;            // [rows][cols] gradient
  float *mom, *param;
  void* out;
  int64_t ldg, ldm, ldp, ldo;
  int64_t x[2], a, c, d;    // byte offsets in the workspace; d: the diagonal of C
  int64_t parts;            // of A's shared sums, [tile][split - 1][CTA][warp] of 8 KB
  int rows, cols, mt, nt;   // mt, nt: tiles of 128 of the smaller and the larger side
  int nsums;                // partial sums of squares, at kMaxSums times its index
  bool transposed, vec_in, vec_out;
  float step;
};
struct OrthoParams {
  Item item[kItems];
  int start[kItems + 1];    // first unit of work of each matrix in this launch
  uint8_t order[kItems];    // the matrices in the order of their units
  char* ws;
  float4* sums;
  float2* scale;            // of each matrix: the two factors that make X of U
  int count, from, last;    // from: which X is read; last: X goes to the caller
  float ca, cb, cc, mu, decay;
  bool nesterov;
  float eps;
};

__device__ __forceinline__ int slot_of(const OrthoParams& p, int unit) {
  int n = 0;
  while (n + 1 < p.count && unit >= p.start[n + 1]) ++n;
  return n;
}

// ------------------------------------------------------------- before the steps
// U of eight neighbouring elements, zeros outside of the matrix; FIRST updates
// the momentum, afterwards it is read.
template <typename T, bool FIRST>
__device__ __forceinline__ void update8(const OrthoParams& p, const Item& it, int64_t r, int c, float (&v)[8]) {
  const T* g = static_cast<const T*>(it.g) + r * it.ldg + c;
  float* m = it.mom ? it.mom + r * it.ldm + c : nullptr;
  const int left = r < it.rows ? it.cols - c : 0;
  if (it.vec_in && left >= 8) {
    Raw8<T> raw;
    raw.load(g);
    raw.get(v);
    if (m) {
      Raw8<float> old;
      old.load(m);
      float z[8];
      old.get(z);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (FIRST) z[e] = fmaf(p.mu, z[e], v[e]);
        v[e] = p.nesterov ? fmaf(p.mu, z[e], v[e]) : z[e];
      }
      if (FIRST) store8(m, z);
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    v[e] = 0.f;
    if (e < left) {
      v[e] = to_f(g[e]);
      if (m) {
        float z = m[e];
        if (FIRST) m[e] = z = fmaf(p.mu, z, v[e]);
        v[e] = p.nesterov ? fmaf(p.mu, z, v[e]) : z;
      }
    }
  }
}

// X = U (kUpX / (|U| + eps)), |U| = root 2^unit: the factor as a power of two,
// which goes first, and a rest near kUpX, so that neither leaves fp32's range.
// (fp32 throughout: double arithmetic takes microseconds here.)
__device__ __forceinline__ float2 factors(float root, int unit, float eps) {
  const float n = root + scalbnf(eps, -unit);
  if (!(n < INFINITY)) return make_float2(1.f / n, 1.f);
  const int k = ilogbf(n);
  return make_float2(scalbnf(1.f, min(127, -(unit + k))), kUpX / scalbnf(n, -k));
}
// Sums of squares of elements within 2^-40 .. 2^40, above (in units of 2^160) and
// below (2^-160).
struct Squares {
  float mid, big, small;
  __device__ __forceinline__ void add(float x) {
    const float a = fabsf(x);
    if (a > 0x1p40f) big = fmaf(x * 0x1p-80f, x * 0x1p-80f, big);
    else if (a < 0x1p-40f) small = fmaf(x * 0x1p80f, x * 0x1p80f, small);
    else mid = fmaf(x, x, mid);         // NaN too
  }
  __device__ __forceinline__ void add(const float4& o) {
    mid += o.x;
    big += o.y;
    small += o.z;
  }
  // The sums over a block, in its first thread.
  __device__ __forceinline__ float4 over_block(float4* box) {
    mid = warp_sum(mid);
    big = warp_sum(big);
    small = warp_sum(small);
    if (threadIdx.x % 32 == 0) box[threadIdx.x / 32] = make_float4(mid, big, small, 0.f);
    __syncthreads();
    if (threadIdx.x == 0)
      for (unsigned w = 1; w < blockDim.x / 32; ++w) add(box[w]);
    return make_float4(mid, big, small, 0.f);
  }
  // Root of the sum and its unit, a power of two.
  __device__ __forceinline__ float root(int& unit) const {
    unit = big > 0.f ? 40 : mid > 0.f ? 0 : -80;
    const float r = big > 0.f ? hypotf(sqrtf(big) * 0x1p40f, sqrtf(mid) * 0x1p-40f)
                              : mid > 0.f ? hypotf(sqrtf(mid), sqrtf(small) * 0x1p-80f) : sqrtf(small);
    return r + (mid + big + small) * 0.f;        // NaN and infinity stay
  }
};

template <typename T>
__global__ void __launch_bounds__(256) ortho_sums_k(const __grid_constant__ OrthoParams p) {
  __shared__ float4 box[8];
  pdl_wait();
  pdl_trigger();
  const int n = slot_of(p, blockIdx.x), part = int(blockIdx.x) - p.start[n];
  const Item& it = p.item[n];
  const uint32_t per_row = uint32_t(it.cols + 7) / 8;               // vectors of eight
  const int64_t total = int64_t(it.rows) * per_row, stride = int64_t(it.nsums) * 256;
  int64_t e = int64_t(part) * 256 + threadIdx.x, row = e / per_row;
  uint32_t col = uint32_t(e - row * per_row);
  const int64_t down = stride / per_row;
  const uint32_t right = uint32_t(stride - down * per_row);
  Squares sum = {};
  auto next = [&] {
    row += down;
    col += right;
    if (col >= per_row) col -= per_row, ++row;
  };
  constexpr int U = 4;                                              // in flight
  if (it.vec_in && !it.mom && it.cols % 8 == 0) {
    for (; e < total; e += U * stride) {
      Raw8<T> raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        raw[u].zero();
        if (row < it.rows) raw[u].load(static_cast<const T*>(it.g) + row * it.ldg + 8 * col);
        next();
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float v[8];
        raw[u].get(v);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum.add(v[k]);
      }
    }
  } else {
    for (; e < total; e += stride) {
      float v[8];
      update8<T, true>(p, it, row, 8 * int(col), v);
#pragma unroll
      for (int k = 0; k < 8; ++k) sum.add(v[k]);
      next();
    }
  }
  const float4 all = sum.over_block(box);
  if (threadIdx.x == 0) p.sums[n * kMaxSums + part] = all;
}

__global__ void __launch_bounds__(256) ortho_scale_k(const __grid_constant__ OrthoParams p) {
  __shared__ float4 box[8];
  pdl_wait();
  pdl_trigger();
  const int n = blockIdx.x;
  Squares sum = {};
#pragma unroll
  for (int i = 0; i < kMaxSums / 256; ++i)
    if (int(threadIdx.x) + 256 * i < p.item[n].nsums) sum.add(p.sums[n * kMaxSums + threadIdx.x + 256 * i]);
  sum.over_block(box);
  if (threadIdx.x == 0) {
    int unit;
    const float root = sum.root(unit);
    p.scale[n] = factors(root, unit, p.eps);
  }
}

__device__ __forceinline__ uint32_t half_pair(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 of_pair(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
// Eight values' first (PART 0) or second number as fp16; v keeps what it leaves.
template <int PART>
__device__ __forceinline__ uint4 take_half8(float* v) {
  constexpr float up = PART ? kUpLow : 1.f, down = PART ? kDownLow : 1.f;
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    w[e] = half_pair(v[2 * e] * up, v[2 * e + 1] * up);
    const float2 f = of_pair(w[e]);
    v[2 * e] = fmaf(-down, f.x, v[2 * e]);
    v[2 * e + 1] = fmaf(-down, f.y, v[2 * e + 1]);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// X = U / (|U| + eps) as an image: one 64 x 64 block per block of threads.
template <typename T>
__global__ void __launch_bounds__(256) ortho_pack_k(const __grid_constant__ OrthoParams p) {
  __shared__ float tile[64][65];
  pdl_wait();
  pdl_trigger();
  const int n = slot_of(p, blockIdx.x);
  const Item& it = p.item[n];
  const int blk = int(blockIdx.x) - p.start[n], rows = 2 * it.mt;
  const int rb = blk % rows, cb = blk / rows, t = threadIdx.x, row = t / 4;
  // the user's matrix: two groups of eight of one row
  const int r0 = 64 * (it.transposed ? cb : rb), c0 = 64 * (it.transposed ? rb : cb);
  float v[2][8];
#pragma unroll
  for (int h = 0; h < 2; ++h) update8<T, false>(p, it, r0 + row, c0 + 8 * (t % 4 * 2 + h), v[h]);
  const float2 scale = p.scale[n];
  if (it.transposed)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 8; ++e) tile[row][8 * (t % 4 * 2 + h) + e] = v[h][e];
  if (it.transposed) __syncthreads();
  char* img = p.ws + it.x[0] + (cb * int64_t(rows) + rb) * kBlock + row * 128;
  const int64_t image = int64_t(it.mt) * it.nt * 4 * kBlock;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int u = t % 4 * 2 + h, at = (u ^ (row & 7)) * 16;
    float z[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = (it.transposed ? tile[8 * u + e][row] : v[h][e]) * scale.x * scale.y;
    *reinterpret_cast<uint4*>(img + at) = take_half8<0>(z);
    *reinterpret_cast<uint4*>(img + image + at) = take_half8<1>(z);
  }
}

// ------------------------------------------------------------------ products
enum { kGram = 0, kPoly = 1, kApply = 2 };
constexpr int kThreads = 320;                 // copies, products, eight warps of arithmetic

// Per CTA of a pair, for tiles of 256 x BN: 128 rows of A's operand and BN / 2 of
// B's by 64 terms, in PARTS parts each.
template <int PARTS, int BN>
struct Tiles {
  static constexpr int kA = 2 * kBlock, kB = BN / 128 * kBlock;
  static constexpr int kStage = PARTS * (kA + kB), kStages = 196608 / kStage;
  static constexpr int kOut = 8 * 4096;       // 4 KB per warp of arithmetic
  static constexpr int kSumsAt = 512 / BN;    // tiles' sums in tensor memory
  static constexpr int kBars = 3 * kStages + 2 * kSumsAt + 9;
  static constexpr int kSmem = 1024 + kStages * kStage + kOut + 8 * kBars + 16;
};
static_assert(Tiles<1, 256>::kSmem <= 232448 && Tiles<1, 128>::kSmem <= 232448 && Tiles<2, 128>::kSmem <= 232448, "shared memory per CTA");

struct Place {
  int item, tile;           // the tile's number among the matrix's
  int i, j;                 // rows 256 i, columns BN j
  int k0, kb;               // first block of 64 terms, and how many (none: nothing to do)
};
// `share` of `shares` of the terms.
template <int PHASE, int BN>
__device__ __forceinline__ Place place_of(const OrthoParams& p, int unit, int share, int shares) {
  Place a;
  const int n = slot_of(p, unit);
  a.item = p.order[n];
  const Item& it = p.item[a.item];
  const int t = unit - p.start[n];
  a.tile = t;
  const int h = (it.mt + 1) / 2, cols = PHASE == kApply ? it.nt : it.mt;
  if (PHASE == kApply) {
    a.i = t % h;
    a.j = t / h;
  } else {                  // 256 x 256 on and above the diagonal, column by column
    const int u = BN == 256 ? t : t / 2;
    int j = int((sqrtf(8.f * float(u) + 1.f) - 1.f) * 0.5f);
    while ((j + 1) * (j + 2) / 2 <= u) ++j;
    while (j * (j + 1) / 2 > u) --j;
    a.i = u - j * (j + 1) / 2;
    a.j = BN == 256 ? j : 2 * j + t % 2;
  }
  const int all = a.j * (BN / 128) < cols ? 2 * (PHASE == kGram ? it.nt : it.mt) : 0;
  a.k0 = all * share / shares;
  a.kb = all * (share + 1) / shares - a.k0;
  return a;
}
// A symmetric matrix holds its 128 x 128 tiles (i, j) with i / 2 <= j / 2.  Rows
// 128 i .. of block column kb lie there as rows, or mirrored, as columns of block
// row kb.
__device__ __forceinline__ bool mirrored(int i, int kb) { return i / 2 > kb / 4; }

// Arrivals, products and commits of the two CTAs.  Arrivals and waits keep the
// default scope: with release and acquire at cluster scope each block of terms
// took 1 us (4096 x 4096: 2361 us).  Copies are plain ones to this CTA's barrier,
// of which a warp tells the leader; tensor copies that complete on the leader's
// barrier themselves were 10% slower on 256 x 256 tiles (rows of 128 bytes).
__device__ __forceinline__ void arrive_at(uint64_t* bar, uint32_t rank) {
  asm volatile(
      "{\n .reg .b32 r;\n mapa.shared::cluster.u32 r, %0, %1;\n mbarrier.arrive.shared::cluster.b64 _, [r];\n}\n" ::"r"(
          smem_u32(bar)),
      "r"(rank)
      : "memory");
}
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.b32 p, %4, 0;\n elect.sync _|q, 0xffffffff;\n"
      " @q tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(acc)
      : "memory");
}
// d <- a b + 2^-kLowBits d, of a pair of CTAs or of one.
template <int CTAS>
__device__ __forceinline__ void mma_onto_low(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc) {
  if constexpr (CTAS == 2)
    asm volatile(
        "{\n .reg .pred p, q;\n setp.eq.b32 p, 0, 0;\n elect.sync _|q, 0xffffffff;\n"
        " @q tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p, %4;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "n"(kLowBits)
        : "memory");
  else
    asm volatile(
        "{\n .reg .pred p, q;\n setp.eq.b32 p, 0, 0;\n elect.sync _|q, 0xffffffff;\n"
        " @q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p, %4;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "n"(kLowBits)
        : "memory");
}
__device__ __forceinline__ void commit_pair(uint64_t* bar, uint32_t leader) {     // the barrier of both CTAs
  asm volatile(
      "{\n .reg .pred q;\n elect.sync _|q, 0xffffffff;\n"
      " @q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n}\n" ::"r"(smem_u32(bar)),
      "h"(uint16_t(3u << leader))
      : "memory");
}

// 32 elements of kUpX X, row 128 tile + 32 q + lane and columns c0 .., to the caller.
template <typename T>
__device__ __forceinline__ void deliver(const OrthoParams& p, const Item& m, int tile, int c0, int q, int lane, uint32_t buf, const float* v) {
  const int row = 128 * tile + 32 * q + lane;
  constexpr float down = 1.f / kUpX;
  const int side = m.transposed ? m.cols : m.rows, wide = m.transposed ? m.rows : m.cols;
  if (m.transposed) {       // a row here is a column there: lanes are neighbours
    if (row >= side) return;
    if (m.out) {
      T* o = static_cast<T*>(m.out) + c0 * m.ldo + row;
#pragma unroll
      for (int e = 0; e < 32; ++e, o += m.ldo)
        if (c0 + e < wide) *o = from_f<T>(v[e] * down);
    }
    if (m.param) {
      float* w = m.param + c0 * m.ldp + row;
#pragma unroll
      for (int e = 0; e < 32; ++e, w += m.ldp)
        if (c0 + e < wide) *w = fmaf(-m.step, v[e] * down, *w * p.decay);
    }
    return;
  }
  // through shared memory: eight lanes then hold a row's
  __syncwarp();
#pragma unroll
  for (int k = 0; k < 8; ++k)
    st_shared4(buf + lane * 128 + (k ^ (lane & 7)) * 16, __float_as_uint(v[4 * k] * down), __float_as_uint(v[4 * k + 1] * down),
               __float_as_uint(v[4 * k + 2] * down), __float_as_uint(v[4 * k + 3] * down));
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int rr = 4 * i + lane / 8, r = 128 * tile + 32 * q + rr, c = c0 + 4 * (lane % 8);
    const float4 x = ld_shared4(buf + rr * 128 + ((lane % 8) ^ (rr & 7)) * 16);
    if (r >= side || c >= wide) continue;
    const float z[4] = {x.x, x.y, x.z, x.w};
    if (m.out) {
      T* o = static_cast<T*>(m.out) + r * m.ldo + c;
      if (m.vec_out && c + 4 <= wide) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(o) = x;
        else *reinterpret_cast<uint2*>(o) = make_uint2(bf16_pair(z[0], z[1]), bf16_pair(z[2], z[3]));
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c + e < wide) o[e] = from_f<T>(z[e]);
      }
    }
    if (m.param) {
      float* w = m.param + r * m.ldp + c;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < wide) w[e] = fmaf(-m.step, z[e], w[e] * p.decay);
    }
  }
  __syncwarp();
}

// Several pairs of a cluster share a tile's terms: the others leave their sums in
// the workspace, and the first adds them in their order.  Every lane its own, 16
// bytes beside its neighbours'.
__device__ __forceinline__ float4* shared_at(const OrthoParams& p, const Item& m, int tile, int share, int shares, int me, int warp) {
  return reinterpret_cast<float4*>(p.ws + m.parts + (((int64_t(tile) * (shares - 1) + share - 1) * 2 + me) * 8 + warp) * 8192);
}
__device__ __forceinline__ void leave_sums(float4* to, int lane, const float (&v)[64]) {
#pragma unroll
  for (int k = 0; k < 16; ++k) __stcg(to + 32 * k + lane, make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]));
}
__device__ __forceinline__ void add_sums(const float4* from, int lane, float (&v)[64]) {
  float4 w[16];
#pragma unroll
  for (int k = 0; k < 16; ++k) w[k] = __ldcg(from + 32 * k + lane);
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    v[4 * k] += w[k].x;
    v[4 * k + 1] += w[k].y;
    v[4 * k + 2] += w[k].z;
    v[4 * k + 3] += w[k].w;
  }
}

// 64 sums of one row, columns 64 cblk .., become elements of A, C or X.
template <int PARTS, int PHASE, typename T>
__device__ __forceinline__ void finish(const OrthoParams& p, const Item& m, int tile, int cblk, int q, int lane, uint32_t buf, float (&v)[64]) {
  const int64_t block = int64_t(cblk) * 2 * m.mt + 2 * tile + q / 2;
  const int64_t half_block = block * kBlock + (q & 1) * 4096;       // this warp's 32 rows
  const int64_t xi = int64_t(m.mt) * m.nt * 4 * kBlock, si = int64_t(m.mt) * m.mt * 4 * kBlock;
  if (PHASE == kGram) {
#pragma unroll
    for (int e = 0; e < 64; ++e) v[e] *= kUpA / (kUpX * kUpX);
  } else {
    // C = b A + c A A, or a X + C X
    const float other = (PHASE == kPoly ? p.cc : 1.f) / kUpA;
    float linear = p.cb;
    if (PHASE == kApply) linear = PARTS == 2 ? p.ca : fmaf(1.f / kUpA, reinterpret_cast<const float*>(p.ws + m.d)[128 * tile + 32 * q + lane], p.ca);
    // the warp's 4 KB are read as they lie, and handed out by rows through shared memory
    const uint4* src = reinterpret_cast<const uint4*>(p.ws + (PHASE == kPoly ? m.a : m.x[p.from]) + half_block) + lane;
    constexpr int kParts = PHASE == kPoly ? PARTS : 2;
    const int64_t image = (PHASE == kPoly ? si : xi) / 16;
    uint4 w[kParts][8];
#pragma unroll
    for (int part = 0; part < kParts; ++part)
#pragma unroll
      for (int k = 0; k < 8; ++k) w[part][k] = src[part * image + 32 * k];
    if (lane == 0) bulk_wait_read<0>();       // the last store has read the buffer
#pragma unroll
    for (int part = kParts - 1; part >= 0; --part) {
      const float factor = part ? linear * kDownLow : linear;
      __syncwarp();
#pragma unroll
      for (int k = 0; k < 8; ++k) st_shared4(buf + (32 * k + lane) * 16, w[part][k].x, w[part][k].y, w[part][k].z, w[part][k].w);
      __syncwarp();
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float4 u = ld_shared4(buf + lane * 128 + (k ^ (lane & 7)) * 16);
        const float z[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 f = of_pair(__float_as_uint(z[e]));
          float &x = v[8 * k + 2 * e], &y = v[8 * k + 2 * e + 1];
          x = fmaf(factor, f.x, part == kParts - 1 ? x * other : x);
          y = fmaf(factor, f.y, part == kParts - 1 ? y * other : y);
        }
      }
    }
    __syncwarp();
  }
  if (PARTS == 1 && PHASE == kPoly && 2 * tile + q / 2 == cblk) {      // the diagonal goes its own way
    float diagonal = 0.f;
    const uint32_t bit = 1u << lane;       // a mask, not an index, which would move v to memory
#pragma unroll
    for (int e = 0; e < 64; ++e) {
      const bool here = (bit >> e % 32 & 1u) && e / 32 == q % 2;
      diagonal += here ? v[e] : 0.f;
      v[e] = here ? 0.f : v[e];
    }
    reinterpret_cast<float*>(p.ws + m.d)[128 * tile + 32 * q + lane] = diagonal;
  }
  if (PHASE == kApply && p.last) {
    deliver<T>(p, m, tile, 64 * cblk, q, lane, buf, v);
    deliver<T>(p, m, tile, 64 * cblk + 32, q, lane, buf, v + 32);
    return;
  }
  char* dst = p.ws + (PHASE == kGram ? m.a : PHASE == kPoly ? m.c : m.x[p.from ^ 1]) + half_block;
  const int64_t image = PHASE == kApply ? xi : si;
#pragma unroll
  for (int part = 0; part < (PHASE == kApply ? 2 : PARTS); ++part) {
    if (lane == 0) bulk_wait_read<0>();       // the last store has read the buffer
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint4 w = part ? take_half8<1>(v + 8 * k) : take_half8<0>(v + 8 * k);
      st_shared4(buf + lane * 128 + (k ^ (lane & 7)) * 16, w.x, w.y, w.z, w.w);
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], 4096;" ::"l"(dst + part * image), "r"(buf) : "memory");
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
  }
}

template <int PARTS, int BN, int PHASE, bool SHARED, typename T>
__device__ __forceinline__ void product_tiles(const OrthoParams& p, int pairs_of_tile) {
  using S = Tiles<PARTS, BN>;
  extern __shared__ char smem_raw[];
  char* smem = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  char* stage_out = smem + S::kStages * S::kStage;
  uint64_t* full = reinterpret_cast<uint64_t*>(stage_out + S::kOut);
  uint64_t *peer = full + S::kStages, *empty = peer + S::kStages, *acc_full = empty + S::kStages, *acc_empty = acc_full + S::kSumsAt,
           *done = acc_empty + S::kSumsAt, *left = done + 1;       // left: a warp's sums of the cluster's other pairs
  uint32_t* tslot = reinterpret_cast<uint32_t*>(left + 8);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  // a cluster of 2 * shares CTAs takes a tile
  const int shares = SHARED ? pairs_of_tile : 1;
  const int units = p.start[p.count], pair = int(blockIdx.x) / (2 * shares), pairs = int(gridDim.x) / (2 * shares);
  const int rank = int(blockIdx.x) % (2 * shares), me = rank % 2, leader = rank - me, share = rank / 2;

  if (threadIdx.x == 0) {
    for (int e = 0; e < S::kStages; ++e) {
      mbar_init(&full[e], 1);
      mbar_init(&peer[e], 1);
      mbar_init(&empty[e], 1);
    }
    for (int e = 0; e < S::kSumsAt; ++e) {
      mbar_init(&acc_full[e], 1);
      mbar_init(&acc_empty[e], 16);        // one arrival per warp of arithmetic, of both CTAs
    }
    mbar_init(done, 1);
    for (int e = 0; e < 8; ++e) mbar_init(&left[e], shares > 1 ? shares - 1 : 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tslot)), "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                // both CTAs' barriers are there
  tc_fence_after();
  const uint32_t tmem = *tslot;      // sum s: columns BN s
  pdl_trigger();                     // this block holds its tensor memory
  pdl_wait();
  Waits wait(&g_err);

  if (warp == 0) {
    if (lane == 0) {
      Ring<S::kStages> at;
      int it = 0;
      for (int u = pair; u < units && !wait.dead; u += pairs) {
        const Place a = place_of<PHASE, BN>(p, u, share, shares);
        const Item& m = p.item[a.item];
        const char* x = p.ws + m.x[p.from];
        const char* sym = p.ws + (PHASE == kPoly ? m.a : m.c);
        const int64_t xi = int64_t(m.mt) * m.nt * 4 * kBlock, si = int64_t(m.mt) * m.mt * 4 * kBlock;
        const int cols = PHASE == kApply ? m.nt : m.mt;       // tiles of 128
        const int ta = 2 * a.i + me, tb = BN == 256 ? 2 * a.j + me : a.j;
        const bool has_a = ta < m.mt, has_b = tb < cols;
        const uint32_t bytes = PARTS * ((has_a ? S::kA : 0) + (has_b ? S::kB : 0));
        const int64_t wide = int64_t(2 * m.mt) * kBlock;      // from one block column to the next
        for (int kb = a.k0; kb < a.k0 + a.kb; ++kb, ++it) {
          if (it >= S::kStages) wait.on(&empty[at.at], at.phase ^ 1, 61);
          if (wait.dead) break;
          char* s = smem + at.at * S::kStage;
          uint64_t* bar = &full[at.at];
          mbar_expect_tx(bar, bytes);
#pragma unroll
          for (int q = 0; q < PARTS; ++q) {
            if (has_a) {
              char* d = s + q * S::kA;
              const char* src = PHASE == kGram ? x + q * xi : sym + q * si;
              if (PHASE == kGram || !mirrored(ta, kb)) {
                bulk_g2s(d, src + kb * wide + int64_t(2 * ta) * kBlock, 2 * kBlock, bar);
              } else {
                src += 2 * ta * wide + int64_t(kb) * kBlock;
                bulk_g2s(d, src, kBlock, bar);
                bulk_g2s(d + kBlock, src + wide, kBlock, bar);
              }
            }
            if (has_b) {
              char* d = s + PARTS * S::kA + q * S::kB;
              const char* src = PHASE == kPoly ? sym + q * si : x + q * xi;
              const int b0 = BN == 256 ? 2 * tb : 2 * tb + me;          // this CTA's first block
              if (PHASE == kGram || (PHASE == kPoly && !mirrored(tb, kb))) {
                bulk_g2s(d, src + kb * wide + int64_t(b0) * kBlock, S::kB, bar);
              } else {
                src += b0 * wide + int64_t(kb) * kBlock;
                bulk_g2s(d, src, kBlock, bar);
                if (BN == 256) bulk_g2s(d + kBlock, src + wide, kBlock, bar);
              }
            }
          }
          at.step();
        }
      }
      // every copy has landed before the block ends, whichever role gave up
      for (int e = max(0, it - S::kStages); e < it; ++e) mbar_wait(&full[e % S::kStages], (e / S::kStages) & 1);
    }
  } else if (warp == 1 && me == 1) {
    // tells the leader what has landed here
    if (lane == 0) {
      Ring<S::kStages> at;
      for (int u = pair; u < units && !wait.dead; u += pairs) {
        const Place a = place_of<PHASE, BN>(p, u, share, shares);
        for (int kb = 0; kb < a.kb; ++kb) {
          wait.on(&full[at.at], at.phase, 65);
          if (wait.dead) break;
          arrive_at(&peer[at.at], leader);
          at.step();
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // kind::f16 with fp16 operands, fp32 sums, M = 256, N = BN
    constexpr uint32_t id = (1u << 4) | uint32_t(BN >> 3) << 17 | (256u >> 4) << 24;
    Ring<S::kStages> at;
    Ring<S::kSumsAt> sum;
    const uint32_t ring = smem_u32(smem);
    bool dead = false;
    for (int u = pair; u < units && !dead; u += pairs) {
      const Place a = place_of<PHASE, BN>(p, u, share, shares);
      const int tb = BN == 256 ? 2 * a.j : a.j;
      for (int kb = 0; kb < a.kb; ++kb) {
        const uint32_t d = tmem + sum.at * BN;
        const bool fresh = PARTS == 2 || kb == 0;
        if (fresh) wait.on(&acc_empty[sum.at], sum.phase ^ 1, 62);
        wait.on(&full[at.at], at.phase, 63);
        wait.on(&peer[at.at], at.phase, 66);
        __syncwarp();
        tc_fence_after();
        const uint32_t s = ring + at.at * S::kStage;
        // mirrored operands have their rows along the terms
        const uint32_t am = PHASE != kGram && mirrored(2 * a.i, kb), bm = PHASE == kApply || (PHASE == kPoly && mirrored(tb, kb));
        const uint32_t idesc = id | am << 15 | bm << 16;
        const uint32_t as = am ? 2048u : 32u, bs = bm ? 2048u : 32u;
        const uint32_t al = (am ? uint32_t(kBlock) : 16u) >> 4 << 16, bl = (bm ? uint32_t(kBlock) : 16u) >> 4 << 16;
        constexpr uint32_t hi = (1024u >> 4) | (1u << 14) | (2u << 29);      // stride 1024, version 1, 128-byte swizzle
        auto desc = [&](uint32_t off, uint32_t lbo) { return uint64_t(((s + off) & 0x3ffff) >> 4 | lbo) | uint64_t(hi) << 32; };
        constexpr uint32_t b0 = PARTS * S::kA;
        if (PARTS == 2) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            mma_pair(d, desc(k * as, al), desc(b0 + S::kB + k * bs, bl), idesc, k > 0 ? 1u : 0u);
            mma_pair(d, desc(S::kA + k * as, al), desc(b0 + k * bs, bl), idesc, 1u);
          }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (PARTS == 2 && k == 0) mma_onto_low<2>(d, desc(0, al), desc(b0, bl), idesc);
          else mma_pair(d, desc(k * as, al), desc(b0 + k * bs, bl), idesc, PARTS == 2 || kb > 0 || k > 0 ? 1u : 0u);
        }
        commit_pair(&empty[at.at], leader);
        at.step();
        if (PARTS == 2 || kb + 1 == a.kb) {
          commit_pair(&acc_full[sum.at], leader);
          sum.step();
        }
        // off the waits' path; what was issued after one gave up is void anyway
        dead = __any_sync(0xffffffffu, wait.dead);
        if (dead) break;
      }
    }
    // no product is in flight when the blocks end and their memory is another's
    asm volatile(
        "{\n .reg .pred q;\n elect.sync _|q, 0xffffffff;\n"
        " @q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(smem_u32(done))
        : "memory");
    mbar_wait(done, 0);
    __syncwarp();
  } else {
    // warp: 32 rows 32 q .. and half of the columns, in blocks of 64
    const int q = warp % 4, half = (warp - 2) / 4;
    constexpr int NB = BN / 128;
    const uint32_t col = tmem + (uint32_t(32 * q) << 16) + (BN / 2) * half;
    const uint32_t buf = smem_u32(stage_out) + uint32_t(warp - 2) * 4096u;
    Ring<S::kSumsAt> sum;
    uint32_t turn = 0;
    // before the end of a tile of which the cluster's pairs have shared the terms: whether this pair finishes it
    auto shared = [&](const Item& m, int tile, float (&v)[64]) {
      if (!SHARED) return true;
      if (share > 0) {
        leave_sums(shared_at(p, m, tile, share, shares, me, warp - 2), lane, v);
        __syncwarp();
        if (lane == 0) {
          asm volatile("fence.acq_rel.cluster;" ::: "memory");
          arrive_at(&left[warp - 2], me);
        }
        __syncwarp();
        return false;
      }
      wait.on_lanes(&left[warp - 2], turn, 72);
      turn ^= 1;
      asm volatile("fence.acq_rel.cluster;" ::: "memory");
      for (int s = 1; s < shares; ++s) add_sums(shared_at(p, m, tile, s, shares, me, warp - 2), lane, v);
      return true;
    };
    bool dead = false;
    for (int u = pair; u < units && !dead; u += pairs) {
      const Place a = place_of<PHASE, BN>(p, u, share, shares);
      if (a.kb == 0) continue;
      const Item& m = p.item[a.item];
      const int tile = 2 * a.i + me, cblk = a.j * (BN / 64) + half * NB, cols = 2 * (PHASE == kApply ? m.nt : m.mt);
      float v[PARTS == 2 ? NB : 1][64];
      if (PARTS == 2) {
        for (int kb = 0; kb < a.kb; ++kb) {
          wait.on(&acc_full[sum.at], sum.phase, 64);
          __syncwarp();
          tc_fence_after();
#pragma unroll
          for (int h = 0; h < 2 * NB; ++h) {
            uint32_t r[32];
            tmem_ld32(col + sum.at * BN + 32 * h, r);
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              float& x = v[h / 2][32 * (h % 2) + e];
              x = (kb > 0 ? x : 0.f) + __uint_as_float(r[e]);
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_at(&acc_empty[sum.at], leader);
          sum.step();
        }
        dead = __any_sync(0xffffffffu, wait.dead);
        if (dead) break;
#pragma unroll
        for (int b = 0; b < NB; ++b)
          if (tile < m.mt && cblk + b < cols && shared(m, a.tile, v[b])) finish<PARTS, PHASE, T>(p, m, tile, cblk + b, q, lane, buf, v[b]);
      } else {
        wait.on(&acc_full[sum.at], sum.phase, 64);
        __syncwarp();
        tc_fence_after();
        dead = __any_sync(0xffffffffu, wait.dead);
#pragma unroll 1
        for (int b = 0; b < NB; ++b) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t r[32];
            tmem_ld32(col + sum.at * BN + 64 * b + 32 * h, r);
#pragma unroll
            for (int e = 0; e < 32; ++e) v[0][32 * h + e] = __uint_as_float(r[e]);
          }
          if (b == NB - 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_at(&acc_empty[sum.at], leader);
          }
          if (!dead && tile < m.mt && cblk + b < cols && shared(m, a.tile, v[0])) finish<PARTS, PHASE, T>(p, m, tile, cblk + b, q, lane, buf, v[0]);
        }
        sum.step();
      }
    }
    if (lane == 0) bulk_wait_all();
    __syncwarp();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                // neither CTA is needed by the other any more
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

// Pairs, and clusters of `shares` pairs.
template <int PARTS, int BN, int PHASE, typename T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) ortho_product_k(const __grid_constant__ OrthoParams p) {
  product_tiles<PARTS, BN, PHASE, false, T>(p, 1);
}
template <int PARTS, typename T>
__global__ void __launch_bounds__(kThreads, 1) ortho_shared_k(const __grid_constant__ OrthoParams p, int shares) {
  product_tiles<PARTS, 128, kGram, true, T>(p, shares);
}

// ------------------------------------------------------------ up to 128 rows
// A matrix whose smaller side is at most 128 and the larger one at most 2048 stays
// in shared memory for all steps: each of up to eight CTAs of a cluster holds all
// rows of 256 columns of X (two parts), forms its columns' part of X X^T, and,
// with the sum of the parts, all of A A and C and its own columns of C X.  The
// parts are exchanged through the workspace (L2).  One launch for all such
// matrices of a list.  A step is a chain of three products on one SM, each too
// short to fill it: its latency is what counts, and launches of their own cost
// more (200 x 96 fp32: 143 us).
constexpr int kSmallRows = 128, kSmallCols = 256, kSmallCtas = 8;
constexpr int kSmallThreads = 512, kSmallUnits = kSmallRows * kSmallCols / 8 / kSmallThreads;
constexpr int kSmallX = 8 * kBlock, kSmallA = 4 * kBlock;             // one part of X, of A or C
constexpr int kSmallSmem = 1024 + 2 * kSmallX + 2 * kSmallA + 32 + 16 * 16 + kSmallRows * 4;
constexpr int kSmallPart = kSmallRows * kSmallRows * 4;                // of X X^T
static_assert(kSmallSmem <= 232448, "shared memory per CTA");

// 32 elements of a row of a block, from unit `first` of eight on, as one or two
// parts of fp16.
template <int PARTS>
__device__ __forceinline__ void put_row(uint32_t at, uint32_t part, int row, int first, float (&v)[32]) {
#pragma unroll
  for (int q = 0; q < PARTS; ++q)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint4 w = q ? take_half8<1>(v + 8 * k) : take_half8<0>(v + 8 * k);
      st_shared4(at + q * part + row * 128 + ((first + k) ^ (row & 7)) * 16, w.x, w.y, w.z, w.w);
    }
}

template <int PARTS, typename T>
__global__ void __cluster_dims__(kSmallCtas, 1, 1) __launch_bounds__(kSmallThreads, 1) ortho_small_k(const __grid_constant__ OrthoParams p, int steps) {
  extern __shared__ char smem_raw[];
  char* smem = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, t = threadIdx.x;
  const Item& m = p.item[blockIdx.x / kSmallCtas];
  const int me = blockIdx.x % kSmallCtas;
  const int cols = m.transposed ? m.rows : m.cols;      // the larger side
  const int ctas = (cols + kSmallCols - 1) / kSmallCols, col0 = me * kSmallCols;
  if (me >= ctas) return;
  const int blocks = (min(cols - col0, kSmallCols) + 63) / 64;       // of 64 columns, here
  const uint32_t sx = smem_u32(smem), sa = sx + 2 * kSmallX;
  uint64_t* bar = reinterpret_cast<uint64_t*>(smem + 2 * kSmallX + 2 * kSmallA);
  uint32_t* tslot = reinterpret_cast<uint32_t*>(bar + 1);
  float4* box = reinterpret_cast<float4*>(bar + 4);
  float* diagonal = reinterpret_cast<float*>(box + 16);        // of C
  if (t == 0) {
    mbar_init(bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(tslot)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tslot;
  pdl_trigger();                     // this block holds its tensor memory
  pdl_wait();
  Waits wait(&g_err);

  // U: units of eight columns of a row, or (transposed, lanes along the columns)
  // of eight rows of a column; a thread's units stay in its registers until the
  // norm, over all columns, is known
  const int units = kSmallUnits / 4 * blocks, line = m.transposed ? 64 * blocks : 8 * blocks;
  float u[kSmallUnits][8];
  if (m.vec_in && !m.mom && m.cols % 8 == 0) {
    Raw8<T> raw[kSmallUnits];
#pragma unroll
    for (int i = 0; i < kSmallUnits; ++i) {
      const int e = t + kSmallThreads * i, hi = e / line, lo = e - hi * line;
      const int r = m.transposed ? col0 + lo : hi, c = m.transposed ? 8 * hi : col0 + 8 * lo;
      raw[i].zero();
      if (i < units && r < m.rows && c < m.cols) raw[i].load(static_cast<const T*>(m.g) + r * m.ldg + c);
    }
#pragma unroll
    for (int i = 0; i < kSmallUnits; ++i) raw[i].get(u[i]);
  } else {
#pragma unroll
    for (int i = 0; i < kSmallUnits; ++i) {
      const int e = t + kSmallThreads * i, hi = e / line, lo = e - hi * line;
      if (i < units) update8<T, true>(p, m, m.transposed ? col0 + lo : hi, m.transposed ? 8 * hi : col0 + 8 * lo, u[i]);
      else
#pragma unroll
        for (int k = 0; k < 8; ++k) u[i][k] = 0.f;
    }
  }
  // the sum of squares in units of the block's largest exponent
  float top = 0.f, sum2 = 0.f;
#pragma unroll
  for (int i = 0; i < kSmallUnits; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) top = fmaxf(top, fabsf(u[i][k]));
  top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));
  if (lane == 0) box[warp].x = top;
  __syncthreads();
  for (int w = 0; w < kSmallThreads / 32; ++w) top = fmaxf(top, box[w].x);
  const int exponent = min(max(int(__float_as_uint(top) >> 23), 1), 253);
  const float down = __uint_as_float(uint32_t(254 - exponent) << 23);
#pragma unroll
  for (int i = 0; i < kSmallUnits; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) sum2 = fmaf(u[i][k] * down, u[i][k] * down, sum2);
  sum2 = warp_sum(sum2);
  if (lane == 0) box[warp].y = sum2;
  __syncthreads();
  sum2 = 0.f;
  for (int w = 0; w < kSmallThreads / 32; ++w) sum2 += box[w].y;
  int unit = exponent - 127;
  if (ctas > 1) {
    float2* all = reinterpret_cast<float2*>(p.ws + m.a);
    if (t == 0) __stcg(all + me, make_float2(sum2, float(unit)));
    cluster_sync_all();
    float2 part[kSmallCtas];
#pragma unroll
    for (int i = 0; i < kSmallCtas; ++i) part[i] = i < ctas ? __ldcg(all + i) : make_float2(0.f, -1000.f);
    float most = part[0].y;
#pragma unroll
    for (int i = 1; i < kSmallCtas; ++i) most = fmaxf(most, part[i].y);
    sum2 = 0.f;
#pragma unroll
    for (int i = 0; i < kSmallCtas; ++i) sum2 += scalbnf(part[i].x, 2 * int(part[i].y - most));
    unit = int(most);
  }
  const float2 scale = factors(sqrtf(sum2), unit, p.eps);
#pragma unroll
  for (int i = 0; i < kSmallUnits; ++i) {
    if (i >= units) break;
    const int e = t + kSmallThreads * i, hi = e / line, lo = e - hi * line;
#pragma unroll
    for (int k = 0; k < 8; ++k) u[i][k] = u[i][k] * scale.x * scale.y;
    if (!m.transposed) {
      const uint32_t at = sx + (lo / 8) * 2 * kBlock + hi * 128 + ((lo % 8) ^ (hi & 7)) * 16;
      uint4 w = take_half8<0>(u[i]);
      st_shared4(at, w.x, w.y, w.z, w.w);
      w = take_half8<1>(u[i]);
      st_shared4(at + kSmallX, w.x, w.y, w.z, w.w);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const __half h = __float2half_rn(u[i][k]), l = __float2half_rn((u[i][k] - __half2float(h)) * kUpLow);
        char* at = smem + (lo / 64) * 2 * kBlock + (8 * hi + k) * 128 + ((lo % 64 / 8) ^ k) * 16 + lo % 8 * 2;
        *reinterpret_cast<__half*>(at) = h;
        *reinterpret_cast<__half*>(at + kSmallX) = l;
      }
    }
  }

  // products: [128 x 64] . [N x 64] or . [64 x N] of one block of terms, the small ones first
  constexpr uint32_t id = (1u << 4) | (128u >> 4) << 24;
  auto product = [&](uint32_t d, uint32_t a, uint32_t a_part, uint32_t b, uint32_t b_part, int n, bool flip) {
    constexpr uint32_t hi = (1024u >> 4) | (1u << 14) | (2u << 29);      // stride 1024, version 1, 128-byte swizzle
    const uint32_t idesc = id | uint32_t(n >> 3) << 17 | uint32_t(flip) << 16, bs = flip ? 2048u : 32u;
    const uint32_t bl = (flip ? uint32_t(2 * kBlock) : 16u) >> 4 << 16;
    auto desc = [&](uint32_t at, uint32_t lbo) { return uint64_t((at & 0x3ffff) >> 4 | lbo) | uint64_t(hi) << 32; };
    if (PARTS == 2) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        mma_ss(d, desc(a + 32 * k, 1u << 16), desc(b + b_part + bs * k, bl), idesc, k > 0 ? 1u : 0u);
        mma_ss(d, desc(a + a_part + 32 * k, 1u << 16), desc(b + bs * k, bl), idesc, 1u);
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (PARTS == 2 && k == 0) mma_onto_low<1>(d, desc(a, 1u << 16), desc(b, bl), idesc);
      else mma_ss(d, desc(a + 32 * k, 1u << 16), desc(b + bs * k, bl), idesc, k > 0 ? 1u : 0u);
    }
  };
  uint32_t phase = 0;
  auto begin = [&] {                 // what the warps wrote is there for the products
    fence_proxy_async_smem();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
  };
  auto finished = [&] {
    wait.on_lanes(bar, phase, 68);
    phase ^= 1;
    tc_fence_after();
  };
  // warp: 32 rows and 32 columns of A and C, and 64 columns of X
  const int q = warp % 4, quarter = warp / 4, row = 32 * q + lane;
  const uint32_t lanes = tmem + (uint32_t(32 * q) << 16);
  const uint32_t a_block = sa + quarter / 2 * 2 * kBlock;       // a block column's 128 rows lie behind one another
  float v[32];
  auto sum = [&](uint32_t from, int n, uint32_t step_cols) {
#pragma unroll
    for (int e = 0; e < 32; ++e) v[e] = 0.f;
    for (int c = 0; c < n; ++c) {
      uint32_t r[32];
      tmem_ld32(from + step_cols * c, r);
#pragma unroll
      for (int e = 0; e < 32; ++e) v[e] += __uint_as_float(r[e]);
    }
  };
  for (int step = 0; step < steps; ++step) {
    begin();
    if (warp == 0) {
      for (int c = 0; c < blocks; ++c) {
        const uint32_t x = sx + c * 2 * kBlock;
        product(tmem + 128 * c, x, kSmallX, x, kSmallX, 128, false);
      }
      commit_to(bar);
    }
    finished();
    sum(lanes + 32 * quarter, blocks, 128);
    if (ctas > 1) {
      // [step parity][CTA][8][thread] of four
      float4* parts = reinterpret_cast<float4*>(p.ws + m.x[step & 1]);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        __stcg(parts + (me * 8 + k) * kSmallThreads + t, make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]));
      cluster_sync_all();
#pragma unroll
      for (int e = 0; e < 32; ++e) v[e] = 0.f;
      for (int i = 0; i < ctas; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float4 z = __ldcg(parts + (i * 8 + k) * kSmallThreads + t);
          v[4 * k] += z.x;
          v[4 * k + 1] += z.y;
          v[4 * k + 2] += z.z;
          v[4 * k + 3] += z.w;
        }
    }
    float A[32];
#pragma unroll
    for (int e = 0; e < 32; ++e) A[e] = v[e] *= kUpA / (kUpX * kUpX);
    put_row<PARTS>(a_block, kSmallA, row, quarter % 2 * 4, v);
    // b A of the rounded A, as A A has it: near a singular value of 1 the two
    // errors cancel (b + 2 c = -0.7)
#pragma unroll
    for (int e = 0; e < 32; ++e) A[e] -= v[e];
    begin();
    if (warp == 0) {
      for (int c = 0; c < 2; ++c) product(tmem + 128 * c, sa + c * 2 * kBlock, kSmallA, sa + c * 2 * kBlock, kSmallA, 128, false);
      commit_to(bar);
    }
    finished();
    sum(lanes + 32 * quarter, 2, 128);
#pragma unroll
    for (int e = 0; e < 32; ++e) v[e] = fmaf(p.cc / kUpA, v[e], p.cb * A[e]);
    if (PARTS == 1 && q == quarter) {         // the diagonal goes its own way
      float own = 0.f;
      const uint32_t bit = 1u << lane;        // a mask, not an index, which would move v to memory
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        const bool here = bit >> e & 1u;
        own += here ? v[e] : 0.f;
        v[e] = here ? 0.f : v[e];
      }
      diagonal[row] = own;
    }
    put_row<PARTS>(a_block, kSmallA, row, quarter % 2 * 4, v);
    begin();
    if (warp == 0) {
      for (int c = 0; c < 2; ++c)
        product(tmem + 256 * c, sa + c * 2 * kBlock, kSmallA, sx + c * kBlock, kSmallX, 64 * blocks, true);
      commit_to(bar);
    }
    finished();
    if (quarter < blocks) {
      const float linear = PARTS == 2 ? p.ca : fmaf(1.f / kUpA, diagonal[row], p.ca);
      const uint32_t x_block = sx + quarter * 2 * kBlock;
#pragma unroll 1
      for (int h = 0; h < 2; ++h) {
        sum(lanes + 64 * quarter + 32 * h, 2, 256);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t at = x_block + row * 128 + ((4 * h + k) ^ (row & 7)) * 16;
          const float4 hi = ld_shared4(at), lo = ld_shared4(at + kSmallX);
          const float zh[4] = {hi.x, hi.y, hi.z, hi.w}, zl[4] = {lo.x, lo.y, lo.z, lo.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 fh = of_pair(__float_as_uint(zh[e])), fl = of_pair(__float_as_uint(zl[e]));
            float &x = v[8 * k + 2 * e], &y = v[8 * k + 2 * e + 1];
            x = fmaf(linear, fh.x, fmaf(linear * kDownLow, fl.x, x * (1.f / kUpA)));
            y = fmaf(linear, fh.y, fmaf(linear * kDownLow, fl.y, y * (1.f / kUpA)));
          }
        }
        if (step + 1 < steps) put_row<2>(x_block, kSmallX, row, 4 * h, v);
        else deliver<T>(p, m, 0, col0 + 64 * quarter + 32 * h, q, lane, sa + warp * 4096, v);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// ---------------------------------------------------------------------- host
int bad(const std::string& why) { return report_error(FO_ERR_ARG, "orthogonalize: " + why); }
int done(cudaError_t e) { return e == cudaSuccess ? FO_OK : report_error(FO_ERR_CUDA, cudaGetErrorString(e)); }

int check_items(const fo_matrix_update* m, int count, int dtype) {
  if (dtype != FO_DTYPE_F32 && dtype != FO_DTYPE_BF16) return bad("unknown dtype");
  if (count < 0 || (count > 0 && !m)) return bad("bad count of matrices");
  for (int i = 0; i < count; ++i) {
    const int64_t lo = m[i].rows < m[i].cols ? m[i].rows : m[i].cols, hi = m[i].rows < m[i].cols ? m[i].cols : m[i].rows;
    if (lo < 0 || lo > 32768 || hi > int64_t(1) << 20) return bad("sides of 0 to 32768 and 2^20");
  }
  return FO_OK;
}
// How many pairs share one of A's sums at most (clusters of eight CTAs), and what
// all but the first of them leave.
constexpr int kMaxShares = 4;
int64_t tiles_of(int64_t mt) { return (mt + 1) / 2 * ((mt + 1) / 2 + 1); }
int most_shares(int64_t mt) { return tiles_of(mt) <= 38 ? kMaxShares : 1; }
int64_t shared_bytes(int64_t mt) { return tiles_of(mt) * (most_shares(mt) - 1) * 16 * 8192; }

// Matrices are worked on at the same time, and a gradient is read twice, around
// the momentum's update: every written address is there once, and no gradient
// but its own matrix's out is one.
bool apart(const fo_matrix_update* items, int count) {
  std::vector<const void*> written;
  written.reserve(size_t(count) * 3);
  auto there = [](const fo_matrix_update& m) { return m.rows > 0 && m.cols > 0; };
  for (int i = 0; i < count; ++i)
    if (there(items[i]))
      for (const void* w : {static_cast<const void*>(items[i].out), static_cast<const void*>(items[i].momentum),
                            static_cast<const void*>(items[i].param)})
        if (w) written.push_back(w);
  std::sort(written.begin(), written.end(), std::less<const void*>());
  if (std::adjacent_find(written.begin(), written.end()) != written.end()) return false;
  for (int i = 0; i < count; ++i)
    if (there(items[i]) && items[i].grad != items[i].out &&
        std::binary_search(written.begin(), written.end(), items[i].grad, std::less<const void*>()))
      return false;
  return true;
}

bool is_small(const fo_matrix_update& m) {
  const int64_t lo = m.rows < m.cols ? m.rows : m.cols, hi = m.rows < m.cols ? m.cols : m.rows;
  return lo <= kSmallRows && hi <= kSmallCols * kSmallCtas;
}
// Operands are pairs where X goes anywhere in fp32: the roundings of single ones are
// small only beside a result's in bf16 (1e-3 and 1.7e-3; 512 x 768 8e-4 of an update
// of parameters, with pairs 1e-6).  And where a side has up to 16 elements, whose few
// roundings do not even out: results were off by up to 1.7 times as much as their own
// rounding, from 17 on by 1.25 times (20 x 20 22 us, in pairs 33).
constexpr int kFew = 16;
bool in_pairs(const fo_matrix_update& m, int dtype) {
  return dtype == FO_DTYPE_F32 || m.param || m.rows <= kFew || m.cols <= kFew;
}
// Small matrices: parts of X X^T of even and odd steps, and of the norm.
int64_t item_bytes(const fo_matrix_update& m, int dtype) {
  if (m.rows == 0 || m.cols == 0) return 0;
  const int parts = in_pairs(m, dtype) ? 2 : 1;
  if (is_small(m)) return 2 * kSmallCtas * kSmallPart + 256;
  const int64_t r = (m.rows + 127) / 128, c = (m.cols + 127) / 128, mt = r < c ? r : c, nt = r < c ? c : r;
  return (2 * mt * nt * 2 + 2 * mt * mt * parts) * 4 * kBlock + shared_bytes(mt) + mt * 512 + kMaxSums * 16 + 16;
}

template <int PARTS, int BN, int PHASE, typename T>
cudaError_t launch_product(const OrthoParams& p, int pairs, cudaStream_t st) {
  auto k = ortho_product_k<PARTS, BN, PHASE, T>;
  static std::atomic<bool> allowed[kMaxDevices];
  const cudaError_t e = allow_smem(k, allowed);
  if (e != cudaSuccess) return e;
  const int units = p.start[p.count];
  return launch_k(k, dim3(2 * unsigned(std::min(units, pairs))), dim3(kThreads), Tiles<PARTS, BN>::kSmem, st, p);
}
template <int PARTS, typename T>
cudaError_t launch_shared(const OrthoParams& p, int shares, cudaStream_t st) {
  auto k = ortho_shared_k<PARTS, T>;
  static std::atomic<bool> allowed[kMaxDevices];
  const cudaError_t e = allow_smem(k, allowed);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * unsigned(shares * p.start[p.count]));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Tiles<PARTS, 128>::kSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = unsigned(2 * shares);
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl_enabled() ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, k, p, shares);
}

// Units of each matrix, those with the longest sums first.
template <int PHASE, int BN>
int64_t plan(OrthoParams& p) {
  auto length = [&p](int i) { return PHASE == kGram ? p.item[i].nt : p.item[i].mt; };
  for (int i = 0; i < p.count; ++i) {
    int at = i;
    for (; at > 0 && length(p.order[at - 1]) < length(i); --at) p.order[at] = p.order[at - 1];
    p.order[at] = uint8_t(i);
  }
  int64_t units = 0;
  for (int i = 0; i < p.count; ++i) {
    p.start[i] = int(units);
    const Item& m = p.item[p.order[i]];
    const int64_t h = (m.mt + 1) / 2;
    if (PHASE == kApply) units += h * (BN == 256 ? (m.nt + 1) / 2 : m.nt);
    else units += h * (h + 1) / 2 * (256 / BN);
  }
  p.start[p.count] = int(units);
  return units;
}

template <int PARTS, int PHASE, typename T>
cudaError_t product(OrthoParams& p, int pairs, cudaStream_t st) {
  // Wide tiles load fewer bytes per product and take 1.7 times as long as narrow
  // ones; narrow ones divide the work into twice as many.  Operands in pairs, whose
  // products are three, load few enough with narrow ones, and a wide tile's sums
  // would not fit into the registers.
  if constexpr (PARTS == 1) {
    const int64_t wide = plan<PHASE, 256>(p), narrow = plan<PHASE, 128>(p);
    if (17 * ((wide + pairs - 1) / pairs) <= 10 * ((narrow + pairs - 1) / pairs)) {
      plan<PHASE, 256>(p);
      return launch_product<PARTS, 256, PHASE, T>(p, pairs, st);
    }
  } else {
    plan<PHASE, 128>(p);
  }
  // A sum of X X^T has the larger side's terms, and few tiles where the smaller side
  // is short: pairs that would have no tile take a part of them, as long as a part
  // is not shorter than 8 blocks of 64 (512 x 2048 fp32: 240 -> 190 us).
  if constexpr (PHASE == kGram) {
    const int64_t units = p.start[p.count];
    int longest = 0, shares = 1;
    bool room = true;
    for (int i = 0; i < p.count; ++i) {
      longest = std::max(longest, 2 * p.item[i].nt);
      room = room && most_shares(p.item[i].mt) == kMaxShares;
    }
    while (room && shares < kMaxShares && 2 * shares * units <= pairs && longest / (2 * shares) >= 8) shares *= 2;
    if (shares > 1) return launch_shared<PARTS, T>(p, shares, st);
  }
  return launch_product<PARTS, 128, PHASE, T>(p, pairs, st);
}

template <int PARTS, typename T>
cudaError_t orthogonalize_small(const OrthoParams& p, int steps, cudaStream_t st) {
  auto k = ortho_small_k<PARTS, T>;
  static std::atomic<bool> allowed[kMaxDevices];
  const cudaError_t e = allow_smem(k, allowed);
  if (e != cudaSuccess) return e;
  return launch_k(k, dim3(kSmallCtas * unsigned(p.count)), dim3(kSmallThreads), kSmallSmem, st, p, steps);
}
template <int PARTS, typename T>
cudaError_t orthogonalize(OrthoParams& p, int steps, cudaStream_t st) {
  int dev = 0, sms = 1;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  const int pairs = sms > 1 ? sms / 2 : 1;
  int64_t units = 0;
  for (int i = 0; i < p.count; ++i) {
    p.start[i] = int(units);
    units += p.item[i].nsums;
  }
  p.start[p.count] = int(units);
  if ((e = launch_k(ortho_sums_k<T>, dim3(unsigned(units)), dim3(256), 0, st, p)) != cudaSuccess) return e;
  if ((e = launch_k(ortho_scale_k, dim3(unsigned(p.count)), dim3(256), 0, st, p)) != cudaSuccess) return e;
  units = 0;
  for (int i = 0; i < p.count; ++i) {
    p.start[i] = int(units);
    units += 4 * int64_t(p.item[i].mt) * p.item[i].nt;
  }
  p.start[p.count] = int(units);
  if ((e = launch_k(ortho_pack_k<T>, dim3(unsigned(units)), dim3(256), 0, st, p)) != cudaSuccess) return e;
  for (int s = 0; s < steps; ++s) {
    p.from = s & 1;
    p.last = s + 1 == steps;
    if ((e = product<PARTS, kGram, T>(p, pairs, st)) != cudaSuccess) return e;
    if ((e = product<PARTS, kPoly, T>(p, pairs, st)) != cudaSuccess) return e;
    if ((e = product<PARTS, kApply, T>(p, pairs, st)) != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace
}  // namespace fo

using namespace fo;

extern "C" {

int64_t fo_orthogonalize_workspace(const fo_matrix_update* items, int count, int dtype) {
  if (check_items(items, count, dtype)) return -1;
  int64_t most = 0;
  for (int i = 0; i < count; i += kItems) {
    int64_t sum = 0;
    for (int k = i; k < count && k < i + kItems; ++k) sum += item_bytes(items[k], dtype);
    if (sum > most) most = sum;
  }
  return most;
}

int fo_orthogonalize(const fo_matrix_update* items, int count, int dtype, int steps, const double* coefficients, double eps,
                     double momentum, int nesterov, double decay, void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check_items(items, count, dtype);
  if (rc) return rc;
  if (steps < 1 || steps > 64) return bad("1 to 64 steps");
  if (!coefficients) return bad("no coefficients");
  for (int i = 0; i < 3; ++i)
    if (!(std::fabs(coefficients[i]) <= 64.0)) return bad("coefficients within +-64");
  if (!(eps >= 1e-30 && eps <= 1e30)) return bad("eps of 1e-30 to 1e30");
  if (!(momentum >= 0.0 && momentum <= 1.0) || !(std::fabs(decay) <= 1e30)) return bad("bad momentum or decay");
  const size_t size = dtype == FO_DTYPE_F32 ? 4 : 2;
  auto odd = [](const void* q, size_t n) { return reinterpret_cast<uintptr_t>(q) % n != 0; };
  for (int i = 0; i < count; ++i) {
    const fo_matrix_update& m = items[i];
    if (m.rows == 0 || m.cols == 0) continue;
    if (!m.grad || odd(m.grad, size) || odd(m.out, size) || odd(m.momentum, 4) || odd(m.param, 4))
      return bad("null or misaligned pointer");
    if (!m.out && !m.param) return bad("neither out nor param is wanted");
    if (m.rows > 1 && (m.grad_stride < 0 || (m.out && m.out_stride < m.cols) || (m.momentum && m.momentum_stride < m.cols) ||
                       (m.param && m.param_stride < m.cols)))
      return bad("bad row stride");
    if (!(std::fabs(m.step) <= 1e30f)) return bad("bad step");
  }
  try {
    if (!apart(items, count)) return bad("a tensor to write stands twice in the list, or is another's gradient");
  } catch (const std::bad_alloc&) {
    return report_error(FO_ERR_OOM, "orthogonalize: no host memory");
  }
  const int64_t need = fo_orthogonalize_workspace(items, count, dtype);
  if (need > 0 && (!workspace || odd(workspace, 256) || workspace_bytes < need))
    return bad("the workspace is missing, misaligned or too small");
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  for (int first = 0; first < count; first += kItems)
   for (const bool small : {true, false})
    for (const bool pairs : {true, false}) {
    OrthoParams p = {};
    p.ws = static_cast<char*>(workspace);
    p.ca = float(coefficients[0]);
    p.cb = float(coefficients[1]);
    p.cc = float(coefficients[2]);
    p.mu = float(momentum);
    p.decay = float(decay);
    p.nesterov = nesterov != 0;
    p.eps = float(eps);
    int64_t at = 0;
    auto take = [&at](int64_t bytes) {
      const int64_t here = at;
      at += bytes;
      return here;
    };
    for (int i = first; i < count && i < first + kItems; ++i) {
      const fo_matrix_update& m = items[i];
      if (m.rows == 0 || m.cols == 0 || is_small(m) != small || in_pairs(m, dtype) != pairs) continue;
      Item& it = p.item[p.count++];
      it.g = m.grad;
      it.mom = m.momentum;
      it.param = m.param;
      it.out = m.out;
      it.ldg = m.grad_stride;
      it.ldm = m.momentum_stride;
      it.ldp = m.param_stride;
      it.ldo = m.out_stride;
      it.rows = int(m.rows);
      it.cols = int(m.cols);
      it.transposed = m.rows > m.cols;
      const int64_t r = (m.rows + 127) / 128, c = (m.cols + 127) / 128;
      it.mt = int(r < c ? r : c);
      it.nt = int(r < c ? c : r);
      if (small) {
        for (int k = 0; k < 2; ++k) it.x[k] = take(kSmallCtas * kSmallPart);
        it.a = take(256);
      } else {
        for (int k = 0; k < 2; ++k) it.x[k] = take(int64_t(it.mt) * it.nt * 4 * kBlock * 2);
        it.a = take(int64_t(it.mt) * it.mt * 4 * kBlock * (pairs ? 2 : 1));
        it.c = take(int64_t(it.mt) * it.mt * 4 * kBlock * (pairs ? 2 : 1));
        it.parts = take(shared_bytes(it.mt));
        it.d = take(int64_t(it.mt) * 512);
      }
      const int64_t per = dtype == FO_DTYPE_F32 ? 4 : 8;
      it.vec_in = aligned16(m.grad) && (m.rows == 1 || m.grad_stride % per == 0) &&
                  (!m.momentum || (aligned16(m.momentum) && (m.rows == 1 || m.momentum_stride % 4 == 0)));
      it.vec_out = aligned16(m.out) && (m.rows == 1 || m.out_stride % per == 0);
      const int64_t sums = (m.rows * ((m.cols + 7) / 8) + 1023) / 1024;       // four groups of eight per thread
      it.nsums = int(sums < kMaxSums ? sums : kMaxSums);
      it.step = m.step;
    }
    if (p.count == 0) continue;
    p.sums = reinterpret_cast<float4*>(p.ws + at);
    p.scale = reinterpret_cast<float2*>(p.sums + p.count * kMaxSums);
    const cudaError_t e =
        dtype == FO_DTYPE_F32 ? (small ? orthogonalize_small<2, float>(p, steps, st) : orthogonalize<2, float>(p, steps, st))
        : pairs               ? (small ? orthogonalize_small<2, bf16>(p, steps, st) : orthogonalize<2, bf16>(p, steps, st))
                              : (small ? orthogonalize_small<1, bf16>(p, steps, st) : orthogonalize<1, bf16>(p, steps, st));
    if (e != cudaSuccess) return done(e);
  }
  return FO_OK;
}

int fo_orthogonalize_error(void* stream) {
  static thread_local unsigned told[kMaxDevices];     // what this thread has reported
  int dev = 0, code = 0;
  cudaError_t e = cudaStreamSynchronize(static_cast<cudaStream_t>(stream));
  if (e == cudaSuccess) e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = gave_up_since(g_err, &told[dev % kMaxDevices], &code);
  if (e != cudaSuccess) return done(e);
  return code ? report_error(FO_ERR_TIMEOUT, "orthogonalize: a kernel timed out waiting (code " + std::to_string(code) + ")") : FO_OK;
}

}  // extern "C"
