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
// numbers (22 bits), and a X is added from both: what the roundings of the
// products' operands leave in the weak directions, which each step multiplies by
// up to a, is then proportional to C, which is small there (off by 0.5 to 0.8e-3
// for bf16 matrices instead of 2e-3 with a in the product).  For fp32 matrices
// all operands are such pairs, and each product three (hi lo, lo hi, hi hi, in
// this order; the fourth is below fp32's rounding).  Sums are fp32 in tensor
// memory; because the tensor cores truncate, those of fp32 matrices are moved to
// registers and added there, rounded, every 64 terms (512: 7e-6 off instead of
// 1.5e-6 on matrices of width 512, torch's fp32 products 2.3e-6).
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
#include <string>

namespace fo {
int report_error(int code, const std::string& msg);

namespace {

__device__ GaveUp g_err;

constexpr int kItems = 32;                    // matrices per launch
constexpr int kBlock = 8192;                  // bytes of a 64 x 64 block
constexpr int kMaxSums = 1024;                // partial sums of squares per matrix
constexpr int kMaxShared = 64;                // tiles of A whose sums are shared, per matrix
constexpr float kUpX = 1024.f, kUpA = 256.f;  // what X, and A and C, are multiplied by as fp16

struct Item {
  const void* g;            // [rows][cols] gradient
  float *mom, *param;
  void* out;
  int64_t ldg, ldm, ldp, ldo;
  int64_t x[2], a, c;       // byte offsets in the workspace
  int64_t parts;            // of A's sums that are shared, [tile][split][CTA][warp] of 8 KB
  int rows, cols, mt, nt;   // mt, nt: tiles of 128 of the smaller and the larger side
  int nsums;                // partial sums of squares, at kMaxSums times its index
  int split;                // units that share one of A's sums
  bool transposed, vec_in, vec_out;
  float step;
};
struct OrthoParams {
  Item item[kItems];
  // First unit of work of each matrix: before the steps in start[0], then in each
  // product; the matrices in the order of their units.
  int start[3][kItems + 1];
  uint8_t order[3][kItems];
  char* ws;
  float4* sums;
  float2* scale;            // of each matrix: the two factors that make X of U
  unsigned* done;           // of each matrix: how many of its units' warps are done, over all steps
  unsigned* shared;         // the same of each tile of A whose sums are shared, kMaxShared for each matrix
  int count, steps;
  float ca, cb, cc, mu, decay;
  bool nesterov;
  float eps;
};

__device__ __forceinline__ int slot_of(const OrthoParams& p, int unit, int which = 0) {
  int n = 0;
  while (n + 1 < p.count && unit >= p.start[which][n + 1]) ++n;
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
  const int n = slot_of(p, blockIdx.x), part = int(blockIdx.x) - p.start[0][n];
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
    p.done[n] = 0;
  }
  if (threadIdx.x < kMaxShared) p.shared[n * kMaxShared + threadIdx.x] = 0;
}

__device__ __forceinline__ uint32_t half_pair(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 of_pair(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
// Eight values as fp16; v keeps what they leave.
__device__ __forceinline__ uint4 take_half8(float* v) {
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    w[e] = half_pair(v[2 * e], v[2 * e + 1]);
    const float2 f = of_pair(w[e]);
    v[2 * e] -= f.x;
    v[2 * e + 1] -= f.y;
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
  const int blk = int(blockIdx.x) - p.start[0][n], rows = 2 * it.mt;
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
    *reinterpret_cast<uint4*>(img + at) = take_half8(z);
    *reinterpret_cast<uint4*>(img + image + at) = take_half8(z);
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
  // Of 32 x 64 elements per warp of arithmetic: both parts, or with wide tiles,
  // which want the room for copies in flight, one.
  static constexpr int kBuffer = BN == 256 ? 4096 : 8192, kOut = 8 * kBuffer;
  static constexpr int kStage = PARTS * (kA + kB), kStages = (229376 - kOut) / kStage;
  static constexpr int kSumsAt = 512 / BN;    // tiles' sums in tensor memory
  static constexpr int kBars = 3 * kStages + 2 * kSumsAt + 9;
  static constexpr int kSmem = 1024 + kStages * kStage + kOut + 8 * kBars + 16;
};
static_assert(Tiles<1, 256>::kSmem <= 232448 && Tiles<1, 128>::kSmem <= 232448 && Tiles<2, 128>::kSmem <= 232448, "shared memory per CTA");

struct Place {
  int item, phase, step;
  int i, j, kb;             // rows 256 i, columns BN j, blocks of 64 terms (none: nothing to do)
  int k0, split, tile;      // its first block; which of the units that share a sum; the tile's number
  bool adds;                // it has the last of the shared terms and adds the others' sums, or is alone
  unsigned need;            // warps of this matrix that are done with what this unit reads
};
template <int BN>
__device__ __forceinline__ Place place_of(const OrthoParams& p, int unit) {
  Place a;
  const int n0 = p.start[kGram][p.count], n1 = p.start[kPoly][p.count], n2 = p.start[kApply][p.count];
  a.step = unit / (n0 + n1 + n2);
  int t = unit - a.step * (n0 + n1 + n2);
  a.phase = t < n0 ? kGram : t < n0 + n1 ? kPoly : kApply;
  t -= a.phase == kGram ? 0 : a.phase == kPoly ? n0 : n0 + n1;
  const int n = slot_of(p, t, a.phase);
  a.item = p.order[a.phase][n];
  const Item& it = p.item[a.item];
  t -= p.start[a.phase][n];
  const int h = (it.mt + 1) / 2, cols = a.phase == kApply ? it.nt : it.mt;
  // units that have something to do (an odd last column's second half has not)
  const unsigned triangle = BN == 256 ? h * (h + 1) / 2 : h * (h + 1) - (it.mt & 1 ? h : 0);
  const unsigned all = 2 * triangle + h * ((it.nt + BN / 128 - 1) / (BN / 128));
  a.need = 16 * (a.step * all + a.phase * triangle);
  a.k0 = a.split = 0;
  a.adds = true;
  if (a.phase == kGram) {
    a.split = t % it.split;
    t /= it.split;
    a.adds = a.split + 1 == it.split;
  }
  a.tile = t;
  if (a.phase == kApply) {
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
  a.kb = a.j * (BN / 128) < cols ? 2 * (a.phase == kGram ? it.nt : it.mt) : 0;
  if (a.phase == kGram && it.split > 1) {
    a.k0 = a.kb * a.split / it.split;
    a.kb = a.kb * (a.split + 1) / it.split - a.k0;
  }
  return a;
}
// Before copies of what other blocks have stored: `need` of their warps have said so.
__device__ __forceinline__ void wait_for(Waits& w, const unsigned* done, unsigned need, int code) {
  if (w.dead || need == 0) return;
  const uint64_t t0 = global_ns();
  while (true) {
    for (int i = 0; i < 64; ++i) {
      unsigned now;
      asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(now) : "l"(done) : "memory");
      if (now >= need) {
        asm volatile("fence.proxy.async;" ::: "memory");
        return;
      }
    }
    if (global_ns() - t0 > w.limit) break;
  }
  w.give_up(code);
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
__device__ __forceinline__ void arrive_leader(uint64_t* bar) {
  asm volatile(
      "{\n .reg .b32 r;\n mapa.shared::cluster.u32 r, %0, 0;\n mbarrier.arrive.shared::cluster.b64 _, [r];\n}\n" ::"r"(
          smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.b32 p, %4, 0;\n elect.sync _|q, 0xffffffff;\n"
      " @q tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(acc)
      : "memory");
}
__device__ __forceinline__ void commit_pair(uint64_t* bar) {     // the barrier of both CTAs
  asm volatile(
      "{\n .reg .pred q;\n elect.sync _|q, 0xffffffff;\n"
      " @q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n}\n" ::"r"(smem_u32(bar)),
      "h"(uint16_t(3))
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

// A warp's 32 rows of a block of A, C or X: 4 KB per part, in the block's order.
__device__ __forceinline__ int64_t rows_at(const Item& m, int tile, int cblk, int q) {
  return (int64_t(cblk) * 2 * m.mt + 2 * tile + q / 2) * kBlock + (q & 1) * 4096;
}
// What the sums of these rows are added to (A or X) is on its way into the warp's
// buffer while the products run.
template <int PARTS, int BN, int PHASE>
__device__ __forceinline__ void fetch(const OrthoParams& p, const Item& m, int step, int tile, int cblk, int q, int lane, char* buf, uint64_t* bar) {
  if (BN == 256 || PHASE == kGram || lane != 0) return;
  const char* src = p.ws + (PHASE == kPoly ? m.a : m.x[step & 1]) + rows_at(m, tile, cblk, q);
  constexpr int kParts = PHASE == kPoly ? PARTS : 2;
  bulk_wait_read<0>();                // the last stores have read the buffer
  mbar_expect_tx(bar, kParts * 4096);
#pragma unroll
  for (int part = 0; part < kParts; ++part)
    bulk_g2s(buf + part * 4096, src + part * (int64_t(m.mt) * (PHASE == kPoly ? m.mt : m.nt) * 4 * kBlock), 4096, bar);
}

// One of the units that share a tile's sums leaves its own in the workspace, and
// the last adds the others' in their order: 32 columns at a time of the warp's 32
// rows (4 KB), every lane its own.
__device__ __forceinline__ char* shared_at(const OrthoParams& p, const Item& m, const Place& a, int split, int me, int warp) {
  return p.ws + m.parts + (((int64_t(a.tile) * (m.split - 1) + split) * 2 + me) * 8 + warp) * 8192;
}
__device__ __forceinline__ void leave_sums(const OrthoParams& p, const Item& m, const Place& a, int me, int warp, int lane, char* buf, float (&v)[64]) {
  const uint32_t mine = smem_u32(buf) + lane * 16;
  char* dst = shared_at(p, m, a, a.split, me, warp);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (lane == 0) bulk_wait_read<0>();
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 8; ++k)
      st_shared4(mine + k * 512, __float_as_uint(v[32 * h + 4 * k]), __float_as_uint(v[32 * h + 4 * k + 1]), __float_as_uint(v[32 * h + 4 * k + 2]),
                 __float_as_uint(v[32 * h + 4 * k + 3]));
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], 4096;" ::"l"(dst + h * 4096), "r"(smem_u32(buf)) : "memory");
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
  }
}
__device__ __forceinline__ void add_sums(const OrthoParams& p, const Item& m, const Place& a, int me, int warp, int lane, float (&v)[64]) {
  float own[64];
#pragma unroll
  for (int e = 0; e < 64; ++e) own[e] = 0.f;
  for (int s = 0; s + 1 < m.split; ++s) {
    const float4* src = reinterpret_cast<const float4*>(shared_at(p, m, a, s, me, warp)) + lane;
    float4 w[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) w[k] = __ldcg(src + 32 * k);
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      own[4 * k] += w[k].x;
      own[4 * k + 1] += w[k].y;
      own[4 * k + 2] += w[k].z;
      own[4 * k + 3] += w[k].w;
    }
  }
#pragma unroll
  for (int e = 0; e < 64; ++e) v[e] += own[e];
}

// 64 sums of one row, columns 64 cblk .., become elements of A, C or X.
template <int PARTS, int BN, int PHASE, typename T>
__device__ __forceinline__ void finish(const OrthoParams& p, const Item& m, int step, int tile, int cblk, int q, int lane, char* buf_ptr, uint64_t* bar,
                                       uint32_t& phase, Waits& wait, float (&v)[64]) {
  const uint32_t buf = smem_u32(buf_ptr), mine = buf + lane * 128;       // a lane reads and writes its own row
  if (PHASE == kGram) {
#pragma unroll
    for (int e = 0; e < 64; ++e) v[e] *= kUpA / (kUpX * kUpX);
    if (lane == 0) bulk_wait_read<0>();       // the last stores have read the buffer
    __syncwarp();
  } else {
    // C = b A + c A A, or a X + C X
    const float linear = PHASE == kPoly ? p.cb : p.ca, other = (PHASE == kPoly ? p.cc : 1.f) / kUpA;
    constexpr int kParts = PHASE == kPoly ? PARTS : 2;
    uint4 w[BN == 256 ? kParts : 1][8];
    if (BN == 256) {          // the warp's 4 KB are read as they lie, past L1, which may hold an older step's
      const uint4* src = reinterpret_cast<const uint4*>(p.ws + (PHASE == kPoly ? m.a : m.x[step & 1]) + rows_at(m, tile, cblk, q)) + lane;
#pragma unroll
      for (int part = 0; part < kParts; ++part)
#pragma unroll
        for (int k = 0; k < 8; ++k) w[part][k] = __ldcg(src + part * (int64_t(m.mt) * (PHASE == kPoly ? m.mt : m.nt) * 4 * kBlock / 16) + 32 * k);
      if (lane == 0) bulk_wait_read<0>();       // the last stores have read the buffer
    } else {
      wait.on_lanes(bar, phase, 69);
      phase ^= 1;
    }
#pragma unroll
    for (int part = kParts - 1; part >= 0; --part) {
      if (BN == 256) {        // and handed out by rows
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 8; ++k)
          st_shared4(buf + (32 * k + lane) * 16, w[BN == 256 ? part : 0][k].x, w[BN == 256 ? part : 0][k].y, w[BN == 256 ? part : 0][k].z,
                     w[BN == 256 ? part : 0][k].w);
        __syncwarp();
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float4 u = ld_shared4(mine + (BN == 256 ? 0 : part * 4096) + (k ^ (lane & 7)) * 16);
        const float z[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 f = of_pair(__float_as_uint(z[e]));
          float &x = v[8 * k + 2 * e], &y = v[8 * k + 2 * e + 1];
          x = fmaf(linear, f.x, part == kParts - 1 ? x * other : x);
          y = fmaf(linear, f.y, part == kParts - 1 ? y * other : y);
        }
      }
    }
    if (BN == 256) __syncwarp();
  }
  if (PHASE == kApply && step + 1 == p.steps) {
    deliver<T>(p, m, tile, 64 * cblk, q, lane, buf, v);
    deliver<T>(p, m, tile, 64 * cblk + 32, q, lane, buf, v + 32);
    fence_proxy_async_smem();                 // before the next copy into the buffer
    __syncwarp();
    return;
  }
  constexpr int kParts = PHASE == kApply ? 2 : PARTS;
  char* dst = p.ws + (PHASE == kGram ? m.a : PHASE == kPoly ? m.c : m.x[step & 1 ^ 1]) + rows_at(m, tile, cblk, q);
#pragma unroll
  for (int part = 0; part < kParts; ++part) {
    const uint32_t at = BN == 256 ? 0 : part * 4096;
    if (BN == 256 && part > 0) {
      if (lane == 0) bulk_wait_read<0>();
      __syncwarp();
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint4 w = take_half8(v + 8 * k);
      st_shared4(mine + at + (k ^ (lane & 7)) * 16, w.x, w.y, w.z, w.w);
    }
    if (BN == 256 || part + 1 == kParts) {
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
#pragma unroll
        for (int o = BN == 256 ? part : 0; o <= part; ++o)
          asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], 4096;" ::"l"(
                           dst + o * (int64_t(m.mt) * (PHASE == kApply ? m.nt : m.mt) * 4 * kBlock)),
                       "r"(buf + (BN == 256 ? 0 : o * 4096))
                       : "memory");
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
      }
    }
  }
}

// All steps of all matrices in one launch.  Units of work (a tile of one of the
// three products of a step of a matrix) have an order, and pairs take them in
// turn; a unit's copies start when the units of the matrix before it are done,
// which every warp that has stored its part says in the matrix's counter.  So
// the products of one matrix fill the gaps of another's, and between two products
// of one lie 2 us instead of a launch's 7 (its blocks fill an SM's shared memory,
// so they cannot start while the last launch's run).  Units wait for earlier ones
// only and all blocks run at the same time (a cooperative launch).
template <int PARTS, int BN, typename T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) ortho_steps_k(const __grid_constant__ OrthoParams p) {
  using S = Tiles<PARTS, BN>;
  extern __shared__ char smem_raw[];
  char* smem = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  char* stage_out = smem + S::kStages * S::kStage;
  uint64_t* full = reinterpret_cast<uint64_t*>(stage_out + S::kOut);
  uint64_t *peer = full + S::kStages, *empty = peer + S::kStages, *acc_full = empty + S::kStages, *acc_empty = acc_full + S::kSumsAt,
           *done = acc_empty + S::kSumsAt, *fetched = done + 1;
  uint32_t* tslot = reinterpret_cast<uint32_t*>(fetched + 8);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int units = p.steps * (p.start[kGram][p.count] + p.start[kPoly][p.count] + p.start[kApply][p.count]);
  const int pair = int(blockIdx.x) / 2, pairs = int(gridDim.x) / 2, me = int(blockIdx.x) % 2;

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
    for (int e = 0; e < 8; ++e) mbar_init(&fetched[e], 1);
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
  Waits wait(&g_err);

  if (warp == 0) {
    if (lane == 0) {
      Ring<S::kStages> at;
      int it = 0;
      for (int u = pair; u < units && !wait.dead; u += pairs) {
        const Place a = place_of<BN>(p, u);
        const Item& m = p.item[a.item];
        const char* x = p.ws + m.x[a.step & 1];
        const char* sym = p.ws + (a.phase == kPoly ? m.a : m.c);
        const int64_t xi = int64_t(m.mt) * m.nt * 4 * kBlock, si = int64_t(m.mt) * m.mt * 4 * kBlock;
        const int cols = a.phase == kApply ? m.nt : m.mt;     // tiles of 128
        const int ta = 2 * a.i + me, tb = BN == 256 ? 2 * a.j + me : a.j;
        const bool has_a = ta < m.mt, has_b = tb < cols;
        const uint32_t bytes = PARTS * ((has_a ? S::kA : 0) + (has_b ? S::kB : 0));
        const int64_t wide = int64_t(2 * m.mt) * kBlock;      // from one block column to the next
        if (a.kb) wait_for(wait, p.done + a.item, a.need, 60);
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
              const char* src = a.phase == kGram ? x + q * xi : sym + q * si;
              if (a.phase == kGram || !mirrored(ta, kb)) {
                bulk_g2s(d, src + kb * wide + int64_t(2 * ta) * kBlock, 2 * kBlock, bar);
              } else {
                src += 2 * ta * wide + int64_t(kb) * kBlock;
                bulk_g2s(d, src, kBlock, bar);
                bulk_g2s(d + kBlock, src + wide, kBlock, bar);
              }
            }
            if (has_b) {
              char* d = s + PARTS * S::kA + q * S::kB;
              const char* src = a.phase == kPoly ? sym + q * si : x + q * xi;
              const int b0 = BN == 256 ? 2 * tb : 2 * tb + me;          // this CTA's first block
              if (a.phase == kGram || (a.phase == kPoly && !mirrored(tb, kb))) {
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
        const Place a = place_of<BN>(p, u);
        for (int kb = 0; kb < a.kb; ++kb) {
          wait.on(&full[at.at], at.phase, 65);
          if (wait.dead) break;
          arrive_leader(&peer[at.at]);
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
      const Place a = place_of<BN>(p, u);
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
        const uint32_t am = a.phase != kGram && mirrored(2 * a.i, kb), bm = a.phase == kApply || (a.phase == kPoly && mirrored(tb, kb));
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
        for (int k = 0; k < 4; ++k)
          mma_pair(d, desc(k * as, al), desc(b0 + k * bs, bl), idesc, PARTS == 2 || kb > 0 || k > 0 ? 1u : 0u);
        commit_pair(&empty[at.at]);
        at.step();
        if (PARTS == 2 || kb + 1 == a.kb) {
          commit_pair(&acc_full[sum.at]);
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
    char* buf = stage_out + (warp - 2) * S::kBuffer;
    uint64_t* in = &fetched[warp - 2];
    uint32_t in_phase = 0;
    Ring<S::kSumsAt> sum;
    bool dead = false;
    for (int u = pair; u < units && !dead; u += pairs) {
      const Place a = place_of<BN>(p, u);
      const Item& m = p.item[a.item];
      const int tile = 2 * a.i + me, cblk = a.j * (BN / 64) + half * NB, cols = 2 * (a.phase == kApply ? m.nt : m.mt);
      float v[64];
      auto get = [&](int b) {
        if (a.phase == kPoly) fetch<PARTS, BN, kPoly>(p, m, a.step, tile, cblk + b, q, lane, buf, in);
        else fetch<PARTS, BN, kApply>(p, m, a.step, tile, cblk + b, q, lane, buf, in);
      };
      auto end = [&](int b) {
        if (BN == 128 && a.phase == kGram && m.split > 1) {
          if (!a.adds) {
            leave_sums(p, m, a, me, warp - 2, lane, buf, v);
            return;
          }
          if (lane == 0) wait_for(wait, p.shared + a.item * kMaxShared + a.tile, 16u * (m.split - 1) * (a.step + 1), 70);
          __syncwarp();
          add_sums(p, m, a, me, warp - 2, lane, v);
        }
        if (a.phase == kGram) finish<PARTS, BN, kGram, T>(p, m, a.step, tile, cblk + b, q, lane, buf, in, in_phase, wait, v);
        else if (a.phase == kPoly) finish<PARTS, BN, kPoly, T>(p, m, a.step, tile, cblk + b, q, lane, buf, in, in_phase, wait, v);
        else finish<PARTS, BN, kApply, T>(p, m, a.step, tile, cblk + b, q, lane, buf, in, in_phase, wait, v);
      };
      bool here = a.kb > 0 && tile < m.mt && cblk < cols;        // the first block of columns
      if (PARTS == 2) {
        for (int kb = 0; kb < a.kb; ++kb) {
          wait.on(&acc_full[sum.at], sum.phase, 64);
          __syncwarp();
          tc_fence_after();
          // the first sum tells that what the unit reads is there
          if (kb == 0 && here && a.phase != kGram) get(0);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t r[32];
            tmem_ld32(col + sum.at * BN + 32 * h, r);
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              float& x = v[32 * h + e];
              x = (kb > 0 ? x : 0.f) + __uint_as_float(r[e]);
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_leader(&acc_empty[sum.at]);
          sum.step();
        }
        dead = __any_sync(0xffffffffu, wait.dead);
        if (dead) break;
        static_assert(PARTS == 1 || NB == 1, "one block of columns");
        if (here) end(0);
      } else if (a.kb > 0) {
        wait.on(&acc_full[sum.at], sum.phase, 64);
        __syncwarp();
        tc_fence_after();
        dead = __any_sync(0xffffffffu, wait.dead);
        if (here && a.phase != kGram) get(0);
#pragma unroll 1
        for (int b = 0; b < NB; ++b) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t r[32];
            tmem_ld32(col + sum.at * BN + 64 * b + 32 * h, r);
#pragma unroll
            for (int e = 0; e < 32; ++e) v[32 * h + e] = __uint_as_float(r[e]);
          }
          if (b == NB - 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_leader(&acc_empty[sum.at]);
          }
          if (dead || !here) continue;
          end(b);
          here = b + 1 < NB && cblk + b + 1 < cols;
          if (here && a.phase != kGram) get(b + 1);
        }
        sum.step();
      }
      // this warp's part is stored: units that read it may start
      if (lane == 0 && a.kb > 0 && !(a.phase == kApply && a.step + 1 == p.steps)) {
        bulk_wait_all();
        asm volatile("fence.proxy.async;" ::: "memory");
        unsigned* count = BN == 256 || a.adds ? p.done + a.item : p.shared + a.item * kMaxShared + a.tile;
        asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(count) : "memory");
      }
      __syncwarp();
    }
    if (lane == 0) {
      bulk_wait_all();
      if (BN == 128 && dead) mbar_wait(in, in_phase);         // no copy is on its way into the buffer
    }
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
constexpr int kSmallSmem = 1024 + 2 * kSmallX + 2 * kSmallA + 32 + 16 * 16;
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
      const uint4 w = take_half8(v + 8 * k);
      st_shared4(at + q * part + row * 128 + ((first + k) ^ (row & 7)) * 16, w.x, w.y, w.z, w.w);
    }
}

template <int PARTS, typename T>
__global__ void __cluster_dims__(kSmallCtas, 1, 1) __launch_bounds__(kSmallThreads, 1) ortho_small_k(const __grid_constant__ OrthoParams p) {
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
      uint4 w = take_half8(u[i]);
      st_shared4(at, w.x, w.y, w.z, w.w);
      w = take_half8(u[i]);
      st_shared4(at + kSmallX, w.x, w.y, w.z, w.w);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const __half h = __float2half_rn(u[i][k]), l = __float2half_rn(u[i][k] - __half2float(h));
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
    for (int k = 0; k < 4; ++k)
      mma_ss(d, desc(a + 32 * k, 1u << 16), desc(b + bs * k, bl), idesc, PARTS == 2 || k > 0 ? 1u : 0u);
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
  for (int step = 0; step < p.steps; ++step) {
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
    begin();
    if (warp == 0) {
      for (int c = 0; c < 2; ++c) product(tmem + 128 * c, sa + c * 2 * kBlock, kSmallA, sa + c * 2 * kBlock, kSmallA, 128, false);
      commit_to(bar);
    }
    finished();
    sum(lanes + 32 * quarter, 2, 128);
#pragma unroll
    for (int e = 0; e < 32; ++e) v[e] = fmaf(p.cc / kUpA, v[e], p.cb * A[e]);
    put_row<PARTS>(a_block, kSmallA, row, quarter % 2 * 4, v);
    begin();
    if (warp == 0) {
      for (int c = 0; c < 2; ++c)
        product(tmem + 256 * c, sa + c * 2 * kBlock, kSmallA, sx + c * kBlock, kSmallX, 64 * blocks, true);
      commit_to(bar);
    }
    finished();
    if (quarter < blocks) {
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
            x = fmaf(p.ca, fh.x, fmaf(p.ca, fl.x, x * (1.f / kUpA)));
            y = fmaf(p.ca, fh.y, fmaf(p.ca, fl.y, y * (1.f / kUpA)));
          }
        }
        if (step + 1 < p.steps) put_row<2>(x_block, kSmallX, row, 4 * h, v);
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
// How many units share one of A's sums at most, and what they leave.
constexpr int kMaxSplit = 8;
int64_t tiles_of(int mt) { return int64_t((mt + 1) / 2) * ((mt + 1) / 2 + 1); }
int most_split(int mt, int nt) {
  const int64_t tiles = tiles_of(mt), most = (152 + tiles - 1) / tiles, want = (2 * nt + 7) / 8;
  return tiles > kMaxShared ? 1 : int(std::min<int64_t>(std::min(most, want), kMaxSplit));
}
int64_t shared_bytes(int mt, int nt) { return tiles_of(mt) * (most_split(mt, nt) - 1) * 16 * 8192; }

bool is_small(const fo_matrix_update& m) {
  const int64_t lo = m.rows < m.cols ? m.rows : m.cols, hi = m.rows < m.cols ? m.cols : m.rows;
  return lo <= kSmallRows && hi <= kSmallCols * kSmallCtas;
}
// Small matrices: parts of X X^T of even and odd steps, and of the norm.
int64_t item_bytes(const fo_matrix_update& m, int parts) {
  if (m.rows == 0 || m.cols == 0) return 0;
  if (is_small(m)) return 2 * kSmallCtas * kSmallPart + 256;
  const int64_t r = (m.rows + 127) / 128, c = (m.cols + 127) / 128, mt = r < c ? r : c, nt = r < c ? c : r;
  return (2 * mt * nt * 2 + 2 * mt * mt * parts) * 4 * kBlock + shared_bytes(int(mt), int(nt)) + kMaxSums * 16 + kMaxShared * 4 + 16;
}

// Units of each matrix in one of the products, those with the longest sums first.
template <int PHASE, int BN>
int64_t plan(OrthoParams& p) {
  auto length = [&p](int i) { return PHASE == kGram ? (p.item[i].nt + p.item[i].split - 1) / p.item[i].split : p.item[i].mt; };
  uint8_t* order = p.order[PHASE];
  for (int i = 0; i < p.count; ++i) {
    int at = i;
    for (; at > 0 && length(order[at - 1]) < length(i); --at) order[at] = order[at - 1];
    order[at] = uint8_t(i);
  }
  int64_t units = 0;
  for (int i = 0; i < p.count; ++i) {
    p.start[PHASE][i] = int(units);
    const Item& m = p.item[order[i]];
    const int64_t h = (m.mt + 1) / 2;
    if (PHASE == kApply) units += h * (BN == 256 ? (m.nt + 1) / 2 : m.nt);
    else units += h * (h + 1) / 2 * (256 / BN) * (PHASE == kGram ? m.split : 1);
  }
  p.start[PHASE][p.count] = int(units);
  return units;
}

// How many units share one of A's sums: a sum of X X^T has the larger side's terms,
// and few tiles; shared by units of 8 blocks of 64 terms, or of an equal part of
// all where that is longer, the longest chain of a step is as long as the others
// (2048 x 512: SHARE).
void share_sums(OrthoParams& p) {
  int64_t all = 0;
  for (int i = 0; i < p.count; ++i) all += tiles_of(p.item[i].mt) * 2 * p.item[i].nt;
  const int64_t part = all / 76 > 8 ? all / 76 : 8;
  for (int i = 0; i < p.count; ++i) {
    const int64_t want = (2 * p.item[i].nt + part - 1) / part;
    const int most = most_split(p.item[i].mt, p.item[i].nt);
    p.item[i].split = int(want < most ? want : most);
  }
}

template <int PARTS, int BN, typename T>
cudaError_t launch_steps(OrthoParams& p, int dev, cudaStream_t st) {
  auto k = ortho_steps_k<PARTS, BN, T>;
  static std::atomic<bool> allowed[kMaxDevices];
  static std::atomic<int> resident[kMaxDevices];      // pairs that run at the same time
  cudaError_t e = allow_smem(k, allowed);
  if (e != cudaSuccess) return e;
  // without wide tiles' numbers of units, a long sum's terms are shared
  for (int i = 0; i < p.count; ++i) p.item[i].split = 1;
  if (BN == 128) share_sums(p);
  const int64_t units = plan<kGram, BN>(p) + plan<kPoly, BN>(p) + plan<kApply, BN>(p);
  if (units * p.steps >= int64_t(1) << 31) return cudaErrorInvalidValue;      // sides are limited: not reached
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Tiles<PARTS, BN>::kSmem;
  cfg.stream = st;
  cfg.gridDim = dim3(2);
  int pairs = dev < kMaxDevices ? resident[dev].load() : 0;
  if (pairs == 0) {
    if ((e = cudaOccupancyMaxActiveClusters(&pairs, k, &cfg)) != cudaSuccess) return e;
    if (pairs < 1) return cudaErrorCooperativeLaunchTooLarge;
    if (dev < kMaxDevices) resident[dev].store(pairs);
  }
  cfg.gridDim = dim3(2 * unsigned(units < pairs ? units : pairs));
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeCooperative;
  attr[0].val.cooperative = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k, static_cast<const OrthoParams&>(p));
}

template <typename T>
cudaError_t orthogonalize_small(const OrthoParams& p, cudaStream_t st) {
  auto k = ortho_small_k<sizeof(T) == 4 ? 2 : 1, T>;
  static std::atomic<bool> allowed[kMaxDevices];
  const cudaError_t e = allow_smem(k, allowed);
  if (e != cudaSuccess) return e;
  return launch_k(k, dim3(kSmallCtas * unsigned(p.count)), dim3(kSmallThreads), kSmallSmem, st, p);
}
template <typename T>
cudaError_t orthogonalize(OrthoParams& p, cudaStream_t st) {
  int dev = 0, sms = 1;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  int64_t units = 0;
  for (int i = 0; i < p.count; ++i) {
    p.start[0][i] = int(units);
    units += p.item[i].nsums;
  }
  p.start[0][p.count] = int(units);
  if ((e = launch_k(ortho_sums_k<T>, dim3(unsigned(units)), dim3(256), 0, st, p)) != cudaSuccess) return e;
  if ((e = launch_k(ortho_scale_k, dim3(unsigned(p.count)), dim3(256), 0, st, p)) != cudaSuccess) return e;
  units = 0;
  for (int i = 0; i < p.count; ++i) {
    p.start[0][i] = int(units);
    units += 4 * int64_t(p.item[i].mt) * p.item[i].nt;
  }
  p.start[0][p.count] = int(units);
  if ((e = launch_k(ortho_pack_k<T>, dim3(unsigned(units)), dim3(256), 0, st, p)) != cudaSuccess) return e;
  // Wide tiles load fewer bytes per product and take 1.7 times as long as narrow
  // ones, which divide the work into twice as many: they are taken where a product
  // has fewer than two rounds of wide ones.  fp32 matrices, whose products are
  // three, load few enough with narrow ones, and a wide tile's sums would not fit
  // into the registers.
  if constexpr (sizeof(T) == 2) {
    if (plan<kApply, 256>(p) >= sms) return launch_steps<1, 256, T>(p, dev, st);
    return launch_steps<1, 128, T>(p, dev, st);
  } else {
    return launch_steps<2, 128, T>(p, dev, st);
  }
}

}  // namespace
}  // namespace fo

using namespace fo;

extern "C" {

int64_t fo_orthogonalize_workspace(const fo_matrix_update* items, int count, int dtype) {
  if (check_items(items, count, dtype)) return -1;
  const int parts = dtype == FO_DTYPE_F32 ? 2 : 1;
  int64_t most = 0;
  for (int i = 0; i < count; i += kItems) {
    int64_t sum = 0;
    for (int k = i; k < count && k < i + kItems; ++k) sum += item_bytes(items[k], parts);
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
  const int64_t need = fo_orthogonalize_workspace(items, count, dtype);
  if (need > 0 && (!workspace || odd(workspace, 256) || workspace_bytes < need))
    return bad("the workspace is missing, misaligned or too small");
  const int parts = dtype == FO_DTYPE_F32 ? 2 : 1;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  for (int first = 0; first < count; first += kItems)
   for (const bool small : {true, false}) {
    OrthoParams p = {};
    p.ws = static_cast<char*>(workspace);
    p.steps = steps;
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
      if (m.rows == 0 || m.cols == 0 || is_small(m) != small) continue;
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
        it.a = take(int64_t(it.mt) * it.mt * 4 * kBlock * parts);
        it.c = take(int64_t(it.mt) * it.mt * 4 * kBlock * parts);
        it.parts = take(shared_bytes(it.mt, it.nt));
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
    p.done = reinterpret_cast<unsigned*>(p.scale + p.count);
    p.shared = p.done + p.count;
    const cudaError_t e = small ? (dtype == FO_DTYPE_F32 ? orthogonalize_small<float>(p, st) : orthogonalize_small<bf16>(p, st))
                          : dtype == FO_DTYPE_F32 ? orthogonalize<float>(p, st) : orthogonalize<bf16>(p, st);
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
