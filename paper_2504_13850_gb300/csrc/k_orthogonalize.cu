// Orthogonalised updates of weight matrices by Newton-Schulz products, for a
// list of matrices at once, with the momentum before and the parameters' update
// after them.
//
//   X = U / (|U|_F + eps), of U or its transpose so that m <= n;  then `steps` times
//   A = X X^T (m x m);  B = a I + b A + c A A;  X <- B X
//
// A and A A are symmetric: only tiles on and above the diagonal are formed and
// stored, 3 m^2 n + m^3 multiplications and additions per step instead of
// 4 m^2 n + 2 m^3.  An operand whose tile lies below the diagonal is read from
// its mirror image as a matrix with the other major-ness, so nothing is
// transposed in memory.
//
// Operands are fp16, not bf16: singular values stay below about 1.3, so the
// range is known and held in the middle of fp16's by powers of two, and each
// rounding costs 2^-12 instead of 2^-9.  For fp32 matrices each operand is a sum
// of two fp16 numbers (22 bits) and each product three (hi hi, hi lo, lo hi);
// the fourth is below fp32's rounding.  Sums are fp32 in tensor memory; because
// the tensor cores truncate, those of fp32 matrices are moved to registers and
// added there, rounded, every 512 terms, and the two small products have a sum
// of their own.
//
// X, A and B lie in the workspace as blocks of 64 x 64 elements of 8 KB in the
// image that a 128-byte-swizzled operand has in shared memory, block rows
// fastest: every operand tile is one or two contiguous copies without a tensor
// map, whatever the number and sizes of the matrices, and the padding of odd
// sizes to 128 is zeros.
#include "fo_scored_tc.cuh"
#include "fo_vec8.cuh"
#include "../../include/fedoptima.h"

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
constexpr float kUpX = 1024.f, kUpA = 256.f;  // what X, and A and B, are multiplied by as fp16

struct Item {
  const void* g;            // [rows][cols] gradient
  float *mom, *param;
  void* out;
  int64_t ldg, ldm, ldp, ldo;
  int64_t x[2], a, b;       // byte offsets in the workspace
  int64_t sums;             // index of its partial sums
  int rows, cols, mt, nt;   // mt, nt: tiles of 128 of the smaller and the larger side
  int nsums, transposed;
  float step;
};
struct OrthoParams {
  Item item[kItems];
  int start[kItems + 1];    // first unit of work of each matrix in this launch
  char* ws;
  double* sums;
  int count, from, last;    // from: which X is read; last: X goes to the caller
  float ca, cb, cc, mu, decay;
  int nesterov;
  double eps;
};

__device__ __forceinline__ int item_of(const OrthoParams& p, int unit) {
  int n = 0;
  while (n + 1 < p.count && unit >= p.start[n + 1]) ++n;
  return n;
}

// ------------------------------------------------------------- before the steps
// U of one element; FIRST updates the momentum, afterwards it is read.
template <typename T, bool FIRST>
__device__ __forceinline__ float update_at(const OrthoParams& p, const Item& it, int64_t r, int64_t c) {
  const float g = to_f(static_cast<const T*>(it.g)[r * it.ldg + c]);
  if (!it.mom) return g;
  float* m = it.mom + r * it.ldm + c;
  float v = *m;
  if (FIRST) *m = v = fmaf(p.mu, v, g);
  return p.nesterov ? fmaf(p.mu, v, g) : v;
}

// Sums of squares.  fp32 squares leave its range beyond 2^+-64; elements far
// from 1 are squared in units of 2^80 or 2^-80 and summed apart.
template <typename T>
__global__ void __launch_bounds__(256) ortho_sums_k(const __grid_constant__ OrthoParams p) {
  __shared__ double box[8];
  pdl_wait();
  pdl_trigger();
  const int n = item_of(p, blockIdx.x), part = int(blockIdx.x) - p.start[n];
  const Item& it = p.item[n];
  const int64_t total = int64_t(it.rows) * it.cols, per = (total + it.nsums - 1) / it.nsums;
  const int64_t end = min(total, (part + 1) * per);
  float mid = 0.f, big = 0.f, small = 0.f;
  for (int64_t e = part * per + threadIdx.x; e < end; e += 256) {
    const int64_t r = e / it.cols;
    const float v = update_at<T, true>(p, it, r, e - r * it.cols), a = fabsf(v);
    if (a > 0x1p40f) big = fmaf(v * 0x1p-80f, v * 0x1p-80f, big);
    else if (a < 0x1p-40f) small = fmaf(v * 0x1p80f, v * 0x1p80f, small);
    else mid = fmaf(v, v, mid);         // NaN too
  }
  double s = double(mid) + double(big) * 0x1p160 + double(small) * 0x1p-160;
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (threadIdx.x % 32 == 0) box[threadIdx.x / 32] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w) s += box[w];
    p.sums[it.sums + part] = s;
  }
}

__device__ __forceinline__ uint32_t half_pair(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 of_pair(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

// X = U / (|U| + eps) as an image: one 64 x 64 block per block of threads.
template <typename T, int PARTS>
__global__ void __launch_bounds__(256) ortho_pack_k(const __grid_constant__ OrthoParams p) {
  __shared__ float tile[64][65];
  __shared__ double box[8];
  pdl_wait();
  pdl_trigger();
  const int n = item_of(p, blockIdx.x);
  const Item& it = p.item[n];
  const int blk = int(blockIdx.x) - p.start[n], rows = 2 * it.mt;
  const int rb = blk % rows, cb = blk / rows, t = threadIdx.x;
  double s = 0.0;
  for (int i = t; i < it.nsums; i += 256) s += p.sums[it.sums + i];
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (t % 32 == 0) box[t / 32] = s;
  // the user's matrix, rows along its rows
  const int r0 = 64 * (it.transposed ? cb : rb), c0 = 64 * (it.transposed ? rb : cb);
  for (int e = t; e < 4096; e += 256) {
    const int r = r0 + e / 64, c = c0 + e % 64;
    tile[e / 64][e % 64] = r < it.rows && c < it.cols ? update_at<T, false>(p, it, r, c) : 0.f;
  }
  __syncthreads();
  s = 0.0;
  for (int w = 0; w < 8; ++w) s += box[w];
  const double norm = sqrt(s) + p.eps;
  // a power of two first, so that neither factor leaves fp32's range
  int k = 0;
  const double part = frexp(norm, &k);          // norm = part 2^k
  const bool fine = isfinite(norm);
  const float s1 = fine ? ldexpf(1.f, min(127, -k)) : float(1.0 / norm), s2 = fine ? float(double(kUpX) / part) : 1.f;
  const int row = t / 4;
  char* img = p.ws + it.x[0] + int64_t(cb * int64_t(rows) + rb) * kBlock + row * 128;
  const int64_t image = int64_t(it.mt) * it.nt * 4 * kBlock;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int u = t % 4 * 2 + h;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (it.transposed ? tile[8 * u + e][row] : tile[row][8 * u + e]) * s1 * s2;
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = half_pair(v[2 * e], v[2 * e + 1]);
    const int at = (u ^ (row & 7)) * 16;
    *reinterpret_cast<uint4*>(img + at) = make_uint4(w[0], w[1], w[2], w[3]);
    if (PARTS == 2) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 f = of_pair(w[e]);
        w[e] = half_pair(v[2 * e] - f.x, v[2 * e + 1] - f.y);
      }
      *reinterpret_cast<uint4*>(img + image + at) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

// ------------------------------------------------------------------ products
enum { kGram = 0, kPoly = 1, kApply = 2 };
constexpr int kThreads = 320;                 // copies, products, eight warps of arithmetic
constexpr int kOperand = 2 * kBlock;          // 128 x 64
constexpr int kSums = 8;                      // blocks of 64 terms between sums in registers (fp32 matrices)

template <int PARTS>
struct Tiles {
  static constexpr int kStage = 2 * PARTS * kOperand, kStages = PARTS == 2 ? 3 : 6;
  static constexpr int kOut = 8 * 4096;       // 4 KB per warp of arithmetic
  static constexpr int kBars = 2 * kStages + 5;
  static constexpr int kSmem = 1024 + kStages * kStage + kOut + 8 * kBars + 16;
  static constexpr uint32_t kCols = PARTS * 256;
};
static_assert(Tiles<2>::kSmem <= 232448 && Tiles<1>::kSmem <= 232448, "shared memory per CTA");

struct Place {
  int item, i, j, kb;       // tile and its blocks of 64 terms
};
template <int PHASE>
__device__ __forceinline__ Place place_of(const OrthoParams& p, int unit) {
  Place a;
  a.item = item_of(p, unit);
  const Item& it = p.item[a.item];
  const int t = unit - p.start[a.item];
  if (PHASE == kApply) {
    a.i = t % it.mt;
    a.j = t / it.mt;
  } else {                  // i <= j, column by column
    int j = int((sqrtf(8.f * float(t) + 1.f) - 1.f) * 0.5f);
    while ((j + 1) * (j + 2) / 2 <= t) ++j;
    while (j * (j + 1) / 2 > t) --j;
    a.j = j;
    a.i = t - j * (j + 1) / 2;
  }
  a.kb = 2 * (PHASE == kGram ? it.nt : it.mt);
  return a;
}

// 128 rows 128 i .. of block column kb, or the columns 128 i .. of block row kb.
__device__ __forceinline__ void copy_rows(char* dst, const char* img, int mt, int i, int kb, uint64_t* bar) {
  bulk_g2s(dst, img + (int64_t(kb) * 2 * mt + 2 * i) * kBlock, kOperand, bar);
}
__device__ __forceinline__ void copy_cols(char* dst, const char* img, int mt, int i, int kb, uint64_t* bar) {
  const char* src = img + (int64_t(2 * i) * 2 * mt + kb) * kBlock;
  bulk_g2s(dst, src, kBlock, bar);
  bulk_g2s(dst + kBlock, src + int64_t(2 * mt) * kBlock, kBlock, bar);
}

template <int PARTS, int PHASE, typename T>
__global__ void __launch_bounds__(kThreads, 1) ortho_product_k(const __grid_constant__ OrthoParams p) {
  using S = Tiles<PARTS>;
  extern __shared__ char smem_raw[];
  char* smem = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  char* stage_out = smem + S::kStages * S::kStage;
  uint64_t* full = reinterpret_cast<uint64_t*>(stage_out + S::kOut);
  uint64_t *empty = full + S::kStages, *acc_full = empty + S::kStages, *acc_empty = acc_full + 2, *done = acc_empty + 2;
  uint32_t* tslot = reinterpret_cast<uint32_t*>(done + 1);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int units = p.start[p.count];

  if (threadIdx.x == 0) {
    for (int e = 0; e < S::kStages; ++e) {
      mbar_init(&full[e], 1);
      mbar_init(&empty[e], 1);
    }
    for (int e = 0; e < 2; ++e) {
      mbar_init(&acc_full[e], 1);
      mbar_init(&acc_empty[e], 8);         // one arrival per warp
    }
    mbar_init(done, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tslot)), "r"(S::kCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tslot;      // sum s: columns 128 PARTS s (and + 128 for the small products)
  pdl_trigger();                     // this block holds its tensor memory
  pdl_wait();
  Waits wait(&g_err);

  if (warp == 0) {
    if (lane == 0) {
      Ring<S::kStages> at;
      int it = 0;
      for (int u = blockIdx.x; u < units && !wait.dead; u += gridDim.x) {
        const Place a = place_of<PHASE>(p, u);
        const Item& m = p.item[a.item];
        const char* x = p.ws + m.x[p.from];
        const char* sym = p.ws + (PHASE == kPoly ? m.a : m.b);
        const int64_t xi = int64_t(m.mt) * m.nt * 4 * kBlock, si = int64_t(m.mt) * m.mt * 4 * kBlock;
        for (int kb = 0; kb < a.kb; ++kb, ++it) {
          if (it >= S::kStages) wait.on(&empty[at.at], at.phase ^ 1, 61);
          if (wait.dead) break;
          char* s = smem + at.at * S::kStage;
          uint64_t* bar = &full[at.at];
          mbar_expect_tx(bar, S::kStage);
#pragma unroll
          for (int q = 0; q < PARTS; ++q) {
            char *da = s + q * kOperand, *db = s + (PARTS + q) * kOperand;
            if (PHASE == kGram) {
              copy_rows(da, x + q * xi, m.mt, a.i, kb, bar);
              copy_rows(db, x + q * xi, m.mt, a.j, kb, bar);
            } else {
              if (a.i <= kb / 2) copy_rows(da, sym + q * si, m.mt, a.i, kb, bar);
              else copy_cols(da, sym + q * si, m.mt, a.i, kb, bar);
              if (PHASE == kApply) copy_cols(db, x + q * xi, m.mt, a.j, kb, bar);
              else if (a.j <= kb / 2) copy_rows(db, sym + q * si, m.mt, a.j, kb, bar);
              else copy_cols(db, sym + q * si, m.mt, a.j, kb, bar);
            }
          }
          at.step();
        }
      }
      // every copy has landed before the block ends, whichever role gave up
      for (int e = max(0, it - S::kStages); e < it; ++e) mbar_wait(&full[e % S::kStages], (e / S::kStages) & 1);
    }
  } else if (warp == 1) {
    // kind::f16 with fp16 operands, fp32 sums, M = N = 128
    constexpr uint32_t id = (1u << 4) | (128u >> 3) << 17 | (128u >> 4) << 24;
    Ring<S::kStages> at;
    uint32_t pass = 0;
    const uint32_t ring = smem_u32(smem);
    for (int u = blockIdx.x; u < units; u += gridDim.x) {
      const Place a = place_of<PHASE>(p, u);
      for (int kb = 0; kb < a.kb; ++kb) {
        const int in = PARTS == 2 ? kb % kSums : kb;
        const uint32_t d = tmem + (pass & 1) * 128 * PARTS;
        if (in == 0) wait.on_lanes(&acc_empty[pass & 1], ((pass >> 1) & 1) ^ 1, 62);
        wait.on_lanes(&full[at.at], at.phase, 63);
        tc_fence_after();
        const uint32_t s = ring + at.at * S::kStage;
        // mirrored operands have their rows along the terms
        const uint32_t am = PHASE != kGram && a.i > kb / 2, bm = PHASE == kApply || (PHASE == kPoly && a.j > kb / 2);
        const uint32_t idesc = id | am << 15 | bm << 16;
        const uint32_t as = am ? 2048u : 32u, bs = bm ? 2048u : 32u;
        const uint32_t al = (am ? uint32_t(kBlock) : 16u) >> 4 << 16, bl = (bm ? uint32_t(kBlock) : 16u) >> 4 << 16;
        constexpr uint32_t hi = (1024u >> 4) | (1u << 14) | (2u << 29);      // stride 1024, version 1, 128-byte swizzle
        auto desc = [&](uint32_t off, uint32_t lbo) { return uint64_t(((s + off) & 0x3ffff) >> 4 | lbo) | uint64_t(hi) << 32; };
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t first = in > 0 || k > 0 ? 1u : 0u;
          const uint64_t ah = desc(k * as, al), bh = desc(PARTS * kOperand + k * bs, bl);
          mma_ss(d, ah, bh, idesc, first);
          if (PARTS == 2) {
            mma_ss(d + 128, ah, desc(3 * kOperand + k * bs, bl), idesc, first);
            mma_ss(d + 128, desc(kOperand + k * as, al), bh, idesc, 1u);
          }
        }
        commit_to(&empty[at.at]);
        at.step();
        if (kb + 1 == a.kb || (PARTS == 2 && in + 1 == kSums)) commit_to(&acc_full[pass++ & 1]);
        // off the waits' path; what was issued after one gave up is void anyway
        if (__any_sync(0xffffffffu, wait.dead)) break;
      }
      if (__any_sync(0xffffffffu, wait.dead)) break;
    }
    // no product is in flight when the block ends and its memory is another's
    commit_to(done);
    mbar_wait(done, 0);
    __syncwarp();
  } else {
    // warp: 32 rows 32 q .. and 64 columns, half a block
    const int q = warp % 4, half = (warp - 2) / 4;
    const uint32_t col = tmem + (uint32_t(32 * q) << 16) + 64 * half;
    const uint32_t buf = smem_u32(stage_out) + uint32_t(warp - 2) * 4096u;
    uint32_t pass = 0;
    for (int u = blockIdx.x; u < units; u += gridDim.x) {
      const Place a = place_of<PHASE>(p, u);
      const Item& m = p.item[a.item];
      float v[64];
      for (int kb = 0; kb < a.kb; kb += PARTS == 2 ? kSums : a.kb, ++pass) {
        wait.on_lanes(&acc_full[pass & 1], (pass >> 1) & 1, 64);
        tc_fence_after();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t from = col + (pass & 1) * 128 * PARTS + 32 * h;
          uint32_t r[32];
          tmem_ld32(from, r);
#pragma unroll
          for (int e = 0; e < 32; ++e) v[32 * h + e] = (PARTS == 2 && kb > 0 ? v[32 * h + e] : 0.f) + __uint_as_float(r[e]);
          if (PARTS == 2) {
            tmem_ld32(from + 128, r);
#pragma unroll
            for (int e = 0; e < 32; ++e) v[32 * h + e] += __uint_as_float(r[e]);
          }
        }
        tc_fence_before();
        arrive_warp(&acc_empty[pass & 1]);
      }
      if (__any_sync(0xffffffffu, wait.dead)) break;
      const int row = 128 * a.i + 32 * q + lane, c0 = 128 * a.j + 64 * half;     // of the smaller and the larger side
      const int64_t block = int64_t(2 * a.j + half) * 2 * m.mt + 2 * a.i + q / 2;
      const int in_block = (q & 1) * 4096 + lane * 128;
      const int64_t si = int64_t(m.mt) * m.mt * 4 * kBlock;
      if (PHASE == kApply && p.last) {
        constexpr float down = 1.f / (kUpX * kUpA);
        const int side = m.transposed ? m.cols : m.rows, other = m.transposed ? m.rows : m.cols;
        if (row < side) {
          const int64_t so = m.transposed ? m.ldo : 1, sp = m.transposed ? m.ldp : 1;
          const int64_t fo = m.transposed ? int64_t(row) : row * m.ldo, fp = m.transposed ? int64_t(row) : row * m.ldp;
#pragma unroll
          for (int e = 0; e < 64; ++e) {
            const int c = c0 + e;
            if (c < other) {
              const float x = v[e] * down;
              if (m.out) static_cast<T*>(m.out)[fo + c * so] = from_f<T>(x);
              if (m.param) {
                float* w = m.param + fp + c * sp;
                *w = fmaf(-m.step, x, *w * p.decay);
              }
            }
          }
        }
        continue;
      }
      if (PHASE == kPoly) {
        const char* src = p.ws + m.a + block * kBlock + in_block;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int off = (k ^ (lane & 7)) * 16;
          float z[8];
#pragma unroll
          for (int part = 0; part < PARTS; ++part) {
            const uint4 w = *reinterpret_cast<const uint4*>(src + part * si + off);
            const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 f = of_pair(ww[e]);
              z[2 * e] = (part ? z[2 * e] : 0.f) + f.x;
              z[2 * e + 1] = (part ? z[2 * e + 1] : 0.f) + f.y;
            }
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int c = 8 * k + e;
            const float diagonal = row == c0 + c ? p.ca * kUpA : 0.f;
            v[c] = fmaf(p.cc / kUpA, v[c], fmaf(p.cb, z[e], diagonal));
          }
        }
      } else {
        constexpr float down = PHASE == kGram ? kUpA / (kUpX * kUpX) : 1.f / kUpA;
#pragma unroll
        for (int e = 0; e < 64; ++e) v[e] *= down;
      }
      char* dst = p.ws + (PHASE == kGram ? m.a : PHASE == kPoly ? m.b : m.x[p.from ^ 1]) + block * kBlock + (q & 1) * 4096;
      const int64_t image = PHASE == kApply ? int64_t(m.mt) * m.nt * 4 * kBlock : si;
#pragma unroll
      for (int part = 0; part < PARTS; ++part) {
        if (lane == 0) bulk_wait_read<0>();       // the last store has read the buffer
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float &x = v[8 * k + 2 * e], &y = v[8 * k + 2 * e + 1];
            w[e] = half_pair(x, y);
            const float2 f = of_pair(w[e]);
            x -= f.x;
            y -= f.y;
          }
          st_shared4(buf + lane * 128 + (k ^ (lane & 7)) * 16, w[0], w[1], w[2], w[3]);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], 4096;" ::"l"(dst + part * image), "r"(buf) : "memory");
          asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
      }
    }
    if (lane == 0) bulk_wait_all();
    __syncwarp();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kCols) : "memory");
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
int64_t item_bytes(const fo_matrix_update& m, int parts) {
  if (m.rows == 0 || m.cols == 0) return 0;
  const int64_t r = (m.rows + 127) / 128, c = (m.cols + 127) / 128, mt = r < c ? r : c, nt = r < c ? c : r;
  return (2 * mt * nt + 2 * mt * mt) * 4 * kBlock * parts + kMaxSums * 8;
}

template <int PARTS, int PHASE, typename T>
cudaError_t product(OrthoParams& p, int sms, cudaStream_t st) {
  auto k = ortho_product_k<PARTS, PHASE, T>;
  static std::atomic<bool> allowed[kMaxDevices];
  const cudaError_t e = allow_smem(k, allowed);
  if (e != cudaSuccess) return e;
  int64_t units = 0;
  for (int i = 0; i < p.count; ++i) {
    p.start[i] = int(units);
    units += PHASE == kApply ? int64_t(p.item[i].mt) * p.item[i].nt : int64_t(p.item[i].mt) * (p.item[i].mt + 1) / 2;
  }
  p.start[p.count] = int(units);
  return launch_k(k, dim3(unsigned(units < sms ? units : sms)), dim3(kThreads), Tiles<PARTS>::kSmem, st, p);
}

template <typename T>
cudaError_t orthogonalize(OrthoParams& p, int steps, cudaStream_t st) {
  constexpr int PARTS = sizeof(T) == 4 ? 2 : 1;
  int dev = 0, sms = 1;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  int64_t units = 0;
  for (int i = 0; i < p.count; ++i) {
    p.start[i] = int(units);
    units += p.item[i].nsums;
  }
  p.start[p.count] = int(units);
  if ((e = launch_k(ortho_sums_k<T>, dim3(unsigned(units)), dim3(256), 0, st, p)) != cudaSuccess) return e;
  units = 0;
  for (int i = 0; i < p.count; ++i) {
    p.start[i] = int(units);
    units += 4 * int64_t(p.item[i].mt) * p.item[i].nt;
  }
  p.start[p.count] = int(units);
  if ((e = launch_k(ortho_pack_k<T, PARTS>, dim3(unsigned(units)), dim3(256), 0, st, p)) != cudaSuccess) return e;
  for (int s = 0; s < steps; ++s) {
    p.from = s & 1;
    p.last = s + 1 == steps;
    if ((e = product<PARTS, kGram, T>(p, sms, st)) != cudaSuccess) return e;
    if ((e = product<PARTS, kPoly, T>(p, sms, st)) != cudaSuccess) return e;
    if ((e = product<PARTS, kApply, T>(p, sms, st)) != cudaSuccess) return e;
  }
  return cudaSuccess;
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
  if (fo_orthogonalize_workspace(items, count, dtype) > 0 &&
      (!workspace || odd(workspace, 256) || workspace_bytes < fo_orthogonalize_workspace(items, count, dtype)))
    return bad("the workspace is missing, misaligned or too small");
  const int parts = dtype == FO_DTYPE_F32 ? 2 : 1;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  for (int first = 0; first < count; first += kItems) {
    OrthoParams p = {};
    p.ws = static_cast<char*>(workspace);
    p.ca = float(coefficients[0]);
    p.cb = float(coefficients[1]);
    p.cc = float(coefficients[2]);
    p.mu = float(momentum);
    p.decay = float(decay);
    p.nesterov = nesterov != 0;
    p.eps = eps;
    int64_t at = 0;
    auto take = [&at](int64_t bytes) {
      const int64_t here = at;
      at += bytes;
      return here;
    };
    for (int i = first; i < count && i < first + kItems; ++i) {
      const fo_matrix_update& m = items[i];
      if (m.rows == 0 || m.cols == 0) continue;
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
      for (int k = 0; k < 2; ++k) it.x[k] = take(int64_t(it.mt) * it.nt * 4 * kBlock * parts);
      it.a = take(int64_t(it.mt) * it.mt * 4 * kBlock * parts);
      it.b = take(int64_t(it.mt) * it.mt * 4 * kBlock * parts);
      const int64_t sums = (m.rows * m.cols + 16383) / 16384;
      it.nsums = int(sums < kMaxSums ? sums : kMaxSums);
      it.step = m.step;
    }
    if (p.count == 0) continue;
    p.sums = reinterpret_cast<double*>(p.ws + at);
    for (int i = 0; i < p.count; ++i) p.item[i].sums = int64_t(i) * kMaxSums;
    const cudaError_t e = dtype == FO_DTYPE_F32 ? orthogonalize<float>(p, steps, st) : orthogonalize<bf16>(p, steps, st);
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
