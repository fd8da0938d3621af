// Scored attention (fo_scored.h): the C entry points, the preparation kernels
// and the CUDA-core kernels, which take every type, head width and stride.
//
// The CUDA-core kernels work on 64 x 64 score tiles with 256 threads, each
// thread 4 x 4 scores.  All operand tiles lie in shared memory as fp32,
// [width][64 tokens]: both products of a tile then read 16-byte vectors along
// the tokens, S = X U^T as one vector of each operand per width step (16 FMAs
// per two reads) and the accumulating product (O += P V, dQ += dS K, ...) as
// four columns of P against NC widths (16 NC FMAs per NC + 4 reads).  Vectors
// are permuted by the width index, so that the transposing copies of a warp
// (8 x 4 widths x 4 tokens) and the vector reads meet no bank twice.  The next
// tile's copies run while the current one is worked on: fp32 elements go to
// their transposed place by 4-byte asynchronous copies, which need no
// registers (loading them with the threads took five times the FMAs' time).
// Padding and rows past the end are stored as zeros: what they hold never
// reaches a sum.
// The backward pass is two kernels of one body: a tile of queries walks the
// keys (dQ), then a tile of keys walks the queries (dK, dV and the table
// gradient); every sum has a fixed order, at the price of forming the scores
// twice.  The first one adds each row's sum of dS, which the rounding of O
// keeps from being zero, to D for the second.  Where tiles of rows are few, or
// differ in length under a causal mask, a cluster of blocks shares one (Share).
// Bound by instruction issue: FMAs are a little over half of the instructions
// and 16 warps per SM fill a little over half of the slots.  2 x 2048 tokens,
// 8 heads of 64, fp32: forward 667 us (25.8 TFLOP/s), backward 2.04 ms (21.0,
// counting 5 products).
#include "fo_common.cuh"
#include "fo_scored.h"
#include "../../include/fedoptima.h"

#include <algorithm>
#include <climits>
#include <cmath>
#include <string>

namespace fo {
int report_error(int code, const std::string& msg);

namespace {

constexpr int kT = 64;             // tile of tokens
constexpr int kThreads = 256;
constexpr int kBiasPart = 2 * kMaxReach + 4;              // floats in shared memory of a head's biases
constexpr int kGradPart = kBiasPart + 256;                // and of its table gradient: by distance, and beyond the reach

// ------------------------------------------------------------- preparation
// Document ids padded to Lp (-1 past the sequence), and the summary of each
// 64 ids: one warp per 64 ids, w of them.
__device__ __forceinline__ void summarise_docs(const ScoredParams& p, int64_t w) {
  const int per = p.Lp / kScoredBlock, lane = threadIdx.x % 32;
  if (w >= int64_t(p.B) * per) return;
  const int64_t b = w / per;
  const int l0 = int(w % per) * kScoredBlock;
  int2 s = make_int2(INT_MAX, -1);
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int l = l0 + lane + 32 * t;
    int id = -1;
    if (l < p.L) {
      id = max(p.ids[b * p.L + l], -1);      // one id for all padding
      s = doc_join(s, id < 0 ? make_int2(int(0x80000000u) | INT_MAX, -1) : make_int2(id, id));
    }
    p.doc[b * p.Lp + l] = id;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    s = doc_join(s, make_int2(__shfl_xor_sync(0xffffffffu, s.x, o), __shfl_xor_sync(0xffffffffu, s.y, o)));
  if (lane == 0) p.blk[w] = s;
}

__global__ void __launch_bounds__(128) scored_docs_k(const __grid_constant__ ScoredParams p) {
  pdl_wait();
  pdl_trigger();
  summarise_docs(p, int64_t(blockIdx.x) * 4 + threadIdx.x / 32);
}

// -D_i = -sum_d dO O and -lse * log2(e), padded to Lp rows per (sequence, head).
// `lanes` lanes per row, VEC: 16-byte loads (8 bf16).
// The blocks from row_blocks on summarise the document ids.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) scored_delta_k(const __grid_constant__ ScoredParams p, int lanes,
                                                      unsigned row_blocks) {
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x >= row_blocks) {
    summarise_docs(p, int64_t(blockIdx.x - row_blocks) * 8 + threadIdx.x / 32);
    return;
  }
  const int per = 32 / lanes, lane = threadIdx.x % 32, sub = lane % lanes;
  const int64_t row = (int64_t(blockIdx.x) * 8 + threadIdx.x / 32) * per + lane / lanes;   // (b, h, l)
  const int64_t rows = int64_t(p.B) * p.H * p.Lp;
  float d = 0.f;
  bool live = false;
  int64_t bh = 0;
  int l = 0;
  if (row < rows) {
    l = int(row % p.Lp);
    bh = row / p.Lp;
    const int b = int(bh / p.H), h = int(bh % p.H);
    live = l < p.L && (!p.ids || p.ids[int64_t(b) * p.L + l] >= 0);
    if (live) {
      const T* o = static_cast<const T*>(p.o.p) + b * p.o.sb + l * p.o.sl + h * p.o.sh;
      const T* g = static_cast<const T*>(p.dout.p) + b * p.dout.sb + l * p.dout.sl + h * p.dout.sh;
      if (VEC) {
        if (sub * 8 < p.D) {
          const uint4 a = reinterpret_cast<const uint4*>(o)[sub], c = reinterpret_cast<const uint4*>(g)[sub];
          const bf16 *ab = reinterpret_cast<const bf16*>(&a), *cb = reinterpret_cast<const bf16*>(&c);
#pragma unroll
          for (int e = 0; e < 8; ++e) d = fmaf(__bfloat162float(ab[e]), __bfloat162float(cb[e]), d);
        }
      } else {
        for (int e = sub; e < p.D; e += lanes) d = fmaf(to_f(o[e]), to_f(g[e]), d);
      }
    }
  }
  for (int o = lanes / 2; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
  if (row < rows && sub == 0) {
    const float lse = live ? p.lse[bh * p.L + l] : -INFINITY;
    p.delta[row] = live ? -d : 0.f;
    p.lse2[row] = lse == -INFINITY ? -INFINITY : -lse * kLog2e;
  }
}

// dtable[h][b] = sum of its partials, one warp each, in a fixed order.
template <typename T>
__global__ void __launch_bounds__(128) scored_table_k(const float* __restrict__ part, T* __restrict__ out, int rows,
                                                      int64_t n) {
  pdl_wait();
  pdl_trigger();
  const int r = blockIdx.x * 4 + threadIdx.x / 32, lane = threadIdx.x % 32;
  if (r >= rows) return;
  float s = 0.f;
  for (int64_t i = lane; i < n; i += 32) s += part[r * n + i];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane == 0) out[r] = from_f<T>(s);
}

// ----------------------------------------------------------- shared helpers
// Float offset of the 16-byte vector g (tokens 4 g .. 4 g + 3) of row d.
__device__ __forceinline__ int at4(int d, int g) { return d * kT + ((g ^ ((d >> 2) & 7)) << 2); }

// Width n of this thread's NC accumulator columns.
template <int NC>
__device__ __forceinline__ int width_of(int tx, int n) {
  return NC == 2 ? 2 * tx + n : 4 * tx + (n & 3) + 64 * (n >> 2);
}

__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// Until at most N of this thread's groups of copies are in flight.
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// 64 tokens from l0 of one (sequence, head) -> dst[width][64], fp32, widths
// rounded up to 32; tokens past the end and padding as zeros.  Asynchronous
// for fp32 (copies_commit / copies_wait).
template <typename T>
__device__ __forceinline__ void load_tile(float* dst, const Strided& t, const ScoredParams& p, int b, int h, int l0) {
  const T* base = static_cast<const T*>(t.p) + b * t.sb + h * t.sh;
  const int32_t* doc = p.doc ? p.doc + int64_t(b) * p.Lp : nullptr;
  const int warp = threadIdx.x / 32, dl = (threadIdx.x % 32) >> 2, rl = threadIdx.x & 3;
  const int n = (p.D + 31) / 32 * (kT / 4);
#pragma unroll 4
  for (int e = warp; e < n; e += kThreads / 32) {
    const int g = e % (kT / 4), d0 = e / (kT / 4) * 32 + 4 * dl, l = l0 + 4 * g + rl;
    const bool live = l < p.L && (!doc || doc[l] >= 0);
    const T* src = base + (live ? l * t.sl : 0);
    float* to = dst + at4(d0, g) + rl;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const bool in = live && d0 + c < p.D;
      if (sizeof(T) == 4) {
        const int bytes = in ? 4 : 0;      // 0: the copy writes a zero
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(
                         static_cast<uint32_t>(__cvta_generic_to_shared(to + c * kT))),
                     "l"(in ? src + d0 + c : base), "r"(bytes)
                     : "memory");
      } else {
        to[c * kT] = in ? to_f(src[d0 + c]) : 0.f;
      }
    }
  }
}

// s[r][c] = sum_d X[d][row r] U[d][column c], widths rounded up to 4.  The
// permutation repeats every 32 widths: unrolled over them its offsets are
// constants xor the thread's vector.
__device__ __forceinline__ void scores(float (&s)[4][4], const float* X, const float* U, int D, int ty, int tx) {
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int c = 0; c < 4; ++c) s[r][c] = 0.f;
#pragma unroll 1
  for (int d0 = 0; d0 < D; d0 += 32, X += 32 * kT, U += 32 * kT) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (d0 + 4 * k >= D) break;
      const float *x = X + 4 * k * kT + ((ty ^ k) << 2), *u = U + 4 * k * kT + ((tx ^ k) << 2);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float4 a = *reinterpret_cast<const float4*>(x + e * kT);
        const float4 w = *reinterpret_cast<const float4*>(u + e * kT);
        const float av[4] = {a.x, a.y, a.z, a.w}, wv[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int c = 0; c < 4; ++c) s[r][c] = fmaf(av[r], wv[c], s[r][c]);
      }
    }
  }
}

// Offset of the vector of rows 4 ty .. 4 ty + 3 of column c of a 64 x 64 tile
// held by columns.
__device__ __forceinline__ int at_p(int c, int ty) { return c * kT + ((ty ^ ((c >> 2) & 15)) << 2); }

__device__ __forceinline__ void put_tile(float* P, const float (&s)[4][4], int ty, int tx) {
#pragma unroll
  for (int c = 0; c < 4; ++c)
    *reinterpret_cast<float4*>(P + at_p(4 * tx + c, ty)) = make_float4(s[0][c], s[1][c], s[2][c], s[3][c]);
}

// acc[r][n] += sum_c P[row r][c] W[width n of this thread][c].
template <int NC>
__device__ __forceinline__ void accumulate(float (&acc)[4][NC], const float* P, const float* W, int ty, int tx) {
  // rows of W this thread reads share one permutation (see width_of)
  const int first = width_of<NC>(tx, 0), turn = (first >> 2) & 7;
  W += first * kT;
#pragma unroll 1
  for (int g0 = 0; g0 < kT / 4; g0 += 4, P += 16 * kT) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float *w_at = W + (((g0 + k) ^ turn) << 2), *p_at = P + 4 * k * kT + ((ty ^ (g0 + k)) << 2);
      float4 w[NC];
#pragma unroll
      for (int n = 0; n < NC; ++n)
        w[n] = *reinterpret_cast<const float4*>(w_at + (NC == 2 ? n : (n & 3) + 64 * (n >> 2)) * kT);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const float4 q = *reinterpret_cast<const float4*>(p_at + c * kT);
        const float qv[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int n = 0; n < NC; ++n) {
          const float wv = c == 0 ? w[n].x : c == 1 ? w[n].y : c == 2 ? w[n].z : w[n].w;
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[r][n] = fmaf(qv[r], wv, acc[r][n]);
        }
      }
    }
  }
}

// An accumulating product reads all 16 NC rows of widths, also those that
// load_tile does not write; they are cleared once.
__device__ __forceinline__ void clear_tail(float* W, int D, int rows) {
  for (int e = (D + 31) / 32 * 32 * kT + threadIdx.x; e < rows * kT; e += kThreads) W[e] = 0.f;
}

template <typename T>
__device__ __forceinline__ void load_bias(float* bias, const ScoredParams& p, int h) {
  if (!p.table) return;
  const T* t = static_cast<const T*>(p.table) + int64_t(h) * p.buckets;
  for (int e = threadIdx.x; e < 2 * p.reach + 1; e += kThreads) bias[e] = bias_of(to_f(t[p.map[e]]));
}

// What decides on a pair besides its positions.
struct Pair {
  int pf;                // the sequence's prefix
  const int32_t* doc;    // its ids, or null
  float slope;
  int row_id[4], col_id[4];
};

__device__ __forceinline__ void ids_of(int (&id)[4], const Pair& c, int l0) {
  if (!c.doc) return;
  const int4 v = *reinterpret_cast<const int4*>(c.doc + l0);
  id[0] = v.x, id[1] = v.y, id[2] = v.z, id[3] = v.w;
}
__device__ __forceinline__ bool pair_allowed(const ScoredParams& p, const Pair& c, int i, int j, int r, int col) {
  if (i >= p.L || j >= p.L) return false;
  if (p.causal && j > i && j >= c.pf) return false;
  return !c.doc || (c.row_id[r] >= 0 && c.row_id[r] == c.col_id[col]);
}
// The biased score of raw product x, and 1 - tanh^2 of the cap (1 without).
__device__ __forceinline__ float pair_score(const ScoredParams& p, const Pair& c, const float* bias, float x, int i,
                                            int j, float* chain) {
  float z = x * p.scale;
  *chain = 1.f;
  if (p.cap > 0.f) {
    // the derivative as 4 e / (1 + e)^2, e = exp(-2 |y|): 1 - tanh^2 would keep
    // nothing but tanh's rounding where the score is at the cap
    const float y = z / p.cap, e = exp2f(-2.f * kLog2e * fabsf(y)), q = 1.f / (1.f + e);
    z = p.cap * tanhf(y);
    *chain = 4.f * e * q * q;
  }
  const int d = j - i;
  if (p.slopes) z -= c.slope * float(abs(d));
  if (p.table) z += bias[min(max(d, -p.reach), p.reach) + p.reach];
  return z;
}

__device__ __forceinline__ Pair pair_of(const ScoredParams& p, int b, int h) {
  Pair c = {};
  c.pf = p.prefix ? p.prefix[b] : 0;
  c.doc = p.doc ? p.doc + int64_t(b) * p.Lp : nullptr;
  c.slope = p.slopes ? p.slopes[h] : 0.f;
  return c;
}
__device__ __forceinline__ int tile_class(const ScoredParams& p, int pf, int b, int q0, int k0) {
  int2 qd = make_int2(0, 0), kd = qd;
  if (p.blk) {
    const int2* blk = p.blk + int64_t(b) * (p.Lp / kScoredBlock);
    qd = blk[q0 / kScoredBlock];
    kd = blk[k0 / kScoredBlock];
  }
  const int cls = scored_class(p, pf, q0, q0 + kT, k0, k0 + kT, p.blk != nullptr, qd, kd);
  return cls == kScoredAll && max(q0, k0) + kT > p.L ? kScoredSome : cls;
}
// The first tile from c0 on of which pairs with the tile at r0 are allowed
// (p.L or more: none); *cls receives its class.
template <bool KEYS_ARE_ROWS>
__device__ __forceinline__ int next_tile(const ScoredParams& p, int pf, int b, int r0, int c0, int* cls) {
  for (; c0 < p.L; c0 += kT) {
    *cls = tile_class(p, pf, b, KEYS_ARE_ROWS ? c0 : r0, KEYS_ARE_ROWS ? r0 : c0);
    if (*cls != kScoredNone) break;
  }
  return c0;
}

template <typename T, int NC>
__device__ __forceinline__ void store_rows(const Strided& t, const ScoredParams& p, const float (&acc)[4][NC],
                                           const float (&mul)[4], int b, int h, int l0, int ty, int tx) {
  T* base = static_cast<T*>(t.p) + b * t.sb + h * t.sh;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int l = l0 + 4 * ty + r;
    if (l >= p.L) continue;
#pragma unroll
    for (int n = 0; n < NC; ++n)
      if (width_of<NC>(tx, n) < p.D) base[l * t.sl + width_of<NC>(tx, n)] = from_f<T>(acc[r][n] * mul[r]);
  }
}

// A cluster of blocks may share a tile of rows: block `rank` of `n` takes every
// n-th allowed tile of columns, and the first one adds up.
struct Share {
  int n, rank;
  __device__ __forceinline__ explicit Share(int n_) : n(n_), rank(int(blockIdx.x) % n_) {}
  // Skips the other blocks' tiles: next_tile of the one after `count` more.
  template <bool KEYS_ARE_ROWS>
  __device__ __forceinline__ int skip(const ScoredParams& p, int pf, int b, int r0, int c0, int* cls, int count) const {
    c0 = next_tile<KEYS_ARE_ROWS>(p, pf, b, r0, c0, cls);
    for (; count > 0 && c0 < p.L; --count) c0 = next_tile<KEYS_ARE_ROWS>(p, pf, b, r0, c0 + kT, cls);
    return c0;
  }
  // This thread's value e of block r's buffer x (a shared-memory array at the
  // same place in every block).
  __device__ __forceinline__ static float of(const float* x, int e, int r) {
    uint32_t at;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                 : "=r"(at)
                 : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(x + e * kThreads + threadIdx.x))), "r"(r));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
    return v;
  }
};

// ----------------------------------------------------------------- forward
template <typename T, int NC>
__global__ void __launch_bounds__(kThreads, NC <= 4 ? 2 : 1) scored_fwd_k(const __grid_constant__ ScoredParams p) {
  extern __shared__ __align__(16) float sm[];
  constexpr int W = 16 * NC;
  constexpr int kTile = W * kT;
  float *Q = sm, *KVs = Q + kTile, *P = KVs + 4 * kTile, *bias = P + kT * kT;    // KVs: two pairs of K and V
  pdl_wait();
  pdl_trigger();
  const Share share(p.share);
  const unsigned work = blockIdx.x / unsigned(share.n);
  const int tiles = (p.L + kT - 1) / kT, bh = work % (p.B * p.H);      // the longest causal tiles first
  const int q0 = (tiles - 1 - int(work / (p.B * p.H))) * kT;
  const int b = bh / p.H, h = bh % p.H, kh = h / p.G;
  const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
  Pair pc = pair_of(p, b, h);
  int cls = 0, cls_next = 0, buf = 0;
  int k0 = share.skip<false>(p, pc.pf, b, q0, 0, &cls, share.rank);
  load_tile<T>(Q, p.q, p, b, h, q0);
  if (k0 < p.L) {
    load_tile<T>(KVs, p.k, p, b, kh, k0);
    load_tile<T>(KVs + kTile, p.v, p, b, kh, k0);
  }
  copies_commit();
  load_bias<T>(bias, p, h);
  clear_tail(KVs + kTile, p.D, W);
  clear_tail(KVs + 3 * kTile, p.D, W);
  ids_of(pc.row_id, pc, q0 + 4 * ty);
  float acc[4][NC] = {}, m[4], sum[4] = {0.f, 0.f, 0.f, 0.f};     // m in units of log2
#pragma unroll
  for (int r = 0; r < 4; ++r) m[r] = -INFINITY;
  while (k0 < p.L) {
    const int k1 = share.skip<false>(p, pc.pf, b, q0, k0 + kT, &cls_next, share.n - 1);
    if (k1 < p.L) {
      load_tile<T>(KVs + 2 * (buf ^ 1) * kTile, p.k, p, b, kh, k1);
      load_tile<T>(KVs + (2 * (buf ^ 1) + 1) * kTile, p.v, p, b, kh, k1);
    }
    copies_commit();
    copies_wait<1>();
    __syncthreads();
    const float *K = KVs + 2 * buf * kTile, *V = K + kTile;
    float s[4][4], chain;
    scores(s, Q, K, p.D, ty, tx);
    if (cls == kScoredSome) ids_of(pc.col_id, pc, k0 + 4 * tx);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = q0 + 4 * ty + r;
      float top = m[r];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int j = k0 + 4 * tx + c;
        s[r][c] = pair_score(p, pc, bias, s[r][c], i, j, &chain) * kLog2e;
        if (cls == kScoredSome && !pair_allowed(p, pc, i, j, r, c)) s[r][c] = -INFINITY;
        top = fmaxf(top, s[r][c]);
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      const float base = top == -INFINITY ? 0.f : top, keep = exp2f(m[r] - base);
      float part = 0.f;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        s[r][c] = exp2f(s[r][c] - base);
        part += s[r][c];
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) part += __shfl_xor_sync(0xffffffffu, part, o);
      sum[r] = sum[r] * keep + part;
      m[r] = top;
#pragma unroll
      for (int n = 0; n < NC; ++n) acc[r][n] *= keep;
    }
    put_tile(P, s, ty, tx);
    __syncthreads();
    accumulate<NC>(acc, P, V, ty, tx);
    __syncthreads();
    k0 = k1;
    cls = cls_next;
    buf ^= 1;
  }
  copies_wait<0>();
  if (share.n > 1) {
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float* x = KVs + r * (NC + 2) * kThreads + threadIdx.x;
      x[0] = m[r];
      x[kThreads] = sum[r];
#pragma unroll
      for (int n = 0; n < NC; ++n) x[(2 + n) * kThreads] = acc[r][n];
    }
    cluster_sync();
    if (share.rank == 0) {
#pragma unroll 1
      for (int o = 1; o < share.n; ++o) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float* x = KVs + r * (NC + 2) * kThreads;
          const float mo = Share::of(x, 0, o), top = fmaxf(m[r], mo), base = top == -INFINITY ? 0.f : top;
          const float keep = exp2f(m[r] - base), add = exp2f(mo - base);
          sum[r] = sum[r] * keep + Share::of(x, 1, o) * add;
          m[r] = top;
#pragma unroll
          for (int n = 0; n < NC; ++n) acc[r][n] = acc[r][n] * keep + Share::of(x, 2 + n, o) * add;
        }
      }
    }
    cluster_sync();                     // the others' memory has been read
    if (share.rank > 0) return;
  }
  float inv[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    inv[r] = sum[r] > 0.f ? 1.f / sum[r] : (sum[r] == 0.f ? 0.f : sum[r]);   // a NaN row stays NaN
    const int l = q0 + 4 * ty + r;
    if (tx == 0 && l < p.L) p.lse[int64_t(bh) * p.L + l] = sum[r] == 0.f ? -INFINITY : m[r] * kLn2 + logf(sum[r]);
  }
  store_rows<T, NC>(p.o, p, acc, inv, b, h, q0, ty, tx);
}

// ---------------------------------------------------------------- backward
// KV false: rows are queries (X = Q, Y = dO) walking keys (U = K, W = V):
//   dQ = sum dS U, and D += sum dS.  D comes from the stored O: where that is
//   bf16, sum P U (under a cap with its derivative) times the sum of dS is taken
//   off dQ, which its rounding would enter (2 x 1000 causal tokens, 8 heads of
//   36: 280 -> 316 us backward).
// KV true: rows are keys (X = K, Y = V) walking the queries of every head of
// the group (U = Q, W = dO): dV = sum P^T W, dK = sum dS^T U, and the partial
// table gradients of this tile.
template <typename T, int NC, bool KV>
__global__ void __launch_bounds__(kThreads, NC <= 4 ? 2 : 1) scored_bwd_k(const __grid_constant__ ScoredParams p) {
  extern __shared__ __align__(16) float sm[];
  constexpr int WD = 16 * NC;
  constexpr int kTile = WD * kT;
  float *X = sm, *Y = X + kTile, *UWs = Y + kTile, *P = UWs + 4 * kTile;        // UWs: two pairs of U and W
  float* bias = P + kT * kT;
  float* dist = bias + kBiasPart;                  // KV true: table gradient by distance
  float* far = dist + kBiasPart;                   // [2][128] sums beyond the reach
  pdl_wait();
  pdl_trigger();
  const int heads = KV ? p.KV : p.H, tiles = (p.L + kT - 1) / kT;
  const Share share(p.share);
  const unsigned work = blockIdx.x / unsigned(share.n);
  const int bh = work % (p.B * heads), slot = int(work / (p.B * heads));
  const int tile = KV ? slot : tiles - 1 - slot, r0 = tile * kT;
  const int b = bh / heads, h0 = KV ? (bh % heads) * p.G : bh % heads, kh = h0 / p.G;
  const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
  const bool grad = KV && p.dtable;
  constexpr bool kFix = !KV && sizeof(T) == 2;
  load_tile<T>(X, KV ? p.k : p.q, p, b, KV ? kh : h0, r0);
  load_tile<T>(Y, KV ? p.v : p.dout, p, b, KV ? kh : h0, r0);
  for (int e = 0; e < 4; ++e) clear_tail(UWs + e * kTile, p.D, WD);
  float lo = 0.f, hi = 0.f;                        // sums of this thread's diagonals beyond the reach
  float eps[4] = {0.f, 0.f, 0.f, 0.f};             // row sums of dS
  float acc0[4][NC] = {}, acc1[4][NC] = {};
  for (int g = 0; g < (KV ? p.G : 1); ++g) {
    const int h = h0 + g;
    Pair pc = pair_of(p, b, h);
    ids_of(pc.row_id, pc, r0 + 4 * ty);
    const float* lse2 = p.lse2 + (int64_t(b) * p.H + h) * p.Lp;
    const float* delta = p.delta + (int64_t(b) * p.H + h) * p.Lp;
    auto load = [&](int buf, int c0) {
      load_tile<T>(UWs + 2 * buf * kTile, KV ? p.q : p.k, p, b, KV ? h : kh, c0);
      load_tile<T>(UWs + (2 * buf + 1) * kTile, KV ? p.dout : p.v, p, b, KV ? h : kh, c0);
    };
    int cls = 0, cls_next = 0, buf = 0;
    int c0 = share.skip<KV>(p, pc.pf, b, r0, 0, &cls, (share.rank + g) % share.n);
    __syncthreads();
    if (c0 < p.L) load(0, c0);
    copies_commit();
    load_bias<T>(bias, p, h);
    if (grad) {
      for (int e = threadIdx.x; e < 2 * p.reach + 1; e += kThreads) dist[e] = 0.f;
      lo = hi = 0.f;
    }
    for (; c0 < p.L;) {
      const int c1 = share.skip<KV>(p, pc.pf, b, r0, c0 + kT, &cls_next, share.n - 1);
      if (c1 < p.L) load(buf ^ 1, c1);
      copies_commit();
      copies_wait<1>();
      __syncthreads();
      const float *U = UWs + 2 * buf * kTile, *W = U + kTile;
      float s[4][4], dp[4][4];
      scores(s, X, U, p.D, ty, tx);
      scores(dp, Y, W, p.D, ty, tx);
      if (cls == kScoredSome) ids_of(pc.col_id, pc, c0 + 4 * tx);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float ds[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = r0 + 4 * ty + r, col = c0 + 4 * tx + c, i = KV ? col : row, j = KV ? row : col;
          const bool ok = cls == kScoredAll || pair_allowed(p, pc, i, j, r, c);
          float chain;
          const float z = pair_score(p, pc, bias, s[r][c], i, j, &chain);
          s[r][c] = ok ? exp2f(fmaf(z, kLog2e, lse2[i])) : 0.f;
          ds[r] = ok ? s[r][c] * (dp[r][c] + delta[i]) : 0.f;
          eps[r] += ds[r];
          dp[r][c] = ds[r] * chain;
          if (kFix) s[r][c] = ok ? s[r][c] * chain : 0.f;
        }
        if (grad) *reinterpret_cast<float4*>(P + at_p(4 * tx + c, ty)) = make_float4(ds[0], ds[1], ds[2], ds[3]);
      }
      if (grad) {
        // each of 127 threads sums one diagonal of the tile of dS in row order
        __syncthreads();
        if (threadIdx.x < 2 * kT - 1) {
          const int e = int(threadIdx.x) - (kT - 1);             // row - column
          float t = 0.f;
#pragma unroll 8
          for (int r = max(0, e); r < min(kT, kT + e); ++r) t += P[at_p(r - e, r >> 2) + (r & 3)];
          const int d = r0 - c0 + e;
          if (d <= -p.reach) lo += t;
          else if (d >= p.reach) hi += t;
          else dist[d + p.reach] += t;
        }
        __syncthreads();
      }
      if (KV || kFix) {
        put_tile(P, s, ty, tx);
        __syncthreads();
        accumulate<NC>(acc0, P, KV ? W : U, ty, tx);
        __syncthreads();
      }
      put_tile(P, dp, ty, tx);
      __syncthreads();
      accumulate<NC>(acc1, P, U, ty, tx);
      __syncthreads();
      c0 = c1;
      cls = cls_next;
      buf ^= 1;
    }
    copies_wait<0>();
    if (grad) {
      __syncthreads();
      if (threadIdx.x < 128) {
        far[threadIdx.x] = lo;
        far[128 + threadIdx.x] = hi;
      }
      __syncthreads();
      if (threadIdx.x < 2) {
        float t = 0.f;
        for (int e = 0; e < 128; ++e) t += far[128 * threadIdx.x + e];
        dist[threadIdx.x ? 2 * p.reach : 0] += t;
      }
      __syncthreads();
      const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
      const int64_t n = int64_t(p.B) * tiles * share.n;
      for (int k = warp; k < p.buckets; k += kThreads / 32) {
        float t = 0.f;
        for (int e = lane; e < 2 * p.reach + 1; e += 32)
          if (p.map[e] == k) t += dist[e];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
        if (lane == 0) p.part[(int64_t(h) * p.buckets + k) * n + (int64_t(b) * tiles + tile) * share.n + share.rank] = t;
      }
    }
  }
  if (share.n > 1) {
    __syncthreads();
    constexpr int kEach = KV ? 2 * NC : kFix ? 2 * NC + 1 : NC + 1;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float* x = UWs + r * kEach * kThreads + threadIdx.x;
#pragma unroll
      for (int n = 0; n < NC; ++n) {
        x[n * kThreads] = acc1[r][n];
        if (KV || kFix) x[(NC + n) * kThreads] = acc0[r][n];
      }
      if (!KV) x[(kEach - 1) * kThreads] = eps[r];
    }
    cluster_sync();
    if (share.rank == 0) {
#pragma unroll 1
      for (int o = 1; o < share.n; ++o) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float* x = UWs + r * kEach * kThreads;
#pragma unroll
          for (int n = 0; n < NC; ++n) {
            acc1[r][n] += Share::of(x, n, o);
            if (KV || kFix) acc0[r][n] += Share::of(x, NC + n, o);
          }
          if (!KV) eps[r] += Share::of(x, kEach - 1, o);
        }
      }
    }
    cluster_sync();                     // the others' memory has been read
    if (share.rank > 0) return;
  }
  const float one[4] = {1.f, 1.f, 1.f, 1.f}, sc[4] = {p.scale, p.scale, p.scale, p.scale};
  if (KV) {
    store_rows<T, NC>(p.dv, p, acc0, one, b, kh, r0, ty, tx);
    store_rows<T, NC>(p.dk, p, acc1, sc, b, kh, r0, ty, tx);
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) eps[r] += __shfl_xor_sync(0xffffffffu, eps[r], o);
      if (kFix) {
#pragma unroll
        for (int n = 0; n < NC; ++n) acc1[r][n] = fmaf(-eps[r], acc0[r][n], acc1[r][n]);
      }
      const int l = r0 + 4 * ty + r;
      if (tx == 0 && l < p.L) p.delta[(int64_t(b) * p.H + h0) * p.Lp + l] -= eps[r];
    }
    store_rows<T, NC>(p.dq, p, acc1, sc, b, h0, r0, ty, tx);
  }
}

// Blocks of `smem` bytes that an SM holds (228 KB with 1 KB reserved for each);
// registers allow two up to head width 64 and one above.  The backward passes
// with a table at widths 33 to 64 do not fit twice: taken for two, 2 x 200
// tokens, 8 heads of 64, took 134 us instead of 107, and 1000 causal ones 337
// instead of 260.
int per_sm(size_t smem, int NC) { return NC <= 4 && 2 * (smem + 1024) <= 233472 ? 2 : 1; }

// How many blocks share a tile of rows (Share): twice as many while the grid
// still fits the SMs.  4 sequences of 200 tokens, 4 heads of 32, took 25.6 /
// 93.9 us forward / backward with a block each and take 23.5 / 73.7.  With a
// causal mask, whose tiles of rows differ in length, up to twice what fits: the
// longest are half as long and start first (2 x 1000 causal tokens, 8 heads of
// 64: 145 / 544 us -> 102 / 314); equal tiles only pay for it (16 x 128
// tokens, 8 heads of 64: 32.8 / 175 us against 38.9 / 235).
int shared_by(const ScoredParams& p, int64_t blocks, int64_t tiles, int per) {
  const int64_t sms = elementwise_blocks(INT64_MAX / 2, kThreads) / 8, room = sms * per * (p.causal ? 2 : 1);
  int n = 1;
  while (n < kMaxShare && 2 * n <= tiles && 2 * n * blocks <= room) n *= 2;
  return n;
}

template <typename T, int NC>
cudaError_t forward_width(ScoredParams p, cudaStream_t st) {
  const int64_t tiles = ceil_div(p.L, kT);
  const size_t smem = (size_t(5 * 16 * NC * kT) + kT * kT + (p.table ? kBiasPart : 0)) * sizeof(float);
  static std::atomic<bool> allowed[kMaxDevices];
  const cudaError_t e = allow_smem(scored_fwd_k<T, NC>, allowed);
  if (e != cudaSuccess) return e;
  p.share = shared_by(p, tiles * p.B * p.H, tiles, per_sm(smem, NC));
  return launch_cluster(scored_fwd_k<T, NC>, tiles * p.B * p.H, kThreads, smem, p.share, st, p);
}
template <typename T, int NC>
cudaError_t backward_width(ScoredParams& p, cudaStream_t st) {
  const int64_t tiles = ceil_div(p.L, kT);
  // the query pass needs the bias, the key pass the table gradient as well
  const size_t tile_bytes = (size_t(6 * 16 * NC * kT) + kT * kT) * sizeof(float);
  const size_t queries = tile_bytes + (p.table ? kBiasPart * sizeof(float) : 0);
  const size_t keys = tile_bytes + (p.table ? (kBiasPart + (p.dtable ? kGradPart : 0)) * sizeof(float) : 0);
  static std::atomic<bool> allowed[2][kMaxDevices];
  cudaError_t e = allow_smem(scored_bwd_k<T, NC, false>, allowed[0]);
  if (e == cudaSuccess) e = allow_smem(scored_bwd_k<T, NC, true>, allowed[1]);
  if (e != cudaSuccess) return e;
  p.share = shared_by(p, tiles * p.B * p.H, tiles, per_sm(queries, NC));
  e = launch_cluster(scored_bwd_k<T, NC, false>, tiles * p.B * p.H, kThreads, queries, p.share, st, p);
  if (e != cudaSuccess) return e;
  p.share = shared_by(p, tiles * p.B * p.KV, tiles, per_sm(keys, NC));
  return launch_cluster(scored_bwd_k<T, NC, true>, tiles * p.B * p.KV, kThreads, keys, p.share, st, p);
}
// Accumulator columns per thread: 16 NC >= head width.
template <typename T>
cudaError_t forward_simt(const ScoredParams& p, cudaStream_t st) {
  return p.D <= 32 ? forward_width<T, 2>(p, st) : p.D <= 64 ? forward_width<T, 4>(p, st) : forward_width<T, 8>(p, st);
}
template <typename T>
cudaError_t backward_simt(ScoredParams& p, cudaStream_t st) {
  return p.D <= 32 ? backward_width<T, 2>(p, st)
                   : p.D <= 64 ? backward_width<T, 4>(p, st) : backward_width<T, 8>(p, st);
}

// ------------------------------------------------------------- host checks
int bad(const std::string& what) { return report_error(FO_ERR_ARG, what); }
int cuda_error(cudaError_t e) { return report_error(FO_ERR_CUDA, cudaGetErrorString(e)); }

constexpr int64_t kMaxLen = 1 << 20, kMaxTiles = 1 << 27;

int check_spec(const fo_attention_spec* s) {
  if (!s) return bad("attention: null spec");
  if (s->batch < 0 || s->len < 0 || s->len > kMaxLen) return bad("attention: batch or len out of range");
  if (s->heads < 1 || s->kv_heads < 1 || s->heads % s->kv_heads) return bad("attention: heads must be a multiple of kv_heads");
  if (s->head_dim < 1 || s->head_dim > 128) return bad("attention: head_dim must be 1..128");
  if (s->dtype != FO_DTYPE_F32 && s->dtype != FO_DTYPE_BF16) return bad("attention: unknown dtype");
  if (!(s->scale > 0.f) || !std::isfinite(s->scale)) return bad("attention: scale must be positive and finite");
  if (!(s->softcap >= 0.f) || !std::isfinite(s->softcap)) return bad("attention: softcap must be finite and not negative");
  if (s->prefix && !s->causal) return bad("attention: a prefix needs the causal mask");
  if (s->table && s->slopes) return bad("attention: one of slopes and table");
  if (s->table) {
    if (!s->bucket_of_host || s->buckets < 1 || s->buckets > 128) return bad("attention: buckets must be 1..128, with their map");
    if (s->reach < 1 || s->reach > kMaxReach) return bad("attention: reach must be 1.." + std::to_string(kMaxReach));
    for (int e = 0; e < 2 * s->reach + 1; ++e)
      if (s->bucket_of_host[e] >= s->buckets) return bad("attention: bucket map entry " + std::to_string(e) + " is not below buckets");
  }
  // one grid dimension holds every tile of 64 tokens, and every 8 rows, of every sequence and head
  const int64_t tiles = (int64_t(s->len) + kT - 1) / kT, bh = int64_t(s->batch) * s->heads;
  if (tiles && bh > kMaxTiles / tiles) return bad("attention: more than 2^27 tiles of 64 tokens");
  return FO_OK;
}

int check_tensor(const fo_strided* t, const fo_attention_spec* s, int heads, bool out, const char* name) {
  const size_t size = s->dtype == FO_DTYPE_F32 ? 4 : 2;
  if (!t || !t->data) return bad(std::string("attention: null ") + name);
  if (reinterpret_cast<uintptr_t>(t->data) % size) return bad(std::string("attention: misaligned ") + name);
  const int64_t st[3] = {t->batch_stride, t->token_stride, t->head_stride};
  const int64_t n[3] = {s->batch, s->len, heads};
  int64_t extent = s->head_dim;        // elements that the dimensions seen so far span
  int order[3] = {0, 1, 2};
  std::sort(order, order + 3, [&](int x, int y) { return st[x] < st[y]; });
  for (int e : order) {
    if (n[e] <= 1) continue;
    // what is written: each dimension steps over all of the smaller ones
    if (st[e] < 0 || st[e] > (int64_t(1) << 40) || (out && st[e] < extent))
      return bad(std::string("attention: strides of ") + name);
    extent += (n[e] - 1) * st[e];
  }
  return FO_OK;
}

Strided strided(const fo_strided* t) {
  return Strided{t->data, t->batch_stride, t->token_stride, t->head_stride};
}

// The tensor-core kernels need 16-byte rows: 8-element multiples of the head
// width, of every stride in use, and an aligned base.
bool wide(const fo_strided* t, const fo_attention_spec* s, int heads) {
  const int64_t st[3] = {t->batch_stride, t->token_stride, t->head_stride};
  const int64_t n[3] = {s->batch, s->len, heads};
  for (int e = 0; e < 3; ++e)
    if (n[e] > 1 && (st[e] % 8 || st[e] < 8)) return false;
  return reinterpret_cast<uintptr_t>(t->data) % 16 == 0;
}

// They also hold biases in units of the scale and the scale in units of the
// cap, which has to stay within fp32's range.
bool ordinary(const fo_attention_spec* s) {
  auto within = [](float x) { return x >= 0x1p-60f && x <= 0x1p60f; };
  return within(s->scale) && (s->softcap == 0.f || within(s->softcap));
}

struct Layout {
  int64_t doc = 0, blk = 0, lse2 = 0, delta = 0, part = 0, bytes = 0;
};
// `part` is sized for the smaller (64-row) tiles of the CUDA-core kernels and
// the blocks that may share one.
Layout layout(const fo_attention_spec* s, bool backward) {
  Layout a;
  auto take = [&a](int64_t bytes) {
    const int64_t at = a.bytes;
    a.bytes += (bytes + 255) / 256 * 256;
    return at;
  };
  const int64_t Lp = (int64_t(s->len) + 127) / 128 * 128, B = s->batch, H = s->heads;
  if (s->documents) {
    a.doc = take(B * Lp * 4);
    a.blk = take(B * (Lp / kScoredBlock) * 8);
  }
  if (backward) {
    a.lse2 = take(B * H * Lp * 4);
    a.delta = take(B * H * Lp * 4);
    const int64_t tiles = (int64_t(s->len) + kT - 1) / kT;
    if (s->table) a.part = take(H * s->buckets * B * tiles * std::min<int64_t>(tiles, kMaxShare) * 4);
  }
  return a;
}

ScoredParams params(const fo_attention_spec* s, const Layout& a, char* ws, bool backward) {
  ScoredParams p = {};
  p.B = s->batch;
  p.L = s->len;
  p.Lp = (s->len + 127) / 128 * 128;
  p.H = s->heads;
  p.KV = s->kv_heads;
  p.G = s->heads / s->kv_heads;
  p.D = s->head_dim;
  p.causal = s->causal != 0;
  p.scale = s->scale;
  p.cap = s->softcap;
  p.slopes = s->slopes;
  p.table = s->table;
  p.prefix = s->prefix;
  if (s->table) {
    p.buckets = s->buckets;
    p.reach = s->reach;
    for (int e = 0; e < 2 * s->reach + 1; ++e) p.map[e] = s->bucket_of_host[e];
  }
  if (s->documents) {
    p.ids = s->documents;
    p.doc = reinterpret_cast<int32_t*>(ws + a.doc);
    p.blk = reinterpret_cast<int2*>(ws + a.blk);
  }
  if (backward) {
    p.lse2 = reinterpret_cast<float*>(ws + a.lse2);
    p.delta = reinterpret_cast<float*>(ws + a.delta);
    p.part = reinterpret_cast<float*>(ws + a.part);
  }
  return p;
}

int check_workspace(const Layout& a, const void* ws, int64_t bytes) {
  if (a.bytes == 0) return FO_OK;
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 256) return bad("attention: null or misaligned workspace");
  if (bytes < a.bytes) return bad("attention: workspace of " + std::to_string(bytes) + " bytes, " + std::to_string(a.bytes) + " needed");
  return FO_OK;
}

}  // namespace
}  // namespace fo

using namespace fo;

extern "C" {

int64_t fo_attention_workspace(const fo_attention_spec* spec, int backward) {
  if (check_spec(spec) != FO_OK) return -1;
  return layout(spec, backward != 0).bytes;
}

int fo_attention_forward(const fo_attention_spec* spec, const fo_strided* q, const fo_strided* k, const fo_strided* v,
                         const fo_strided* o, float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check_spec(spec);
  if (rc != FO_OK) return rc;
  if (spec->batch == 0 || spec->len == 0) return FO_OK;
  if ((rc = check_tensor(q, spec, spec->heads, false, "q")) || (rc = check_tensor(k, spec, spec->kv_heads, false, "k")) ||
      (rc = check_tensor(v, spec, spec->kv_heads, false, "v")) || (rc = check_tensor(o, spec, spec->heads, true, "o")))
    return rc;
  if (!lse) return bad("attention: null lse");
  const Layout a = layout(spec, false);
  if ((rc = check_workspace(a, workspace, workspace_bytes))) return rc;
  ScoredParams p = params(spec, a, static_cast<char*>(workspace), false);
  p.q = strided(q);
  p.k = strided(k);
  p.v = strided(v);
  p.o = strided(o);
  p.lse = lse;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  const int64_t runs = int64_t(p.B) * (p.Lp / kScoredBlock);
  if (p.ids) e = launch_k(scored_docs_k, dim3(unsigned((runs + 3) / 4)), dim3(128), 0, st, p);
  bool tc = spec->dtype == FO_DTYPE_BF16 && p.D % 8 == 0 && ordinary(spec) && wide(q, spec, p.H) &&
            wide(k, spec, p.KV) && wide(v, spec, p.KV) && wide(o, spec, p.H);
  if (e == cudaSuccess && tc) e = scored_fwd_tc(p, st, &tc);
  if (e == cudaSuccess && !tc) e = spec->dtype == FO_DTYPE_F32 ? forward_simt<float>(p, st) : forward_simt<bf16>(p, st);
  return e == cudaSuccess ? FO_OK : cuda_error(e);
}

int fo_attention_backward(const fo_attention_spec* spec, const fo_strided* q, const fo_strided* k, const fo_strided* v,
                          const fo_strided* o, const float* lse, const fo_strided* dout, const fo_strided* dq,
                          const fo_strided* dk, const fo_strided* dv, void* dtable, void* workspace,
                          int64_t workspace_bytes, void* stream) {
  int rc = check_spec(spec);
  if (rc != FO_OK) return rc;
  if (dtable && !spec->table) return bad("attention: dtable without a table");
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool f32 = spec->dtype == FO_DTYPE_F32;
  if (spec->batch == 0 || spec->len == 0) {
    if (!dtable) return FO_OK;
    cudaError_t e = cudaMemsetAsync(dtable, 0, size_t(spec->heads) * spec->buckets * (f32 ? 4 : 2), st);
    return e == cudaSuccess ? FO_OK : cuda_error(e);
  }
  if ((rc = check_tensor(q, spec, spec->heads, false, "q")) || (rc = check_tensor(k, spec, spec->kv_heads, false, "k")) ||
      (rc = check_tensor(v, spec, spec->kv_heads, false, "v")) || (rc = check_tensor(o, spec, spec->heads, false, "o")) ||
      (rc = check_tensor(dout, spec, spec->heads, false, "dout")) ||
      (rc = check_tensor(dq, spec, spec->heads, true, "dq")) ||
      (rc = check_tensor(dk, spec, spec->kv_heads, true, "dk")) ||
      (rc = check_tensor(dv, spec, spec->kv_heads, true, "dv")))
    return rc;
  if (!lse) return bad("attention: null lse");
  const Layout a = layout(spec, true);
  if ((rc = check_workspace(a, workspace, workspace_bytes))) return rc;
  ScoredParams p = params(spec, a, static_cast<char*>(workspace), true);
  p.q = strided(q);
  p.k = strided(k);
  p.v = strided(v);
  p.o = strided(o);
  p.dout = strided(dout);
  p.dq = strided(dq);
  p.dk = strided(dk);
  p.dv = strided(dv);
  p.lse = const_cast<float*>(lse);
  p.dtable = dtable;
  const int64_t rows = int64_t(p.B) * p.H * p.Lp;
  const bool vec = !f32 && p.D % 8 == 0 && wide(o, spec, spec->heads) && wide(dout, spec, spec->heads);
  const int lanes = p.D <= 32 ? 8 : p.D <= 64 ? (vec ? 8 : 16) : vec ? 16 : 32;
  const unsigned blocks = unsigned((rows + 8 * (32 / lanes) - 1) / (8 * (32 / lanes)));
  const int64_t runs = p.ids ? int64_t(p.B) * (p.Lp / kScoredBlock) : 0;
  auto delta = f32 ? scored_delta_k<float, false> : vec ? scored_delta_k<bf16, true> : scored_delta_k<bf16, false>;
  cudaError_t e = launch_k(delta, dim3(blocks + unsigned((runs + 7) / 8)), dim3(256), 0, st, p, lanes, blocks);
  bool tc = vec && ordinary(spec) && wide(q, spec, p.H) && wide(k, spec, p.KV) && wide(v, spec, p.KV) &&
            wide(dq, spec, p.H) && wide(dk, spec, p.KV) && wide(dv, spec, p.KV);
  if (e == cudaSuccess && tc) e = scored_bwd_tc(p, st, &tc);
  if (e == cudaSuccess && !tc) e = f32 ? backward_simt<float>(p, st) : backward_simt<bf16>(p, st);
  if (e == cudaSuccess && dtable) {
    const int n = p.H * p.buckets;
    const int64_t parts = int64_t(p.B) * ceil_div(p.L, tc ? 128 : kT) * p.share;     // of the kernel that ran
    e = f32 ? launch_k(scored_table_k<float>, dim3((n + 3) / 4), dim3(128), 0, st, p.part, static_cast<float*>(dtable),
                       n, parts)
            : launch_k(scored_table_k<bf16>, dim3((n + 3) / 4), dim3(128), 0, st, p.part, static_cast<bf16*>(dtable),
                       n, parts);
  }
  return e == cudaSuccess ? FO_OK : cuda_error(e);
}

int fo_attention_error(void* stream) {
  static thread_local unsigned told[kMaxDevices][2];     // what this thread has reported
  int dev = 0, fwd = 0, bwd = 0;
  cudaError_t e = cudaStreamSynchronize(static_cast<cudaStream_t>(stream));
  if (e == cudaSuccess) e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = scored_fwd_error(&told[dev % kMaxDevices][0], &fwd);
  if (e == cudaSuccess) e = scored_bwd_error(&told[dev % kMaxDevices][1], &bwd);
  if (e != cudaSuccess) return cuda_error(e);
  if (!fwd && !bwd) return FO_OK;
  return report_error(FO_ERR_TIMEOUT, "an attention kernel timed out waiting (code " + std::to_string(fwd ? fwd : bwd) + ")");
}

}  // extern "C"
