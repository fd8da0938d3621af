// Scored attention: attention whose scores are capped by a tanh, biased by
// distance (a slope per head, or a learned table indexed by distance buckets)
// and masked by causality, a visible prefix and document ids.  Shared by the
// entry points and the CUDA-core kernels (k_scored.cu) and the tensor-core
// kernels (k_scored_fwd.cu, k_scored_bwd.cu).
//
// For query i and key j of one sequence and head (d = j - i):
//   z_ij = scale q_i . k_j;  with a cap c:  z_ij <- c tanh(z_ij / c)
//   z_ij <- z_ij - slope_h |d|   or   z_ij + table[h][buckets[clamp(d, -R, R) + R]]
//   P = softmax over the allowed j, O = P V, lse_i = log sum_j exp z_ij
// and backward, with D_i = sum_d dO_id O_id:
//   dV = P^T dO,  dP = dO V^T,  dS = P (dP - D),
//   dtable[h][b] = sum over pairs of bucket b of dS,
//   dS <- dS (1 - tanh^2),  dQ = scale dS K,  dK = scale dS^T Q
// (dK and dV summed over the query heads that share a key head).
#pragma once
#include <cuda_runtime.h>

#include <atomic>
#include <cstddef>
#include <cstdint>

namespace fo {

constexpr int kMaxReach = 512;       // largest |distance| with a bucket of its own
constexpr int kScoredBlock = 64;     // tokens per entry of the document summary
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

struct Strided {
  void* p;
  int64_t sb, sl, sh;   // batch, token and head strides in elements
};

// Everything a kernel needs besides its tensor maps; passed by value.
struct ScoredParams {
  Strided q, k, v, o, dout, dq, dk, dv;
  float* lse;              // [B][H][L], -inf for a row that allows no key
  // workspace
  int32_t* doc;            // [B][Lp] document ids, -1 past the sequence; null without documents
  int2* blk;               // [B][Lp / 64] summary of each 64 ids (see doc_summary)
  float* lse2;             // [B][H][Lp] -lse * log2(e), -inf where P is zero
  float* delta;            // [B][H][Lp] -D
  float* part;             // [H][buckets][B * key tiles * share] partial table gradients
  const float* slopes;     // [H] or null
  const void* table;       // [H][buckets] in the tensors' type, or null
  const int32_t* prefix;   // [B] or null
  const int32_t* ids;      // [B][L] document ids as given, or null
  void* dtable;
  int B, L, Lp, H, KV, G, D;
  int causal, buckets, reach;
  int stages;              // shared-memory stages of the backward tensor-core kernels
  int share;               // blocks (a cluster) that share a tile of rows
  float scale, cap;
  uint8_t map[2 * kMaxReach + 1];
};

constexpr int kMaxShare = 8;      // the portable cluster size

enum { kScoredNone = 0, kScoredAll = 1, kScoredSome = 2 };

#ifdef __CUDACC__
// A table's entry as a bias: finite ones end at +-2^15.  Beside a key of
// ordinary score the probability is 0 (or 1) all the same; but a row of nothing
// but keys masked by -1e9 or the type's lowest value would lose its scores in
// the bias's rounding forward, and backward, where P comes from lse, give
// anything from 0 to infinity.
__device__ __forceinline__ float bias_of(float t) {
  constexpr float kEnd = 32768.f;
  return fabsf(t) > kEnd && !isinf(t) ? copysignf(kEnd, t) : t;
}

// Sets a kernel's shared-memory limits the first time it is launched on the
// current device (`done`: one flag per device, static in the launcher).
constexpr int kMaxDevices = 64;
constexpr int kSmemLimit = 232448;      // 227 KB per block
template <typename K>
cudaError_t allow_smem(K kernel, std::atomic<bool> (&done)[kMaxDevices]) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 0 && dev < kMaxDevices && done[dev]) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, int(cudaSharedmemCarveoutMaxShared));
  if (e == cudaSuccess && dev >= 0 && dev < kMaxDevices) done[dev] = true;
  return e;
}

// Launches `blocks` clusters of `share` blocks.
template <typename K, typename P>
cudaError_t launch_cluster(K kernel, int64_t blocks, int threads, size_t smem, int share, cudaStream_t st, const P& p) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(blocks * share));
  cfg.blockDim = dim3(unsigned(threads));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = unsigned(share);
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl_enabled() ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}
// Every thread of the cluster has come here, and sees what the others wrote.
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Summary of a run of document ids: x the smallest id >= 0 (INT_MAX when there
// is none) with its sign bit set when the run holds padding, y the largest id.
__device__ __forceinline__ int2 doc_join(int2 a, int2 b) {
  const int x = min(a.x & 0x7fffffff, b.x & 0x7fffffff) | ((a.x | b.x) & 0x80000000);
  return make_int2(x, max(a.y, b.y));
}
// Whether none, all or some of the pairs of queries [q0, q1) and keys [k0, k1)
// are allowed (conservative towards "some"); pf is the sequence's prefix.
__device__ __forceinline__ int scored_class(const ScoredParams& p, int pf, int q0, int q1, int k0, int k1, bool docs,
                                            int2 qd, int2 kd) {
  bool all = true;
  if (p.causal) {
    if (k0 > q1 - 1 && k0 >= pf) return kScoredNone;
    all = k1 - 1 <= q0 || k1 <= pf;
  }
  if (docs) {
    const int qm = qd.x & 0x7fffffff, km = kd.x & 0x7fffffff;
    if (max(qm, km) > min(qd.y, kd.y)) return kScoredNone;
    all = all && qd.x >= 0 && kd.x >= 0 && qm == qd.y && km == kd.y && qm == km;
  }
  return all ? kScoredAll : kScoredSome;
}
#endif

// Tensor-core paths (bf16, head width a multiple of 8, 16-byte aligned rows).
// Each returns a cudaError_t; `ok` tells whether a tensor map was refused.
cudaError_t scored_fwd_tc(const ScoredParams& p, cudaStream_t st, bool* ok);
cudaError_t scored_bwd_tc(ScoredParams& p, cudaStream_t st, bool* ok);    // sets p.share
// The code of a bounded wait that gave up on the current device since `told`
// (which is brought up to date), 0 for none.
cudaError_t scored_fwd_error(unsigned* told, int* code);
cudaError_t scored_bwd_error(unsigned* told, int* code);

}  // namespace fo
