// Pieces shared by the tensor-core kernels of scored attention
// (k_scored_fwd.cu, k_scored_bwd.cu): bounded waits, the list of blocks a tile
// walks, tensor maps and fast exponentials.
#pragma once
#include "fo_common.cuh"
#include "fo_ptx.cuh"
#include "fo_scored.h"
#include "fo_tc.h"

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
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// A role's waits: after one has given up (about two seconds) the rest return
// at once, so the kernel ends soon and its error word is set.
struct Waits {
  int* err;
  bool dead = false;
  __device__ __forceinline__ explicit Waits(int* e) : err(e) {}
  __device__ __forceinline__ void on(uint64_t* bar, uint32_t parity, int code) {
    if (dead || mbar_wait(bar, parity)) return;
    atomicExch(err, code);
    dead = true;
  }
  // The same for a whole warp, which stays converged and agrees on the outcome.
  __device__ __forceinline__ void on_warp(uint64_t* bar, uint32_t parity, int code) {
    if (!dead && !mbar_wait(bar, parity)) {
      atomicExch(err, code);
      dead = true;
    }
    dead = __any_sync(0xffffffffu, dead);
  }
};

// Walks the set bits of a bitmap in shared memory in ascending order.
struct Bits {
  const uint32_t *a, *b;    // the union of two maps (b may equal a)
  int words, w;
  uint32_t left;
  __device__ __forceinline__ Bits(const uint32_t* a_, const uint32_t* b_, int words_)
      : a(a_), b(b_), words(words_), w(0), left(words_ > 0 ? a_[0] | b_[0] : 0u) {}
  // The next block, or -1.
  __device__ __forceinline__ int next() {
    while (!left) {
      if (++w >= words) return -1;
      left = a[w] | b[w];
    }
    const int bit = __ffs(int(left)) - 1;
    left &= left - 1;
    return 32 * w + bit;
  }
};
__device__ __forceinline__ bool bit_of(const uint32_t* map, int i) { return (map[i >> 5] >> (i & 31)) & 1u; }

// Clears the rows of padded tokens of a swizzled tile of `rows` rows and
// `subs` 64-column sub-tiles (a whole warp; a row's swizzled units stay within
// its 128 bytes), so that what they hold meets no product as an operand summed
// over tokens.
__device__ __forceinline__ void clear_padding(char* tile, int rows, int subs, const int32_t* doc, int l0, int L) {
  const int lane = threadIdx.x % 32;
  for (int r = lane; r < rows; r += 32)
    if (l0 + r < L && doc[l0 + r] < 0)
      for (int s = 0; s < subs; ++s)
#pragma unroll
        for (int u = 0; u < 8; ++u) st_shared4(smem_u32(tile) + s * rows * 128 + r * 128 + u * 16, 0u, 0u, 0u, 0u);
  fence_proxy_async_smem();
  __syncwarp();
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
