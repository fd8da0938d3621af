// Embedding lookup with scaling, and the gradient of its table.
//
//   out[t] = scale * table[id_t]                   (zeros where id_t is not in 0 .. vocab - 1)
//   dtable[v] = scale * sum over id_t = v of dout[t]
//
// The gradient sorts the tokens by id (a stable radix sort, so equal ids stay
// in the order of the tokens), walks the sorted tokens in pieces of equal
// length, and joins the sums of rows that cross pieces: every sum has a fixed
// order, and a token that fills half of the batch is shared by as many warps
// as the others.  Rows without a token are cleared by warps of the same launch.
// Both directions are bound by HBM: lookup reads the used rows and writes out,
// the gradient reads dout and writes the table's gradient.
#include "fo_vec8.cuh"
#include "../../include/fedoptima.h"

#include <string>

namespace fo {
int report_error(int code, const std::string& msg);

namespace {

// ------------------------------------------------------------------ lookup
template <typename I>
__device__ __forceinline__ int64_t row_of(const I* ids, int64_t t, int64_t vocab) {
  const int64_t v = ids[t];
  return v >= 0 && v < vocab ? v : -1;
}

// An item is 256 columns of one token; each warp has U items in flight.
template <typename I, typename S, typename T, bool VEC, int U>
__global__ void __launch_bounds__(256) lookup_k(const I* ids, const S* table, T* out, int64_t ldo, int64_t items, int chunks,
                                                int64_t vocab, int width, float scale) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x % 32;
  const int64_t warps = int64_t(gridDim.x) * (blockDim.x / 32), warp = int64_t(blockIdx.x) * (blockDim.x / 32) + threadIdx.x / 32;
  for (int64_t i0 = warp * U; i0 < items; i0 += warps * U) {
    int64_t at[U], token[U];
    int c0[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = i0 + u;
      token[u] = i < items ? i / chunks : -1;
      c0[u] = i < items ? int(i - token[u] * chunks) * 256 : 0;
      at[u] = i < items ? row_of(ids, token[u], vocab) : -1;
    }
    if constexpr (VEC) {
      Raw8<S> raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0[u] + lane * 8;
        if (at[u] >= 0 && c < width) raw[u].load(table + at[u] * width + c);
        else raw[u].zero();
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0[u] + lane * 8;
        if (token[u] < 0 || c >= width) continue;
        float v[8];
        raw[u].get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = at[u] >= 0 ? v[e] * scale : 0.f;
        store8(out + token[u] * ldo + c, v);
      }
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (token[u] < 0) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int c = c0[u] + e * 32 + lane;
          v[e] = at[u] >= 0 && c < width ? to_f(table[at[u] * width + c]) * scale : 0.f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int c = c0[u] + e * 32 + lane;
          if (c < width) out[token[u] * ldo + c] = from_f<T>(v[e]);
        }
      }
    }
  }
}

// ------------------------------------------------------------------ sorting
// Keys are ids, or `vocab` for tokens without a row, which end up last.  A
// pass orders the tokens by kDigit bits of their key and keeps the order of
// equal digits.
constexpr int kDigit = 9, kBins = 1 << kDigit;
constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32;
constexpr int kMaxSortBlocks = 152;

struct SortParams {
  const void* ids;
  int wide_ids;            // 64-bit ids
  const uint32_t *key_in, *token_in;
  uint32_t *key_out, *token_out;
  uint32_t* counts;        // [blocks][kBins] of this pass
  uint32_t vocab, n, per;  // tokens, tokens per block
  int shift;
};

__device__ __forceinline__ uint32_t sort_key(const SortParams& p, uint32_t i) {
  if (p.key_in) return p.key_in[i];
  const int64_t v = p.wide_ids ? static_cast<const int64_t*>(p.ids)[i] : int64_t(static_cast<const int32_t*>(p.ids)[i]);
  return v >= 0 && v < int64_t(p.vocab) ? uint32_t(v) : p.vocab;
}

__global__ void __launch_bounds__(kSortThreads) sort_count_k(const __grid_constant__ SortParams p) {
  __shared__ uint32_t bins[kBins];
  pdl_wait();
  pdl_trigger();
  for (int i = threadIdx.x; i < kBins; i += kSortThreads) bins[i] = 0;
  __syncthreads();
  const uint32_t first = blockIdx.x * p.per, end = min(p.n, first + p.per);
  for (uint32_t i = first + threadIdx.x; i < end; i += kSortThreads)
    atomicAdd(&bins[sort_key(p, i) >> p.shift & (kBins - 1)], 1u);
  __syncthreads();
  for (int i = threadIdx.x; i < kBins; i += kSortThreads) p.counts[blockIdx.x * kBins + i] = bins[i];
}

// Exclusive sums of one value per thread over the block, in thread order.
__device__ __forceinline__ uint32_t block_before(uint32_t v, uint32_t* box) {
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  uint32_t s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t u = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += u;
  }
  if (lane == 31) box[warp] = s;
  __syncthreads();
  uint32_t before = 0;
  for (int w = 0; w < warp; ++w) before += box[w];
  return before + s - v;
}

// Each block places its tokens behind those of smaller digits and those of the
// same digit in earlier blocks.  A warp takes 32 neighbouring tokens at a time;
// a round of the block is 32 kSortWarps of them.
__global__ void __launch_bounds__(kSortThreads) sort_place_k(const __grid_constant__ SortParams p) {
  static_assert(kBins == kSortThreads, "one bin per thread");
  __shared__ uint32_t base[kBins];
  __shared__ uint16_t mine[kSortWarps][kBins];
  __shared__ uint32_t box[kSortWarps];
  pdl_wait();
  pdl_trigger();
  const int t = threadIdx.x, lane = t % 32, warp = t / 32;
  uint32_t all = 0, before = 0;
#pragma unroll 8
  for (unsigned b = 0; b < gridDim.x; ++b) {
    const uint32_t c = p.counts[b * kBins + t];
    all += c;
    if (b < blockIdx.x) before += c;
  }
  base[t] = block_before(all, box) + before;
  const uint32_t first = blockIdx.x * p.per, end = min(p.n, first + p.per);
  for (uint32_t round = first; round < end; round += kSortThreads) {
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) mine[w][t] = 0;
    __syncthreads();
    const uint32_t i = round + t;
    const bool in = i < end;
    const uint32_t key = in ? sort_key(p, i) : 0u, digit = key >> p.shift & (kBins - 1);
    const uint32_t peers = __match_any_sync(0xffffffffu, in ? digit : uint32_t(kBins));
    const uint32_t rank = __popc(peers & ((1u << lane) - 1u));
    if (in && rank == 0) mine[warp][digit] = uint16_t(__popc(peers));
    __syncthreads();
    // the place of each warp's first token of this digit, relative to base
    uint32_t rel = 0;
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
      const uint32_t c = mine[w][t];
      mine[w][t] = uint16_t(rel);
      rel += c;
    }
    __syncthreads();
    if (in) {
      const uint32_t to = base[digit] + mine[warp][digit] + rank;
      p.key_out[to] = key;
      p.token_out[to] = p.token_in ? p.token_in[i] : i;
    }
    __syncthreads();
    base[t] += rel;
  }
}

// ------------------------------------------------------------------ sums
// A warp sums kPiece sorted tokens over 256 columns.  A row whose tokens all
// lie in one piece is written there; the others leave a sum per piece in
// `part` ([piece][first or last][width]), which join_k adds up.
constexpr int kPiece = 32;

struct GradParams {
  const void* dout;
  const uint32_t *key, *token;
  void* dtable;
  float* part;
  int64_t ldo;
  uint32_t n, vocab;
  int width, chunks, accumulate;
  float scale;
  int64_t sum_items, clear_items;
};

template <typename S, bool VEC>
__device__ __forceinline__ void write_row(const GradParams& p, uint32_t v, int c0, int lane, const float (&a)[8]) {
  S* row = static_cast<S*>(p.dtable) + int64_t(v) * p.width;
  if constexpr (VEC) {
    const int c = c0 + lane * 8;
    if (c >= p.width) return;
    float z[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = a[e] * p.scale;
    if (p.accumulate) {
      Raw8<S> old;
      old.load(row + c);
      float o[8];
      old.get(o);
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] += o[e];
    }
    store8(row + c, z);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = c0 + e * 32 + lane;
      if (c < p.width) row[c] = from_f<S>(fmaf(a[e], p.scale, p.accumulate ? to_f(row[c]) : 0.f));
    }
  }
}
template <bool VEC>
__device__ __forceinline__ float* part_at(const GradParams& p, uint32_t piece, int last, int c0, int lane) {
  return p.part + (int64_t(piece) * 2 + last) * p.chunks * 256 + c0 + lane * 8;
}

template <typename T, typename S, bool VEC>
__global__ void __launch_bounds__(256) grad_k(const __grid_constant__ GradParams p) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x % 32;
  const int64_t warps = int64_t(gridDim.x) * (blockDim.x / 32);
  for (int64_t item = int64_t(blockIdx.x) * (blockDim.x / 32) + threadIdx.x / 32; item < p.sum_items + p.clear_items; item += warps) {
    if (item >= p.sum_items) {      // 32 rows of the table: those without a token are cleared
      const uint32_t v = uint32_t(item - p.sum_items) * 32 + lane;
      uint32_t lo = 0, hi = p.n;
      while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (p.key[mid] < v) lo = mid + 1;
        else hi = mid;
      }
      uint32_t clear = __ballot_sync(0xffffffffu, v < p.vocab && (lo >= p.n || p.key[lo] != v));
      while (clear) {
        const uint32_t row = uint32_t(item - p.sum_items) * 32 + __ffs(int(clear)) - 1;
        clear &= clear - 1;
        S* d = static_cast<S*>(p.dtable) + int64_t(row) * p.width;
        if constexpr (VEC) {
          const float z[8] = {};
          for (int c = lane * 8; c < p.width; c += 256) store8(d + c, z);
        } else {
          for (int c = lane; c < p.width; c += 32) d[c] = from_f<S>(0.f);
        }
      }
      continue;
    }
    const uint32_t piece = uint32_t(item / p.chunks), first = piece * kPiece;
    const int c0 = int(item - int64_t(piece) * p.chunks) * 256;
    const uint32_t i = first + lane;
    const uint32_t my_key = i < p.n ? p.key[i] : p.vocab, my_token = i < p.n ? p.token[i] : 0u;
    const uint32_t left = first ? p.key[first - 1] : p.vocab;
    const uint32_t right = first + kPiece < p.n ? p.key[first + kPiece] : p.vocab;
    const uint32_t k0 = __shfl_sync(0xffffffffu, my_key, 0);
    if (k0 >= p.vocab) continue;    // only tokens without a row from here on
    float a[8] = {};
    uint32_t current = k0;
    bool open = left == k0;         // the row began in an earlier piece
    auto flush = [&](uint32_t next) {
      const bool on = next == p.vocab + 1u;          // the end of the piece
      const bool goes_on = on && right == current;
      if (!open && !goes_on) {
        write_row<S, VEC>(p, current, c0, lane, a);
      } else {
        float4* d = reinterpret_cast<float4*>(part_at<VEC>(p, piece, open ? 0 : 1, c0, lane));
        d[0] = make_float4(a[0], a[1], a[2], a[3]);
        d[1] = make_float4(a[4], a[5], a[6], a[7]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) a[e] = 0.f;
      open = false;
      current = next;
    };
    constexpr int kAhead = 4;
    for (int r = 0; r < kPiece; r += kAhead) {
      float v[kAhead][8];
      uint32_t key[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        key[u] = __shfl_sync(0xffffffffu, my_key, r + u);
        const uint32_t token = __shfl_sync(0xffffffffu, my_token, r + u);
        const T* d = static_cast<const T*>(p.dout) + int64_t(token) * p.ldo;
        if constexpr (VEC) {
          Raw8<T> raw;
          const int c = c0 + lane * 8;
          if (key[u] < p.vocab && c < p.width) raw.load(d + c);
          else raw.zero();
          raw.get(v[u]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int c = c0 + e * 32 + lane;
            v[u][e] = key[u] < p.vocab && c < p.width ? to_f(d[c]) : 0.f;
          }
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (key[u] >= p.vocab) break;
        if (key[u] != current) flush(key[u]);
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] += v[u][e];
      }
    }
    flush(p.vocab + 1u);
  }
}

// Rows that cross pieces: one block per piece in which such a row begins and
// 256 columns; its warps take neighbouring runs of the later pieces.
template <typename S, bool VEC>
__global__ void __launch_bounds__(256) join_k(const __grid_constant__ GradParams p) {
  __shared__ float box[8][256];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const uint32_t pieces = (p.n + kPiece - 1) / kPiece;
  const uint32_t piece = blockIdx.x;
  const int c0 = int(blockIdx.y) * 256;
  const uint32_t first = piece * kPiece, next = first + kPiece;
  if (next >= p.n) return;
  const uint32_t v = p.key[next - 1];
  if (v >= p.vocab || p.key[next] != v) return;             // its last row ends here
  if (p.key[first] == v && first && p.key[first - 1] == v) return;   // it began earlier
  // the last piece that holds the row
  uint32_t lo = piece + 1, hi = pieces - 1;
  while (lo < hi) {
    const uint32_t mid = (lo + hi + 1) / 2;
    if (p.key[mid * kPiece] == v) lo = mid;
    else hi = mid - 1;
  }
  const uint32_t count = lo - piece + 1, per = (count + 7) / 8;
  float a[8] = {};
  for (uint32_t i = warp * per; i < min(count, (warp + 1) * per); ++i) {
    const float4* d = reinterpret_cast<const float4*>(part_at<VEC>(p, piece + i, i == 0 ? 1 : 0, c0, lane));
    const float4 x = d[0], y = d[1];
    a[0] += x.x, a[1] += x.y, a[2] += x.z, a[3] += x.w, a[4] += y.x, a[5] += y.y, a[6] += y.z, a[7] += y.w;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) box[warp][e * 32 + lane] = a[e];
  __syncthreads();
  if (warp) return;
  for (int w = 1; w < 8; ++w)
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] += box[w][e * 32 + lane];
  write_row<S, VEC>(p, v, c0, lane, a);
}

// ------------------------------------------------------------------ host
int bad(const char* why) { return report_error(FO_ERR_ARG, std::string("embedding: ") + why); }
int done(cudaError_t e) { return e == cudaSuccess ? FO_OK : report_error(FO_ERR_CUDA, cudaGetErrorString(e)); }
bool known(int dtype) { return dtype == FO_DTYPE_F32 || dtype == FO_DTYPE_BF16; }
size_t size_of(int dtype) { return dtype == FO_DTYPE_F32 ? 4 : 2; }
bool odd(const void* p, size_t size) { return !p || reinterpret_cast<uintptr_t>(p) % size; }

int check(int ids_bits, int64_t tokens, int table_dtype, int dtype, int64_t vocab, int64_t width) {
  if (ids_bits != 32 && ids_bits != 64) return bad("ids have 32 or 64 bits");
  if (!known(table_dtype) || !known(dtype) || (table_dtype == FO_DTYPE_BF16 && dtype == FO_DTYPE_F32))
    return bad("tables and activations are fp32 or bf16, and fp32 activations have an fp32 table");
  if (tokens < 0 || tokens > int64_t(1) << 30) return bad("0 to 2^30 tokens");
  if (vocab < 1 || vocab > int64_t(1) << 30 || width < 1 || width > int64_t(1) << 20)
    return bad("1 to 2^30 rows of 1 to 2^20 columns");
  return FO_OK;
}

struct SortLayout {
  int64_t key[2], token[2], counts, part, bytes;
  unsigned blocks, per;
};
SortLayout layout(int64_t tokens, int64_t width) {
  SortLayout a;
  int64_t at = 0;
  auto take = [&at](int64_t bytes) {
    const int64_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  for (int i = 0; i < 2; ++i) {
    a.key[i] = take(4 * tokens);
    a.token[i] = take(4 * tokens);
  }
  const int64_t want = (tokens + 2 * kSortThreads - 1) / (2 * kSortThreads);
  a.blocks = unsigned(want < kMaxSortBlocks ? want : kMaxSortBlocks);
  a.per = unsigned((tokens + a.blocks - 1) / a.blocks);
  a.counts = take(int64_t(a.blocks) * kBins * 4);
  const int64_t pieces = (tokens + kPiece - 1) / kPiece;
  a.part = take(pieces * 2 * ((width + 255) / 256 * 256) * 4);
  a.bytes = at;
  return a;
}

template <typename I, typename S, typename T>
cudaError_t lookup(const void* ids, const void* table, void* out, int64_t ldo, int64_t tokens, int64_t vocab, int width,
                   float scale, bool vec, cudaStream_t st) {
  const int chunks = (width + 255) / 256;
  const int64_t items = tokens * chunks;
  constexpr int U = 2;
  const dim3 grid(unsigned(elementwise_blocks((items + U - 1) / U * 32, 256)));
  return launch_k(vec ? lookup_k<I, S, T, true, U> : lookup_k<I, S, T, false, U>, grid, dim3(256), 0, st,
                  static_cast<const I*>(ids), static_cast<const S*>(table), static_cast<T*>(out), ldo, items, chunks, vocab,
                  width, scale);
}
template <typename T, typename S, bool VEC>
cudaError_t gradient(const GradParams& p, cudaStream_t st) {
  const dim3 grid(unsigned(elementwise_blocks((p.sum_items + p.clear_items) * 32, 256)));
  cudaError_t e = launch_k(grad_k<T, S, VEC>, grid, dim3(256), 0, st, p);
  const unsigned pieces = unsigned((p.n + kPiece - 1) / kPiece);
  if (e == cudaSuccess && pieces > 1) e = launch_k(join_k<S, VEC>, dim3(pieces, unsigned(p.chunks)), dim3(256), 0, st, p);
  return e;
}

}  // namespace
}  // namespace fo

using namespace fo;

extern "C" {

int fo_embedding(const void* ids, int ids_bits, int64_t tokens, const void* table, int table_dtype, int64_t vocab,
                 int64_t width, double scale, void* out, int64_t out_stride, int dtype, void* stream) {
  int rc = check(ids_bits, tokens, table_dtype, dtype, vocab, width);
  if (rc || tokens == 0) return rc;
  if (odd(ids, ids_bits / 8) || odd(table, size_of(table_dtype)) || odd(out, size_of(dtype)))
    return bad("null or misaligned pointer");
  if (tokens > 1 && (out_stride < width || out_stride > INT64_MAX / 8 / tokens)) return bad("bad row stride of out");
  const bool vec = width % 8 == 0 && aligned16(table) && aligned16(out) &&
                   (tokens == 1 || out_stride % (dtype == FO_DTYPE_F32 ? 4 : 8) == 0);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  auto go = [&](auto f) { return done(f(ids, table, out, out_stride, tokens, vocab, int(width), float(scale), vec, st)); };
  if (ids_bits == 32)
    return dtype == FO_DTYPE_F32 ? go(lookup<int32_t, float, float>)
           : table_dtype == FO_DTYPE_F32 ? go(lookup<int32_t, float, bf16>) : go(lookup<int32_t, bf16, bf16>);
  return dtype == FO_DTYPE_F32 ? go(lookup<int64_t, float, float>)
         : table_dtype == FO_DTYPE_F32 ? go(lookup<int64_t, float, bf16>) : go(lookup<int64_t, bf16, bf16>);
}

int64_t fo_embedding_workspace(int64_t tokens, int64_t width) {
  if (check(32, tokens, FO_DTYPE_F32, FO_DTYPE_F32, 1, width)) return -1;
  return tokens ? layout(tokens, width).bytes : 0;
}

int fo_embedding_grad(const void* dout, int64_t dout_stride, int dtype, const void* ids, int ids_bits, int64_t tokens,
                      void* dtable, int table_dtype, int64_t vocab, int64_t width, double scale, int accumulate,
                      void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check(ids_bits, tokens, table_dtype, dtype, vocab, width);
  if (rc) return rc;
  if (odd(dtable, size_of(table_dtype))) return bad("dtable is null or misaligned");
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (tokens == 0) return accumulate ? FO_OK : done(cudaMemsetAsync(dtable, 0, size_t(vocab) * width * size_of(table_dtype), st));
  if (odd(ids, ids_bits / 8) || odd(dout, size_of(dtype))) return bad("null or misaligned pointer");
  if (tokens > 1 && (dout_stride < 0 || dout_stride > INT64_MAX / 8 / tokens)) return bad("bad row stride of dout");
  const SortLayout a = layout(tokens, width);
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 || workspace_bytes < a.bytes)
    return bad("the workspace is missing, misaligned or too small");
  char* ws = static_cast<char*>(workspace);
  SortParams s;
  s.ids = ids;
  s.wide_ids = ids_bits == 64;
  s.key_in = s.token_in = nullptr;
  s.counts = reinterpret_cast<uint32_t*>(ws + a.counts);
  s.vocab = uint32_t(vocab);
  s.n = uint32_t(tokens);
  s.per = a.per;
  int from = 1;
  for (s.shift = 0; vocab >> s.shift; s.shift += kDigit) {      // the largest key is vocab
    const int to = 1 - from;
    s.key_out = reinterpret_cast<uint32_t*>(ws + a.key[to]);
    s.token_out = reinterpret_cast<uint32_t*>(ws + a.token[to]);
    cudaError_t e = launch_k(sort_count_k, dim3(a.blocks), dim3(kSortThreads), 0, st, s);
    if (e == cudaSuccess) e = launch_k(sort_place_k, dim3(a.blocks), dim3(kSortThreads), 0, st, s);
    if (e != cudaSuccess) return done(e);
    s.key_in = s.key_out;
    s.token_in = s.token_out;
    from = to;
  }
  GradParams p;
  p.dout = dout;
  p.key = s.key_in;
  p.token = s.token_in;
  p.dtable = dtable;
  p.part = reinterpret_cast<float*>(ws + a.part);
  p.ldo = dout_stride;
  p.n = uint32_t(tokens);
  p.vocab = uint32_t(vocab);
  p.width = int(width);
  p.chunks = int((width + 255) / 256);
  p.accumulate = accumulate != 0;
  p.scale = float(scale);
  p.sum_items = (tokens + kPiece - 1) / kPiece * p.chunks;
  p.clear_items = accumulate ? 0 : (vocab + 31) / 32;
  const bool vec = width % 8 == 0 && aligned16(dtable) && aligned16(dout) &&
                   (tokens == 1 || dout_stride % (dtype == FO_DTYPE_F32 ? 4 : 8) == 0);
  if (dtype == FO_DTYPE_F32) return done(vec ? gradient<float, float, true>(p, st) : gradient<float, float, false>(p, st));
  if (table_dtype == FO_DTYPE_F32) return done(vec ? gradient<bf16, float, true>(p, st) : gradient<bf16, float, false>(p, st));
  return done(vec ? gradient<bf16, bf16, true>(p, st) : gradient<bf16, bf16, false>(p, st));
}

}  // extern "C"
