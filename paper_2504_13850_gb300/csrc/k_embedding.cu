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

#include <atomic>
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

// An item is up to 256 U columns of one token, all in flight in one warp, which
// reads the next item's id while they are: a row's address waits for its id, and
// memory for both is twice as far (65536 x 2048 bf16: 71 -> 62 us).
template <typename I, typename S, typename T, bool VEC, int U>
__global__ void __launch_bounds__(256) lookup_k(const I* ids, const S* table, T* out, int64_t ldo, int64_t items, int groups,
                                                int64_t vocab, int width, float scale) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x % 32;
  const int64_t warps = int64_t(gridDim.x) * (blockDim.x / 32);
  int64_t i = int64_t(blockIdx.x) * (blockDim.x / 32) + threadIdx.x / 32;
  if (i >= items) return;
  int64_t token = i / groups, at = row_of(ids, token, vocab);
  while (true) {
    const int c0 = int(i - token * groups) * 256 * U;
    const int64_t then = i + warps, next_token = then < items ? then / groups : token;
    const S* row = table + (at < 0 ? 0 : at) * width;
    T* to = out + token * ldo;
    const float by = scale;
    const bool fine = at >= 0;
    if constexpr (VEC) {
      Raw8<S> raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + u * 256 + lane * 8;
        if (fine && c < width) raw[u].load(row + c);
        else raw[u].zero();
      }
      at = row_of(ids, next_token, vocab);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + u * 256 + lane * 8;
        if (c >= width) break;
        float v[8];
        raw[u].get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fine ? v[e] * by : 0.f;
        store8(to + c, v);
      }
    } else {
      S loose[U][8];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) loose[u][e] = row[min(c0 + u * 256 + e * 32 + lane, width - 1)];
      at = row_of(ids, next_token, vocab);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int c = c0 + u * 256 + e * 32 + lane;
          if (c < width) to[c] = from_f<T>(fine ? to_f(loose[u][e]) * by : 0.f);
        }
    }
    if (then >= items) return;
    i = then;
    token = next_token;
  }
}

// ------------------------------------------------------------------ sorting
// Keys are ids, or `vocab` for tokens without a row, which end up last.  A
// pass orders the tokens by kDigit bits of their key and keeps the order of
// equal digits.
constexpr int kMaxDevices = 64;
constexpr int kDigit = 9, kBins = 1 << kDigit;
constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32;
constexpr int kMaxSortBlocks = 152;

// The lanes that hold this lane's digit, by a vote on each of its bits: a match of
// whole words takes a turn for each value that the warp holds (16384 tokens of
// 100000 evenly drawn ids in one block: 52 instead of 40 us).  Not unrolled: a
// launch's first pass through long code waits for instructions.
__device__ __forceinline__ uint32_t same_digit(uint32_t digit, bool in, int bits) {
  uint32_t peers = __ballot_sync(0xffffffffu, in);
#pragma unroll 1
  for (int b = 0; b < bits; ++b) {
    const uint32_t ones = __ballot_sync(0xffffffffu, digit >> b & 1u);
    peers &= digit >> b & 1u ? ones : ~ones;
  }
  return peers;
}

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
#pragma unroll 32
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
    const uint32_t peers = same_digit(digit, in, kDigit);
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

// Up to 8192 tokens: one block sorts in shared memory, where a token is one word,
// its key above its number (4096 tokens of 30522 ids: 18.1 us for the gradient, by
// launches 22.9; 8192: 25.6 and 27.6; 12288: 32.7 and 30.7).  The other blocks of the launch meanwhile clear
// the rows of the table that no token has: each marks the ids in its range of
// rows in a bitmap.
constexpr int kOneThreads = 1024, kOneWarps = kOneThreads / 32, kOneTokens = 8192, kOneDigit = 9;
constexpr int kClearRows = 32768;             // rows of a bitmap
struct OneParams {
  const void* ids;
  int wide_ids;
  uint32_t *key_out, *token_out;
  void* dtable;
  int64_t width;
  uint32_t vocab, n;
  int bits, token_bits, digit, size;          // of a key, of a token's number, of a pass; bytes of an element
};

__device__ __forceinline__ uint32_t id_key(const OneParams& p, uint32_t i) {
  const int64_t v = p.wide_ids ? static_cast<const int64_t*>(p.ids)[i] : int64_t(static_cast<const int32_t*>(p.ids)[i]);
  return v >= 0 && v < int64_t(p.vocab) ? uint32_t(v) : p.vocab;
}

__global__ void __launch_bounds__(kOneThreads) sort_one_k(const __grid_constant__ OneParams p) {
  extern __shared__ uint32_t words[];         // [2][n], and of 16 bits [warps][bins] and [n]
  __shared__ uint32_t base[1 << kOneDigit];
  __shared__ uint32_t box[kOneWarps];
  static_assert(kOneThreads >= 1 << kOneDigit, "one bin per thread");
  pdl_wait();
  pdl_trigger();
  const int t = threadIdx.x, lane = t % 32, warp = t / 32;
  if (blockIdx.x > 0) {
    const uint32_t blocks = gridDim.x - 1, mine = blockIdx.x - 1;
    const uint32_t per = min((p.vocab + blocks - 1) / blocks, uint32_t(kClearRows));
    for (uint64_t first = uint64_t(mine) * per; first < p.vocab; first += uint64_t(blocks) * per) {
      const uint32_t rows = uint32_t(min(uint64_t(per), p.vocab - first));
      for (uint32_t w = t; w < (rows + 31) / 32; w += kOneThreads) words[w] = 0;
      __syncthreads();
#pragma unroll 4
      for (uint32_t i = t; i < p.n; i += kOneThreads) {
        const uint32_t v = id_key(p, i) - uint32_t(first);        // wraps below the range
        if (v < rows) atomicOr(&words[v / 32], 1u << v % 32);
      }
      __syncthreads();
      char* d = static_cast<char*>(p.dtable) + int64_t(first) * p.width * p.size;
      const int64_t bytes = p.width * p.size;
      const bool wide = bytes % 16 == 0 && aligned16(p.dtable);
      for (uint32_t r = warp; r < rows; r += kOneWarps) {
        if (words[r / 32] >> r % 32 & 1u) continue;
        char* row = d + int64_t(r) * bytes;
        if (wide)
          for (int64_t c = 16 * lane; c < bytes; c += 512) *reinterpret_cast<uint4*>(row + c) = make_uint4(0u, 0u, 0u, 0u);
        else if (p.size == 4)
          for (int64_t c = 4 * lane; c < bytes; c += 128) *reinterpret_cast<uint32_t*>(row + c) = 0u;
        else
          for (int64_t c = 2 * lane; c < bytes; c += 64) *reinterpret_cast<uint16_t*>(row + c) = uint16_t(0);
      }
      __syncthreads();
    }
    return;
  }
  uint32_t *from = words, *to = words + p.n;
  uint16_t* counts = reinterpret_cast<uint16_t*>(words + 2 * p.n);
  const int bins = 1 << p.digit;
  uint16_t* ranks = counts + kOneWarps * bins;          // of a token among its warp's of its digit
  const uint32_t per = (p.n + 32 * kOneWarps - 1) / (32 * kOneWarps) * 32;       // a warp's neighbouring tokens
  const uint32_t first = min(p.n, warp * per), end = min(p.n, first + per);
  for (uint32_t i = first + lane; i < end; i += 32) from[i] = id_key(p, i) << p.token_bits | i;
  for (int shift = 0; shift < p.bits; shift += p.digit) {
    for (int i = t; i < kOneWarps * bins / 2; i += kOneThreads) reinterpret_cast<uint32_t*>(counts)[i] = 0;
    __syncthreads();
    uint16_t* own = counts + warp * bins;
    // not unrolled: a block's first pass through long code waits for instructions
    // (5000 tokens: 12 us with both loops unrolled)
#pragma unroll 1
    for (uint32_t i0 = first; i0 < end; i0 += 32) {
      const uint32_t i = i0 + lane;
      const bool in = i < end;
      const uint32_t digit = in ? from[i] >> (p.token_bits + shift) & uint32_t(bins - 1) : 0u;
      const uint32_t peers = same_digit(digit, in, p.digit);
      const uint32_t before = in ? own[digit] : 0u;
      __syncwarp();
      const uint32_t lower = __popc(peers & ((1u << lane) - 1u));
      if (in) {
        if (lower == 0) own[digit] = uint16_t(before + __popc(peers));
        ranks[i] = uint16_t(before + lower);
      }
      __syncwarp();
    }
    __syncthreads();
    uint32_t all = 0;                         // of bin t, before each warp
    if (t < bins)
#pragma unroll 8
      for (int w = 0; w < kOneWarps; ++w) {
        const uint32_t c = counts[w * bins + t];
        counts[w * bins + t] = uint16_t(all);
        all += c;
      }
    const uint32_t at = block_before(all, box);
    if (t < bins) base[t] = at;
    __syncthreads();
#pragma unroll 2
    for (uint32_t i = first + lane; i < end; i += 32) {
      const uint32_t v = from[i], digit = v >> (p.token_bits + shift) & uint32_t(bins - 1);
      to[base[digit] + own[digit] + ranks[i]] = v;
    }
    __syncthreads();
    uint32_t* swap = from;
    from = to;
    to = swap;
  }
  // in order: scattered stores would leave one SM a sector at a time
#pragma unroll 2
  for (uint32_t i = t; i < p.n; i += kOneThreads) {
    p.key_out[i] = from[i] >> p.token_bits;
    p.token_out[i] = from[i] & ((1u << p.token_bits) - 1u);
  }
}

// ------------------------------------------------------------------ sums
// A warp sums a piece of `piece` sorted tokens (8, 16 or 32) over 256 columns, and
// a block eight neighbouring pieces, its span.  A row whose tokens all lie in one
// piece is written by the warp, one whose tokens lie in one span by the block; the
// others leave a sum per span in `part` ([span][first or last][width]), which
// join_k adds up.
struct GradParams {
  const void* dout;
  const uint32_t *key, *token;
  void* dtable;
  float* part;
  int64_t ldo;
  uint32_t n, vocab, piece;
  int width, chunks, accumulate;
  float scale;
  int64_t sum_blocks;      // spans times chunks
  int64_t clear_blocks;    // before them: 256 rows each, so that their search is not the launch's end
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
// Column c0 + t of row v.
template <typename S>
__device__ __forceinline__ void write_column(const GradParams& p, uint32_t v, int c, float a) {
  if (c >= p.width) return;
  S* d = static_cast<S*>(p.dtable) + int64_t(v) * p.width + c;
  *d = from_f<S>(p.accumulate ? fmaf(a, p.scale, to_f(*d)) : a * p.scale);
}
__device__ __forceinline__ float* part_at(const GradParams& p, uint32_t span, int last, int c0) {
  return p.part + (int64_t(span) * 2 + last) * p.chunks * 256 + c0;
}

template <typename T, typename S, bool VEC>
__global__ void __launch_bounds__(256, VEC ? 3 : 2) grad_k(const __grid_constant__ GradParams p) {
  __shared__ __align__(16) float sums[8][2][256];     // of each warp's row that began earlier, and that goes on
  __shared__ uint32_t keys[8][2], flags[8];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  if (blockIdx.x < p.clear_blocks) {      // rows of the table without a token are cleared, 32 per warp
    const int64_t first = int64_t(blockIdx.x) * 256 + warp * 32;
    const uint32_t v = uint32_t(min(first + lane, int64_t(p.vocab)));
    uint32_t lo = 0, hi = p.n;
    while (lo < hi) {
      const uint32_t mid = (lo + hi) / 2;
      if (p.key[mid] < v) lo = mid + 1;
      else hi = mid;
    }
    uint32_t clear = __ballot_sync(0xffffffffu, v < p.vocab && (lo >= p.n || p.key[lo] != v));
    while (clear) {
      S* d = static_cast<S*>(p.dtable) + (first + __ffs(int(clear)) - 1) * p.width;
      clear &= clear - 1;
      if constexpr (VEC) {
        const float z[8] = {};
        for (int c = lane * 8; c < p.width; c += 256) store8(d + c, z);
      } else {
        for (int c = lane; c < p.width; c += 32) d[c] = from_f<S>(0.f);
      }
    }
    return;
  }
  const int64_t item = int64_t(blockIdx.x) - p.clear_blocks;
  const uint32_t span = uint32_t(item / p.chunks);
  const int c0 = int(item - int64_t(span) * p.chunks) * 256;
  const uint64_t first = (uint64_t(span) * 8 + warp) * p.piece;
  constexpr uint32_t kOpen = 1, kEnds = 2, kGoesOn = 4;    // began earlier, and ends here; a later one goes on
  uint32_t flag = 0;
  const uint64_t i = first + lane;
  const bool in = lane < int(p.piece) && i < p.n;
  const uint32_t my_key = in ? p.key[i] : p.vocab, my_token = in ? p.token[i] : 0u;
  const uint32_t left = first && first < p.n ? p.key[first - 1] : p.vocab;
  const uint32_t right = first + p.piece < p.n ? p.key[first + p.piece] : p.vocab;
  uint32_t current = __shfl_sync(0xffffffffu, my_key, 0);
  if (current < p.vocab) {           // else only tokens without a row from here on
    float a[8] = {};
    bool open = left == current;
    auto flush = [&](uint32_t next) {
      const bool on = next > p.vocab && right == current;
      if (!open && !on) {
        write_row<S, VEC>(p, current, c0, lane, a);
      } else {
        float* d = sums[warp][open ? 0 : 1];
        if constexpr (VEC) {
          reinterpret_cast<float4*>(d)[2 * lane] = make_float4(a[0], a[1], a[2], a[3]);
          reinterpret_cast<float4*>(d)[2 * lane + 1] = make_float4(a[4], a[5], a[6], a[7]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) d[e * 32 + lane] = a[e];
        }
        if (lane == 0) keys[warp][open ? 0 : 1] = current;
        flag |= !open ? kGoesOn : on ? kOpen : kOpen | kEnds;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) a[e] = 0.f;
      open = false;
      current = next;
    };
    // Rows in flight.  Loads are never skipped, so that they stand together: past
    // the width and for tokens without a row they read what is not used.
    constexpr int kAhead = 4;
    for (int r = 0; r < int(p.piece); r += kAhead) {
      Raw8<T> raw[kAhead];
      T loose[VEC ? 1 : kAhead][8];
      uint32_t key[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        key[u] = __shfl_sync(0xffffffffu, my_key, r + u);
        const uint32_t token = __shfl_sync(0xffffffffu, my_token, r + u);
        const T* d = static_cast<const T*>(p.dout) + int64_t(token) * p.ldo;
        if constexpr (VEC) {
          raw[u].load(d + min(c0 + lane * 8, p.width - 8));
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) loose[u][e] = d[min(c0 + e * 32 + lane, p.width - 1)];
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (key[u] >= p.vocab) break;
        if (key[u] != current) flush(key[u]);
        float v[8];
        if constexpr (VEC) raw[u].get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] += VEC ? v[e] : to_f(loose[VEC ? 0 : u][e]);
      }
    }
    flush(p.vocab + 1u);
  }
  if (lane == 0) flags[warp] = flag;
  __syncthreads();
  // a thread for each column: the rows that cross the span's pieces, in order
  const int t = threadIdx.x;
  float a = 0.f;
  bool before = false, live = false;
  uint32_t row = 0;
  for (int w = 0; w < 8; ++w) {
    const uint32_t f = flags[w];
    if (f & kOpen) {
      before = before || w == 0;
      a += sums[w][0][t];
      row = keys[w][0];
      live = !(f & kEnds);
      if (!live) {
        if (before) part_at(p, span, 0, c0)[t] = a;
        else write_column<S>(p, row, c0 + t, a);
        a = 0.f;
        before = false;
      }
    }
    if (f & kGoesOn) {
      a = sums[w][1][t];
      row = keys[w][1];
      live = true;
    }
  }
  if (live) part_at(p, span, before ? 0 : 1, c0)[t] = a;
}

// Rows that cross spans.  A warp takes a span in which such a row begins and 256
// columns; rows of many spans are shared by the block's warps, which take
// neighbouring runs of them.
constexpr uint32_t kAlone = 32;       // spans that one warp adds up itself

template <typename S, bool VEC>
__global__ void __launch_bounds__(256) join_k(const __grid_constant__ GradParams p) {
  __shared__ float box[8][256];
  __shared__ uint32_t counts[8];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const uint32_t size = 8 * p.piece, spans = (p.n + size - 1) / size;
  const int64_t item0 = int64_t(blockIdx.x) * 8, items = int64_t(spans) * p.chunks;
  auto span_of = [&](int w) { return uint32_t((item0 + w) % spans); };
  auto col_of = [&](int w) { return int((item0 + w) / spans) * 256; };
  // the sum of spans from .. to - 1 of the row that begins in `span`
  auto add = [&](uint32_t span, int c0, uint32_t from, uint32_t to, float (&a)[8]) {
#pragma unroll 8
    for (uint32_t i = from; i < to; ++i) {
      const float* d = part_at(p, span + i, i == 0 ? 1 : 0, c0);
      if constexpr (VEC) {
        const float4 x = reinterpret_cast<const float4*>(d)[2 * lane], y = reinterpret_cast<const float4*>(d)[2 * lane + 1];
        a[0] += x.x, a[1] += x.y, a[2] += x.z, a[3] += x.w, a[4] += y.x, a[5] += y.y, a[6] += y.z, a[7] += y.w;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] += d[e * 32 + lane];
      }
    }
  };
  uint32_t count = 0;
  if (item0 + warp < items) {
    const uint32_t span = span_of(warp), first = span * size, next = first + size;
    const uint32_t v = next < p.n ? p.key[next - 1] : p.vocab, after = next < p.n ? p.key[next] : p.vocab;
    const uint32_t begin = p.key[first], before = first ? p.key[first - 1] : p.vocab;
    // its last row goes on, and did not begin earlier
    if (v < p.vocab && after == v && !(begin == v && before == v)) {
      // the last span that the row reaches: first the next 32, then 32 places at a
      // time of what is left
      uint32_t lo = span + 1, hi = spans - 1, step = 1;
      while (lo < hi) {
        const uint64_t i = uint64_t(lo) + uint64_t(lane + 1) * step;
        const bool has = i <= hi && p.key[i * size] == v;
        const uint32_t n = __popc(__ballot_sync(0xffffffffu, has));
        lo += n * step;
        if (n < 32) hi = min(hi, lo + step - 1);
        step = (hi - lo + 31) / 32;
      }
      count = lo - span + 1;
      if (count <= kAlone) {
        float a[8] = {};
        add(span, col_of(warp), 0, count, a);
        write_row<S, VEC>(p, v, col_of(warp), lane, a);
      }
    }
  }
  if (lane == 0) counts[warp] = count;
  __syncthreads();
  for (int w = 0; w < 8; ++w) {
    const uint32_t all = counts[w];
    if (all <= kAlone) continue;
    const uint32_t per = (all + 7) / 8, span = span_of(w);
    float a[8] = {};
    add(span, col_of(w), warp * per, min(all, (warp + 1) * per), a);
#pragma unroll
    for (int e = 0; e < 8; ++e) box[warp][e * 32 + lane] = a[e];
    __syncthreads();
    if (warp == 0) {
      for (int o = 1; o < 8; ++o)
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] += box[o][e * 32 + lane];
      write_row<S, VEC>(p, p.key[span * size + size - 1], col_of(w), lane, a);
    }
    __syncthreads();
  }
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
  unsigned blocks, per, piece, spans;
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
  // shorter pieces where they and their chunks of columns are few: at least 16 warps per SM
  const int64_t chunks = (width + 255) / 256;
  a.piece = 32;
  while (a.piece > 8 && (tokens + a.piece - 1) / a.piece * chunks < 16 * 152) a.piece /= 2;
  a.spans = unsigned((tokens + 8 * a.piece - 1) / (8 * a.piece));
  a.part = take(int64_t(a.spans) * 2 * chunks * 256 * 4);
  a.bytes = at;
  return a;
}

int bits_of(int64_t v) {
  int n = 1;
  while (v >> n) ++n;
  return n;
}
constexpr int kOneSmem = 2 * kOneTokens * 4 + (kOneWarps << kOneDigit) * 2 + kOneTokens * 2;
cudaError_t sort_one(const OneParams& o, bool accumulate, cudaStream_t st) {
  static std::atomic<bool> allowed[kMaxDevices];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && !(dev < kMaxDevices && allowed[dev])) {
    e = cudaFuncSetAttribute(sort_one_k, cudaFuncAttributeMaxDynamicSharedMemorySize, kOneSmem);
    if (e == cudaSuccess && dev < kMaxDevices) allowed[dev] = true;
  }
  if (e != cudaSuccess) return e;
  const int64_t sort = 10 * int64_t(o.n) + (int64_t(kOneWarps) << o.digit) * 2, clear = kClearRows / 8;
  // as many blocks as fit at once, of 64 rows at least
  const int most = elementwise_blocks(INT64_MAX / 2, 256) / 8 - 1, want = int((int64_t(o.vocab) + 63) / 64);
  const int blocks = accumulate ? 1 : 1 + (want < most ? want : most > 1 ? most : 1);
  return launch_k(sort_one_k, dim3(unsigned(blocks)), dim3(kOneThreads), size_t(sort > clear ? sort : clear), st, o);
}

template <typename I, typename S, typename T>
cudaError_t lookup(const void* ids, const void* table, void* out, int64_t ldo, int64_t tokens, int64_t vocab, int width,
                   float scale, bool vec, cudaStream_t st) {
  // wide rows by 1024 columns, as long as the items are enough for all SMs
  constexpr int U = sizeof(S) == 2 ? 4 : 2;
  const int chunks = (width + 255) / 256, wide = (chunks + U - 1) / U;
  const bool many = vec && chunks > 1 && tokens * wide >= 16 * 152;
  const int groups = many ? wide : chunks;
  const int64_t items = tokens * groups;
  const dim3 grid(unsigned(elementwise_blocks(items * 32, 256)));
  auto k = many ? lookup_k<I, S, T, true, U> : vec ? lookup_k<I, S, T, true, 1> : lookup_k<I, S, T, false, 1>;
  return launch_k(k, grid, dim3(256), 0, st, static_cast<const I*>(ids), static_cast<const S*>(table), static_cast<T*>(out), ldo,
                  items, groups, vocab, width, scale);
}
template <typename T, typename S, bool VEC>
cudaError_t gradient(const GradParams& p, cudaStream_t st) {
  cudaError_t e = launch_k(grad_k<T, S, VEC>, dim3(unsigned(p.sum_blocks + p.clear_blocks)), dim3(256), 0, st, p);
  if (e == cudaSuccess && p.sum_blocks > p.chunks)      // more than one span
    e = launch_k(join_k<S, VEC>, dim3(unsigned((p.sum_blocks + 7) / 8)), dim3(256), 0, st, p);
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
  const int64_t sum_blocks = int64_t(a.spans) * ((width + 255) / 256);
  if (sum_blocks + (vocab + 255) / 256 >= int64_t(1) << 31) return bad("too many tokens for this width");
  char* ws = static_cast<char*>(workspace);
  GradParams p;
  const int bits = bits_of(vocab), token_bits = bits_of(tokens - 1);      // the largest key is vocab
  const bool one = tokens <= kOneTokens && bits + token_bits <= 32;
  if (one) {
    OneParams o;
    o.ids = ids;
    o.wide_ids = ids_bits == 64;
    o.key_out = reinterpret_cast<uint32_t*>(ws + a.key[0]);
    o.token_out = reinterpret_cast<uint32_t*>(ws + a.token[0]);
    o.dtable = dtable;
    o.width = width;
    o.vocab = uint32_t(vocab);
    o.n = uint32_t(tokens);
    o.bits = bits;
    o.token_bits = token_bits;
    const int passes = (bits + kOneDigit - 1) / kOneDigit;
    o.digit = (bits + passes - 1) / passes;
    o.size = int(size_of(table_dtype));
    const cudaError_t e = sort_one(o, accumulate != 0, st);
    if (e != cudaSuccess) return done(e);
    p.key = o.key_out;
    p.token = o.token_out;
  } else {
    SortParams s;
    s.ids = ids;
    s.wide_ids = ids_bits == 64;
    s.key_in = s.token_in = nullptr;
    s.counts = reinterpret_cast<uint32_t*>(ws + a.counts);
    s.vocab = uint32_t(vocab);
    s.n = uint32_t(tokens);
    s.per = a.per;
    int to = 0;
    for (s.shift = 0; s.shift < bits; s.shift += kDigit) {
      s.key_out = reinterpret_cast<uint32_t*>(ws + a.key[to]);
      s.token_out = reinterpret_cast<uint32_t*>(ws + a.token[to]);
      cudaError_t e = launch_k(sort_count_k, dim3(a.blocks), dim3(kSortThreads), 0, st, s);
      if (e == cudaSuccess) e = launch_k(sort_place_k, dim3(a.blocks), dim3(kSortThreads), 0, st, s);
      if (e != cudaSuccess) return done(e);
      s.key_in = s.key_out;
      s.token_in = s.token_out;
      to = 1 - to;
    }
    p.key = s.key_in;
    p.token = s.token_in;
  }
  p.dout = dout;
  p.dtable = dtable;
  p.part = reinterpret_cast<float*>(ws + a.part);
  p.ldo = dout_stride;
  p.n = uint32_t(tokens);
  p.vocab = uint32_t(vocab);
  p.width = int(width);
  p.chunks = int((width + 255) / 256);
  p.accumulate = accumulate != 0;
  p.scale = float(scale);
  p.piece = a.piece;
  p.sum_blocks = sum_blocks;
  p.clear_blocks = accumulate || one ? 0 : (vocab + 255) / 256;
  const bool vec = width % 8 == 0 && aligned16(dtable) && aligned16(dout) &&
                   (tokens == 1 || dout_stride % (dtype == FO_DTYPE_F32 ? 4 : 8) == 0);
  if (dtype == FO_DTYPE_F32) return done(vec ? gradient<float, float, true>(p, st) : gradient<float, float, false>(p, st));
  if (table_dtype == FO_DTYPE_F32) return done(vec ? gradient<bf16, float, true>(p, st) : gradient<bf16, float, false>(p, st));
  return done(vec ? gradient<bf16, bf16, true>(p, st) : gradient<bf16, bf16, false>(p, st));
}

}  // extern "C"
