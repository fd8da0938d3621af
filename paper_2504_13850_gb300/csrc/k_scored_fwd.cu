// Scored attention forward on the tensor cores (fo_scored.h): bf16, head width
// a multiple of 8 up to 128.
//
// A CTA owns NT tiles of 128 queries of one (sequence, head) and walks the
// allowed blocks of 128 keys once, with the running maximum and sum of an
// online softmax.  Warp roles: 8 NT softmax warps, one TMA warp, one MMA warp,
// and one that clears padded tokens out of V where there are any.
// Per tile and block:
//   S = Q K^T into 128 TMEM columns -> cap, bias and mask in registers ->
//   P~ = 2^(c x - M) as bf16 back into the columns it came from, the A
//   operand of O += P~ V (P never touches shared memory).
// The two tiles take turns: one's softmax runs while the other's products do,
// and each K and V block is read once for 256 queries.  K and V share one ring
// of TMA-filled stages.  A query row is shared by two threads, 64 keys each,
// which exchange their maxima through shared memory once per block: sixteen
// warps hide the TMEM and barrier latencies that eight (one thread per row)
// left exposed, at half of the registers.
// O is rescaled in TMEM only when a row's maximum has grown by more than 2^8,
// so a step normally touches O not at all; P~ is then at most 2^8, which fp32
// sums and bf16's exponent hold without loss.
// Scores stay in raw units x with exponent factor c (scale * log2(e), or
// log2(e) after a cap), so an uncapped, unbiased score costs half a packed FMA
// and one exponential.  The cap's tanh (shape_scores) is off by 2e-7 of one at
// most, against the 2^-11 relative error of the hardware's tanh.
// The bias kind and the cap are template parameters: the branches cost
// instruction fetches even when not taken.
// Rounding: P~ to bf16 before its product, O once when stored.
#include "fo_scored_tc.cuh"

namespace fo {

namespace {

__device__ GaveUp g_err;

struct FwdParams {
  ScoredParams s;
  CUtensorMap q, k, v;
};

template <int DP, int NT>
struct Fwd {
  static constexpr int kSub = 16384;                       // 128 rows x 64 bf16
  static constexpr int kTileBytes = DP / 64 * kSub;
  static constexpr int kStages = NT == 2 ? (DP == 64 ? 6 : 4) : (DP == 64 ? 4 : 2);
  static constexpr int kThreads = 256 * NT + (NT == 2 ? 96 : 64);
  static constexpr int kCols = NT == 2 ? 512 : 256;         // TMEM columns
  static constexpr int kBars = 2 + 3 * kStages + 3 * NT;
  static constexpr int kOps = (NT + kStages) * kTileBytes;
  static constexpr int kXch = 2 * NT * 256;                 // floats: [step parity][tile][half][row]
  // operands, barriers (and the TMEM slot), exchanged maxima, bias, bitmaps
  static size_t smem(int L, bool table) {
    const int words = (L + 4095) / 4096;
    return 1024 + kOps + 8 * (kBars + 1) + 4 * kXch + (table ? 4 * kBiasFloats : 0) + size_t(4) * words * (2 * NT + 1);
  }
};

// Minus infinity where key j0 + e is not allowed: from `lim` on by position,
// or of another document than `id`.
__device__ __forceinline__ void mask_keys(uint32_t (&r)[32], int j0, int lim, const int32_t* doc, int id) {
  const int n = lim - j0;
#pragma unroll
  for (int e = 0; e < 32; ++e)
    if (e >= n) r[e] = 0xff800000u;
  if (doc) {
    const int4* d = reinterpret_cast<const int4*>(doc + j0);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int4 v = __ldg(d + e);
      if (v.x != id) r[4 * e] = 0xff800000u;
      if (v.y != id) r[4 * e + 1] = 0xff800000u;
      if (v.z != id) r[4 * e + 2] = 0xff800000u;
      if (v.w != id) r[4 * e + 3] = 0xff800000u;
    }
  }
}

__device__ __forceinline__ float max_of(const uint32_t (&r)[32]) {
  float m[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    m[k] = __uint_as_float(r[8 * k]);
#pragma unroll
    for (int e = 1; e < 7; e += 2)
      m[k] = max3(m[k], __uint_as_float(r[8 * k + e]), __uint_as_float(r[8 * k + e + 1]));
    m[k] = fmaxf(m[k], __uint_as_float(r[8 * k + 7]));
  }
  return fmaxf(max3(m[0], m[1], m[2]), m[3]);
}

template <int DP, int NT, int BIAS, int CAP>
__global__ void __launch_bounds__(Fwd<DP, NT>::kThreads, 3 - NT) scored_fwd_tc_k(const __grid_constant__ FwdParams fp) {
  using F = Fwd<DP, NT>;
  const ScoredParams& p = fp.s;
  extern __shared__ __align__(1024) char smem_raw[];
  char* sm = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);    // 1024-byte aligned
  char* sQ = sm;
  char* ring = sm + NT * F::kTileBytes;
  uint64_t* bars = reinterpret_cast<uint64_t*>(sm + F::kOps);
  uint64_t *qfull = bars, *full = bars + 1, *empty = full + F::kStages, *clean = empty + F::kStages,
           *sfull = clean + F::kStages, *pfull = sfull + NT, *ofull = pfull + NT, *done = ofull + NT;
  uint32_t* tslot = reinterpret_cast<uint32_t*>(bars + F::kBars);
  float* xch = reinterpret_cast<float*>(bars + F::kBars + 1);
  float* bias = xch + F::kXch;
  const int words = (p.L + 4095) / 4096;
  uint32_t* act = reinterpret_cast<uint32_t*>(bias + (BIAS == kBiasTable ? kBiasFloats : 0));   // [NT][words]: blocks of the tile
  uint32_t* some = act + NT * words;                                        // [NT][words]: blocks that need the mask
  uint32_t* padded = some + NT * words;                                     // [words]: blocks that hold padding

  const int warp = __shfl_sync(0xffffffffu, int(threadIdx.x) / 32, 0), lane = threadIdx.x % 32;
  const int tiles = (p.L + 128 * NT - 1) / (128 * NT), bh = blockIdx.x % (p.B * p.H);
  const int q0 = (tiles - 1 - int(blockIdx.x / (p.B * p.H))) * 128 * NT;   // the longest causal rows first
  const int b = bh / p.H, h = bh % p.H, kh = h / p.G;
  // one tile walks at most one block, which the TMA warp can clear itself
  constexpr int kTma = 8 * NT, kMma = 8 * NT + 1, kClean = NT == 2 ? kMma + 1 : kTma;
  if (warp == kMma) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tslot)),
                 "r"(F::kCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (warp == kTma && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&fp.q)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&fp.k)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&fp.v)) : "memory");
    mbar_init(qfull, 1);
    for (int e = 0; e < F::kStages; ++e) {
      mbar_init(&full[e], 1);
      mbar_init(&empty[e], 1);
      mbar_init(&clean[e], 1);
    }
    for (int e = 0; e < NT; ++e) {
      mbar_init(&sfull[e], 1);
      mbar_init(&pfull[e], 8);         // one arrival per warp
      mbar_init(&ofull[e], 1);
    }
    mbar_init(done, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  pdl_wait();
  if (warp == kTma && lane == 0) {       // the queries, while the rest is prepared
    mbar_expect_tx(qfull, NT * F::kTileBytes);
    for (int t = 0; t < NT; ++t)
      for (int s = 0; s < DP / 64; ++s)
        tma_4d(sQ + t * F::kTileBytes + s * F::kSub, &fp.q, qfull, 64 * s, q0 + 128 * t, h, b);
  }
  // score units: raw products without a cap, natural ones after it
  const float unit = CAP ? 1.f : p.scale, c = unit * kLog2e;
  const int pf = p.prefix ? p.prefix[b] : 0;
  if (BIAS == kBiasTable) load_bias(bias, p, h, 1.f / unit, threadIdx.x, F::kThreads);
  for (int w = warp; w < words; w += F::kThreads / 32) {
    const int k0 = (32 * w + lane) * 128;
    const int2* blk = p.blk ? p.blk + int64_t(b) * (p.Lp / kScoredBlock) : nullptr;
    int2 kd = make_int2(0, 0);
    if (blk && k0 < p.L) kd = doc_join(blk[k0 / 64], blk[k0 / 64 + 1]);
    bool any = false;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int i0 = q0 + 128 * t;
      int cls = kScoredNone;
      if (k0 < p.L && i0 < p.L) {
        int2 qd = make_int2(0, 0);
        if (blk) qd = doc_join(blk[i0 / 64], blk[i0 / 64 + 1]);
        cls = scored_class(p, pf, i0, i0 + 128, k0, k0 + 128, blk != nullptr, qd, kd);
        if (cls == kScoredAll && k0 + 128 > p.L) cls = kScoredSome;
      }
      const uint32_t on = __ballot_sync(0xffffffffu, cls != kScoredNone);
      const uint32_t mask = __ballot_sync(0xffffffffu, cls == kScoredSome);
      any = any || cls != kScoredNone;
      if (lane == 0) {
        act[t * words + w] = on;
        some[t * words + w] = mask;
      }
    }
    const uint32_t pad = __ballot_sync(0xffffffffu, any && kd.x < 0);
    if (lane == 0) padded[w] = pad;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tslot;     // S / P of tile t: columns 128 t; O: 128 NT + DP t
  pdl_trigger();                    // this block holds its tensor memory
  Waits wait(&g_err);
  const uint32_t* act1 = act + (NT - 1) * words;

  if (warp == kTma) {
    if (lane == 0) {
      Bits list(act, act1, words);
      Ring<F::kStages> at;
      int it = 0;
      for (int jb = list.next(); jb >= 0 && !wait.dead; jb = list.next())
        for (int kv = 0; kv < 2; ++kv, ++it) {
          if (it >= F::kStages) wait.on(&empty[at.at], at.phase ^ 1, 21);
          if (wait.dead) break;
          mbar_expect_tx(&full[at.at], F::kTileBytes);
          for (int s = 0; s < DP / 64; ++s)
            tma_4d(ring + at.at * F::kTileBytes + s * F::kSub, kv ? &fp.v : &fp.k, &full[at.at], 64 * s, jb * 128, kh, b);
          at.step();
        }
      // every copy has landed before the block ends, whichever role gave up
      mbar_wait(qfull, 0);
      for (int e = max(0, it - F::kStages); e < it; ++e) mbar_wait(&full[e % F::kStages], (e / F::kStages) & 1);
    }
  } else if (warp == kMma) {
    constexpr uint32_t id_s = instr_desc(128, false, false), id_o = instr_desc(DP, false, true);
    const uint32_t ring_at = smem_u32(ring);
    auto issue_s = [&](int t, int slot) {
      const Operand<16> q(smem_u32(sQ) + t * F::kTileBytes), k(ring_at + slot * F::kTileBytes);
#pragma unroll
      for (int e = 0; e < DP / 16; ++e) {
        const uint32_t off = (e >> 2) * F::kSub + 32 * (e & 3);
        mma_ss(tmem + 128 * t, q.at(off), k.at(off), id_s, e > 0 ? 1u : 0u);
      }
      commit_to(&sfull[t]);
    };
    Bits list(act, act1, words);
    uint64_t* landed = any_bit(padded, words) ? clean : full;      // V has landed, without padding
    int cur = list.next();
    bool on[2] = {list.on[0], list.on[1]};
    uint32_t step[2] = {0, 0};
    Ring<F::kStages, 2> k_at(0), v_at(1);
    wait.on_lanes(qfull, 0, 22);
    if (cur >= 0) {
      wait.on_lanes(&full[0], 0, 23);
      tc_fence_after();
      if (on[0]) issue_s(0, 0);
      if (NT == 2 && on[1]) issue_s(1, 0);
      commit_to(&empty[0]);
      k_at.step();
    }
    while (cur >= 0) {
      const int nxt = list.next();
      wait.on_lanes(&landed[v_at.at], v_at.phase, 24);
      if (nxt >= 0) wait.on_lanes(&full[k_at.at], k_at.phase, 25);
      const Operand<F::kSub> v(ring_at + v_at.at * F::kTileBytes);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const bool then = nxt >= 0 && list.on[t];
        if (on[t]) {
          wait.on_lanes(&pfull[t], step[t] & 1, 26);
          tc_fence_after();
        }
        if (on[t]) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            mma_ts(tmem + 128 * NT + DP * t, tmem + 128 * t + 64 * (e >> 2) + 8 * (e & 3), v.at(2048 * e), id_o,
                   e > 0 ? 1u : step[t]);
          commit_to(&ofull[t]);
        }
        if (then) issue_s(t, k_at.at);
        if (t == NT - 1) {
          commit_to(&empty[v_at.at]);
          if (nxt >= 0) commit_to(&empty[k_at.at]);
        }
        if (on[t]) ++step[t];
      }
      v_at.step();
      k_at.step();
      on[0] = list.on[0];
      on[1] = list.on[1];
      cur = nxt;
      // off the waits' path; what was issued after one gave up is void anyway
      if (__any_sync(0xffffffffu, wait.dead)) break;
    }
    // no product is in flight when the block ends and its memory is another's
    commit_to(done);
    mbar_wait(done, 0);
    __syncwarp();
  } else if (warp < kTma) {
    const int t = warp / 8, half = warp / 4 % 2, quarter = warp % 4, row = 32 * quarter + lane;
    const int i0 = q0 + 128 * t + 32 * quarter, i = i0 + lane;
    const uint32_t lanes = uint32_t(32 * quarter) << 16;
    const uint32_t s_col = tmem + lanes + 128 * t + 64 * half, o_col = tmem + lanes + 128 * NT + DP * t + DP / 2 * half;
    const uint32_t masked = smem_u32(some + t * words);
    const Shape a = shape_of(p, h, unit, bias);
    const int lim = min(p.causal ? max(i + 1, pf) : p.L, p.L);
    const int32_t* doc = p.doc ? p.doc + int64_t(b) * p.Lp : nullptr;
    int id = doc && i < p.L ? doc[i] : 0;
    if (id < 0) id = INT32_MIN;               // padding equals nothing, itself included
    float* my_max = xch + 256 * t + 128 * half + row;          // + 256 NT on odd steps
    const float* other_max = xch + 256 * t + 128 * (1 - half) + row;
    const int pair = 1 + 4 * t + quarter;     // the named barrier of the two warps of these rows
    float m = -INFINITY;
    F2 sum2 = f2(0.f, 0.f);
    int step = 0;
    BitList list(act + t * words, words);
    for (int jb = list.next(); jb >= 0; jb = list.next(), ++step) {
      const int j0 = jb * 128 + 64 * half, flip = (step & 1) * 256 * NT;
      wait.on_lanes(&sfull[t], step & 1, 27);
      tc_fence_after();
      uint32_t r0[32], r1[32];
      tmem_ld32_issue(s_col, r0);
      tmem_ld32_issue(s_col + 32, r1);
      tmem_ld32_wait(r0);
      tmem_ld32_wait(r1);
      shape_scores<32, BIAS, CAP, 1, false>(r0, nullptr, a, j0 - i, j0 - i0 - 31, j0 - i0 + 31);
      shape_scores<32, BIAS, CAP, 1, false>(r1, nullptr, a, j0 + 32 - i, j0 - i0 + 1, j0 - i0 + 63);
      if ((BitList::word(masked, jb >> 5) >> (jb & 31)) & 1u) {
        mask_keys(r0, j0, lim, doc, id);
        mask_keys(r1, j0 + 32, lim, doc, id);
      }
      const float top = fmaxf(max_of(r0), max_of(r1));
      my_max[flip] = top;
      asm volatile("bar.sync %0, 64;" ::"r"(pair) : "memory");
      const float now = max3(m, top, other_max[flip]);
      if (step == 0) {
        m = now;
      } else {
        const bool need = (now - m) * c > 8.f;
        if (__any_sync(0xffffffffu, need)) {
          const float keep = need ? ex2((m - now) * c) : 1.f;
          wait.on_lanes(&ofull[t], (step - 1) & 1, 28);
          tc_fence_after();
#pragma unroll 1
          for (int g = 0; g < DP / 32; ++g) {
            uint32_t o[16];
            tmem_ld16_issue(o_col + 16 * g, o);
            tmem_ld16_wait(o);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * keep);
            tmem_st16(o_col + 16 * g, o);
          }
          sum2 = mul2(sum2, f2(keep, keep));
          if (need) m = now;
        }
      }
      const float base = m == -INFINITY ? 0.f : -m * c;
      const F2 c2 = f2(c, c), base2 = f2(base, base);
      F2 part = f2(0.f, 0.f);
      // columns 0..31 -> words 0..15 of r0, then 32..63 -> words 16..31
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float x, y;
        split(fma2(f2u(r0[2 * e], r0[2 * e + 1]), c2, base2), x, y);
        x = ex2(x);
        y = ex2(y);
        sum2 = add2(sum2, f2(x, y));
        r0[e] = bf16_pair(x, y);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float x, y;
        split(fma2(f2u(r1[2 * e], r1[2 * e + 1]), c2, base2), x, y);
        x = ex2(x);
        y = ex2(y);
        part = add2(part, f2(x, y));
        r0[16 + e] = bf16_pair(x, y);
      }
      sum2 = add2(sum2, part);
      tmem_st32(s_col, r0);
      tmem_st_wait();
      tc_fence_before();
      arrive_warp(&pfull[t]);
    }
    // the row's sum over both halves (the last step's maxima have been read:
    // this is the other buffer)
    float sum, other;
    split(sum2, sum, other);
    sum += other;
    my_max[(step & 1) * 256 * NT] = sum;
    asm volatile("bar.sync %0, 64;" ::"r"(pair) : "memory");
    const float theirs = other_max[(step & 1) * 256 * NT];
    sum = half ? theirs + sum : sum + theirs;
    const float inv = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);     // a NaN row stays NaN
    if (step > 0) {
      wait.on_lanes(&ofull[t], (step - 1) & 1, 29);
      tc_fence_after();
    }
    if (half == 0 && i < p.L) p.lse[int64_t(bh) * p.L + i] = sum == 0.f ? -INFINITY : m * c * kLn2 + logf(sum);
    bf16* out = static_cast<bf16*>(p.o.p) + b * p.o.sb + int64_t(i) * p.o.sl + h * p.o.sh;
#pragma unroll 1
    for (int g = 0; g < DP / 64; ++g) {
      const int col = DP / 2 * half + 32 * g;
      uint32_t o[32];
      if (step > 0) {
        tmem_ld32(o_col + 32 * g, o);
      } else {
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = 0u;
      }
      if (i >= p.L) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (col + 8 * e >= p.D) break;
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          w[k] = bf16_pair(__uint_as_float(o[8 * e + 2 * k]) * inv, __uint_as_float(o[8 * e + 2 * k + 1]) * inv);
        reinterpret_cast<uint4*>(out + col)[e] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
  if (warp == kClean && any_bit(padded, words)) {
    __syncwarp();
    Bits list(act, act1, words);
    Ring<F::kStages, 2> v_at(1);
    for (int jb = list.next(); jb >= 0 && !wait.dead; jb = list.next()) {
      wait.on_warp(&full[v_at.at], v_at.phase, 25);
      if (bit_of(padded, jb))
        clear_padding(ring + v_at.at * F::kTileBytes, 128, DP / 64, p.doc + int64_t(b) * p.Lp + jb * 128);
      arrive_warp(&clean[v_at.at]);
      v_at.step();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kMma) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(F::kCols) : "memory");
  }
}

template <int DP, int NT>
struct Launch {
  const FwdParams& fp;
  cudaStream_t st;
  template <int BIAS, int CAP>
  cudaError_t operator()() const {
    using F = Fwd<DP, NT>;
    const size_t smem = F::smem(fp.s.L, BIAS == kBiasTable);
    auto k = scored_fwd_tc_k<DP, NT, BIAS, CAP>;
    static std::atomic<bool> allowed[kMaxDevices];
    const cudaError_t e = allow_smem(k, allowed);
    if (e != cudaSuccess) return e;
    const int64_t tiles = ceil_div(fp.s.L, 128 * NT);
    return launch_k(k, dim3(unsigned(tiles * fp.s.B * fp.s.H)), dim3(F::kThreads), smem, st, fp);
  }
};

}  // namespace

cudaError_t scored_fwd_tc(const ScoredParams& p, cudaStream_t st, bool* ok) {
  FwdParams fp;
  fp.s = p;
  *ok = scored_map(&fp.q, p.q, p, p.H, 128) && scored_map(&fp.k, p.k, p, p.KV, 128) &&
        scored_map(&fp.v, p.v, p, p.KV, 128);
  if (!*ok) return cudaSuccess;
  // Two query tiles per CTA share each K and V block and overlap softmax with
  // products; a sequence of one tile would leave the second one empty.
  if (p.L <= 128)
    return p.D <= 64 ? with_shape(p, Launch<64, 1>{fp, st}) : with_shape(p, Launch<128, 1>{fp, st});
  return p.D <= 64 ? with_shape(p, Launch<64, 2>{fp, st}) : with_shape(p, Launch<128, 2>{fp, st});
}

cudaError_t scored_fwd_error(unsigned* told, int* code) { return gave_up_since(g_err, told, code); }

}  // namespace fo
