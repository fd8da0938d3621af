// Scored attention backward on the tensor cores (fo_scored.h): bf16, head
// width a multiple of 8 up to 128.
//
// One kernel body, launched twice.  A CTA keeps a tile of 128 rows of X and Y
// in shared memory and walks blocks of 64 rows of U and W:
//   KV = false  rows are queries:  X = Q, Y = dO, U = K, W = V
//               S = X U^T, dP = Y W^T,  dQ += dS U, table gradient
//   KV = true   rows are keys:     X = K, Y = V, U = Q, W = dO, over every
//               query head of the group
//               S^T = X U^T, dP^T = Y W^T,  dV += P^T W, dK += dS^T U
// so each gradient is a sum in one CTA, in a fixed order, without atomics; the
// price is that S and dP are formed twice (7 products instead of 5).  An
// alternative that adds dQ in global memory would save two products and lose
// reproducibility.
// S and dP take 64 TMEM columns each, twice: two warpgroups of 128 threads (one
// row each) process alternate blocks, so that one's arithmetic runs while the
// other's products do.  P and dS go back to TMEM as bf16 over the scores they
// came from, as A operands of the accumulating products; no score touches
// shared memory.  Row statistics come from scored_delta_k; for KV = true they
// are per column and ride along in each stage.
// The table gradient sums dS in fp32 by distance: each warp turns 32 x 32
// patches through shared memory so that a lane sums a diagonal, in arrays of
// its own by distance; patches beyond the reach are one sum per thread.  It is
// stored in the table's type: D comes from the rounded O, so further bits would
// carry no information.
// Rounding: P and dS to bf16 before their products, each gradient once.
#include "fo_scored_tc.cuh"

namespace fo {

namespace {

__device__ int g_err;     // set by a wait that gave up

struct BwdParams {
  ScoredParams s;
  CUtensorMap x, y, u, w;
};

constexpr int kThreads = 320;           // two warpgroups, the TMA warp, the MMA warp
constexpr int kTma = 8, kMma = 9;
constexpr int kMaxStages = 4;
constexpr int kPatch = 32 * 33;         // floats of a warp's 32 x 32 patch, rows 33 apart

template <int DP, bool KV>
struct Bwd {
  static constexpr int kX = DP / 64 * 16384;        // 128 rows
  static constexpr int kU = DP / 64 * 8192;         // 64 rows
  static constexpr int kStats = KV ? 512 : 0;       // lse and D of 64 queries
  static constexpr int kStage = 2 * kU + (KV ? 1024 : 0);
  static constexpr int kBars = 1 + 2 * kMaxStages + 2 * 2 + 1;
  static constexpr int kBias = 2 * kMaxReach + 4;
  // X, Y, stages, barriers (and the TMEM slot), bias (one per warpgroup when
  // heads change along the walk), bitmaps, table-gradient arrays
  static size_t smem(int L, int stages, bool table, bool grad, int reach) {
    const int words = (L + 2047) / 2048;
    size_t n = 1024 + 2 * kX + size_t(stages) * kStage + 8 * (kBars + 1) + size_t(4) * words * 3;
    if (table) n += 4 * kBias * (KV ? 2 : 1);
    if (grad) n += 4 * (8 * kPatch + 8 * dist_floats(reach)) + 2 * kMaxReach + 4;
    return n;
  }
  __host__ __device__ static int dist_floats(int reach) { return (2 * reach + 1 + 3) / 4 * 4; }
};

template <int DP, bool KV>
__global__ void __launch_bounds__(kThreads, 1) scored_bwd_tc_k(const __grid_constant__ BwdParams bp) {
  using F = Bwd<DP, KV>;
  const ScoredParams& p = bp.s;
  extern __shared__ __align__(1024) char smem_raw[];
  char* sm = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  char *sX = sm, *sY = sm + F::kX, *ring = sm + 2 * F::kX;
  const int stages = p.stages, words = (p.L + 2047) / 2048;
  uint64_t* bars = reinterpret_cast<uint64_t*>(ring + stages * F::kStage);
  uint64_t *xfull = bars, *full = bars + 1, *empty = full + kMaxStages, *sfull = empty + kMaxStages, *pfull = sfull + 2,
           *afull = pfull + 2;
  uint32_t* tslot = reinterpret_cast<uint32_t*>(bars + F::kBars);
  uint32_t* act = reinterpret_cast<uint32_t*>(bars + F::kBars + 1);
  uint32_t *some = act + words, *padded = some + words;
  float* bias = reinterpret_cast<float*>(padded + words);
  const bool grad = !KV && p.dtable;
  float* patch = bias + (p.table ? F::kBias * (KV ? 2 : 1) : 0);
  float* dist = patch + 8 * kPatch;
  const int nd = F::dist_floats(p.reach);
  uint8_t* map = reinterpret_cast<uint8_t*>(dist + 8 * nd);

  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int heads = KV ? p.KV : p.H, tiles = (p.L + 127) / 128, bh = blockIdx.x % (p.B * heads);
  const int slot0 = int(blockIdx.x / (p.B * heads)), tile = KV ? slot0 : tiles - 1 - slot0;   // longest causal first
  const int r0 = tile * 128, b = bh / heads, h0 = KV ? (bh % heads) * p.G : bh % heads, kh = h0 / p.G;
  const int groups = KV ? p.G : 1;
  if (threadIdx.x == 0) {
    mbar_init(xfull, 1);
    for (int e = 0; e < stages; ++e) {
      mbar_init(&full[e], 1);
      mbar_init(&empty[e], 1);
    }
    for (int e = 0; e < 2; ++e) {
      mbar_init(&sfull[e], 1);
      mbar_init(&pfull[e], 128);
    }
    mbar_init(afull, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMma) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tslot)), "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (warp == kTma && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&bp.x)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&bp.y)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&bp.u)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&bp.w)) : "memory");
  }
  pdl_wait();
  const float unit = p.cap > 0.f ? 1.f : p.scale, c = unit * kLog2e;
  const int pf = p.prefix ? p.prefix[b] : 0;
  const int2* blk = p.blk ? p.blk + int64_t(b) * (p.Lp / kScoredBlock) : nullptr;
  if (p.table && !KV)
    for (int e = threadIdx.x; e < 2 * p.reach + 1; e += kThreads)
      bias[e] = __bfloat162float(static_cast<const bf16*>(p.table)[int64_t(h0) * p.buckets + p.map[e]]) / unit;
  if (grad) {
    for (int e = threadIdx.x; e < 8 * nd; e += kThreads) dist[e] = 0.f;
    for (int e = threadIdx.x; e < 2 * p.reach + 1; e += kThreads) map[e] = p.map[e];
  }
  {
    int2 rd = make_int2(0, 0);
    if (blk) rd = doc_join(blk[r0 / 64], blk[r0 / 64 + 1]);
    for (int w = warp; w < words; w += kThreads / 32) {
      const int c0 = (32 * w + lane) * 64;
      int cls = kScoredNone;
      bool pad = false;
      if (c0 < p.L) {
        int2 cd = make_int2(0, 0);
        if (blk) cd = blk[c0 / 64];
        cls = KV ? scored_class(p, pf, c0, c0 + 64, r0, r0 + 128, blk != nullptr, cd, rd)
                 : scored_class(p, pf, r0, r0 + 128, c0, c0 + 64, blk != nullptr, rd, cd);
        // keys past the end are zeros in shared memory, not absent; queries
        // past the end have lse = +infinity
        if (!KV && cls == kScoredAll && c0 + 64 > p.L) cls = kScoredSome;
        pad = cd.x < 0 && cls != kScoredNone;
      }
      const uint32_t on = __ballot_sync(0xffffffffu, cls != kScoredNone);
      const uint32_t mask = __ballot_sync(0xffffffffu, cls == kScoredSome);
      const uint32_t pads = __ballot_sync(0xffffffffu, pad);
      if (lane == 0) {
        act[w] = on;
        some[w] = mask;
        padded[w] = pads;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // S and dP of stage s: columns 128 s and 128 s + 64; sums at 256 and 256 + DP
  const uint32_t tmem = *tslot;
  pdl_trigger();
  Waits wait(&g_err);

  if (warp == kTma) {
    if (lane == 0) {
      mbar_expect_tx(xfull, 2 * F::kX);
      for (int s = 0; s < DP / 64; ++s) {
        tma_4d(sX + s * 16384, &bp.x, xfull, 64 * s, r0, KV ? kh : h0, b);
        tma_4d(sY + s * 16384, &bp.y, xfull, 64 * s, r0, KV ? kh : h0, b);
      }
      int it = 0;
      for (int g = 0; g < groups && !wait.dead; ++g) {
        Bits list(act, act, words);
        const int64_t stat = (int64_t(b) * p.H + h0 + g) * p.Lp;
        for (int cb = list.next(); cb >= 0; cb = list.next(), ++it) {
          const int slot = it % stages;
          if (it >= stages) wait.on(&empty[slot], (it / stages - 1) & 1, 31);
          if (wait.dead) break;
          char* st = ring + slot * F::kStage;
          mbar_expect_tx(&full[slot], 2 * F::kU + F::kStats);
          for (int s = 0; s < DP / 64; ++s) {
            tma_4d(st + s * 8192, &bp.u, &full[slot], 64 * s, cb * 64, KV ? h0 + g : kh, b);
            tma_4d(st + F::kU + s * 8192, &bp.w, &full[slot], 64 * s, cb * 64, KV ? h0 + g : kh, b);
          }
          if (KV) {
            bulk_g2s(st + 2 * F::kU, p.lse2 + stat + cb * 64, 256, &full[slot]);
            bulk_g2s(st + 2 * F::kU + 256, p.delta + stat + cb * 64, 256, &full[slot]);
          }
        }
      }
      if (wait.dead) {   // let the copies in flight land before the block ends
        mbar_wait(xfull, 0);
        for (int e = max(0, it - stages); e < it; ++e) mbar_wait(&full[e % stages], (e / stages) & 1);
      }
    }
  } else if (warp == kMma) {
    constexpr uint32_t id_s = instr_desc(64, false, false), id_a = instr_desc(DP, false, true);
    int blocks = 0;
    for (int w = 0; w < words; ++w) blocks += __popc(act[w]);
    const int total = blocks * groups;
    const int32_t* doc = p.doc ? p.doc + int64_t(b) * p.Lp : nullptr;
    Bits list(act, act, words);
    // wait for the operands of step n, then S and dP into TMEM stage n % 2
    auto scores = [&](int n) {
      int cb = list.next();
      if (cb < 0) {              // the next head of the group walks the same blocks
        list = Bits(act, act, words);
        cb = list.next();
      }
      const int slot = n % stages;
      char* st = ring + slot * F::kStage;
      wait.on_warp(&full[slot], (n / stages) & 1, 32);
      if (bit_of(padded, cb)) {
        clear_padding(st, 64, DP / 64, doc, cb * 64, p.L);
        if (KV) clear_padding(st + F::kU, 64, DP / 64, doc, cb * 64, p.L);
      }
      tc_fence_after();
      if (lane == 0 && !wait.dead) {
        const uint32_t x = smem_u32(sX), y = smem_u32(sY), u = smem_u32(st), w = u + F::kU, d = tmem + 128 * (n & 1);
#pragma unroll
        for (int e = 0; e < DP / 16; ++e) {
          const uint32_t rx = (e >> 2) * 16384 + 32 * (e & 3), ru = (e >> 2) * 8192 + 32 * (e & 3);
          mma_f16(d, smem_desc(x + rx, 16, 1024), smem_desc(u + ru, 16, 1024), id_s, e > 0 ? 1u : 0u);
        }
#pragma unroll
        for (int e = 0; e < DP / 16; ++e) {
          const uint32_t rx = (e >> 2) * 16384 + 32 * (e & 3), ru = (e >> 2) * 8192 + 32 * (e & 3);
          mma_f16(d + 64, smem_desc(y + rx, 16, 1024), smem_desc(w + ru, 16, 1024), id_s, e > 0 ? 1u : 0u);
        }
        mma_commit(&sfull[n & 1]);
      }
    };
    wait.on_warp(xfull, 0, 33);
    if (total > 0) scores(0);
    if (total > 1) scores(1);
    for (int n = 0; n < total && !wait.dead; ++n) {
      wait.on_warp(&pfull[n & 1], (n >> 1) & 1, 34);
      tc_fence_after();
      if (lane == 0 && !wait.dead) {
        const uint32_t u = smem_u32(ring + (n % stages) * F::kStage), w = u + F::kU, a = tmem + 128 * (n & 1);
        if (KV) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            mma_f16_ta(tmem + 256, a + 8 * e, smem_desc(w + 2048 * e, 8192, 1024), id_a, n > 0 || e > 0 ? 1u : 0u);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
          mma_f16_ta(tmem + 256 + (KV ? DP : 0), a + 64 + 8 * e, smem_desc(u + 2048 * e, 8192, 1024), id_a,
                     n > 0 || e > 0 ? 1u : 0u);
        mma_commit(&empty[n % stages]);
        if (n + 1 == total) mma_commit(afull);
      }
      if (n + 2 < total) scores(n + 2);
    }
  } else {
    const int wg = warp / 4, quarter = warp % 4, i0 = r0 + 32 * quarter, i = i0 + lane;
    const uint32_t lanes = uint32_t(32 * quarter) << 16;
    const uint32_t s_col = tmem + lanes + 128 * wg, d_col = s_col + 64;
    const int32_t* doc = p.doc ? p.doc + int64_t(b) * p.Lp : nullptr;
    int id = doc && i < p.L ? doc[i] : 0;
    if (id < 0) id = INT32_MIN;            // padding equals nothing, itself included
    const float cap = p.cap, cap_in = cap > 0.f ? 2.f * kLog2e * p.scale / cap : 0.f;
    const int reach = p.reach;
    float row_lse = 0.f, row_d = 0.f;
    if (!KV) {
      const int64_t at = (int64_t(b) * p.H + h0) * p.Lp + i;
      row_lse = p.lse2[at];
      row_d = p.delta[at];
    }
    float lo_sum = 0.f, hi_sum = 0.f;      // table gradient beyond the reach
    float* my_patch = patch + warp * kPatch;
    float* my_dist = dist + warp * nd;
    float* my_bias = bias + (KV ? wg * F::kBias : 0);
    int n = 0;
    for (int g = 0; g < groups; ++g) {
      const float slope = p.slopes ? -p.slopes[h0 + g] / unit : 0.f;
      if (KV && p.table) {
        asm volatile("bar.sync %0, 128;" ::"r"(1 + wg) : "memory");
        for (int e = threadIdx.x % 128; e < 2 * reach + 1; e += 128)
          my_bias[e] = __bfloat162float(static_cast<const bf16*>(p.table)[int64_t(h0 + g) * p.buckets + p.map[e]]) / unit;
        asm volatile("bar.sync %0, 128;" ::"r"(1 + wg) : "memory");
      }
      Bits list(act, act, words);
      for (int cb = list.next(); cb >= 0; cb = list.next(), ++n) {
        if ((n & 1) != wg) continue;
        const bool mask = bit_of(some, cb);
        const int slot = n % stages;
        if (KV) wait.on_warp(&full[slot], (n / stages) & 1, 35);   // its statistics
        wait.on_warp(&sfull[wg], (n >> 1) & 1, 36);
        tc_fence_after();
        const uint32_t stats = smem_u32(ring + slot * F::kStage + 2 * F::kU);
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
          const int c0 = cb * 64 + 32 * half;
          uint32_t s[32], t[32];
          tmem_ld32_issue(s_col + 32 * half, s);
          tmem_ld32_issue(d_col + 32 * half, t);
          tmem_ld32_wait(s);
          tmem_ld32_wait(t);
          // scores: cap (its derivative goes to `chain` below), then bias.
          // For rows i and columns c0 + e the distance j - i is
          // c0 + e - i (rows are queries) or i - c0 - e (rows are keys).
          uint32_t pr[32];
          if (cap > 0.f) {
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const float q = rcp(1.f + ex2(__uint_as_float(s[e]) * cap_in));
              s[e] = __float_as_uint(q);
              pr[e] = __float_as_uint(fmaf(-2.f * cap, q, cap));
            }
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) pr[e] = s[e];
          }
          if (p.table) {
            const int lo = KV ? i0 - c0 - 31 : c0 - i0 - 31, hi = lo + 62, d = KV ? i - c0 : c0 - i;
            if (lo >= reach || hi <= -reach) {
              const float z = my_bias[lo >= reach ? 2 * reach : 0];
#pragma unroll
              for (int e = 0; e < 32; ++e) pr[e] = __float_as_uint(__uint_as_float(pr[e]) + z);
            } else if (lo >= -reach && hi <= reach) {
              const float* z = my_bias + d + reach;
#pragma unroll
              for (int e = 0; e < 32; ++e) pr[e] = __float_as_uint(__uint_as_float(pr[e]) + z[KV ? -e : e]);
            } else {
#pragma unroll
              for (int e = 0; e < 32; ++e)
                pr[e] = __float_as_uint(__uint_as_float(pr[e]) +
                                        my_bias[min(max(KV ? d - e : d + e, -reach), reach) + reach]);
            }
          } else if (slope != 0.f) {
            const float d = float(c0 - i);
#pragma unroll
            for (int e = 0; e < 32; ++e)
              pr[e] = __float_as_uint(fmaf(slope, fabsf(d + float(e)), __uint_as_float(pr[e])));
          }
          // P = 2^(c x - lse), dS = P (dP - D)
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            float4 l4 = make_float4(row_lse, row_lse, row_lse, row_lse), d4 = make_float4(row_d, row_d, row_d, row_d);
            if (KV) {
              l4 = ld_shared4(stats + 128 * half + 16 * q);
              d4 = ld_shared4(stats + 256 + 128 * half + 16 * q);
            }
            const float lv[4] = {l4.x, l4.y, l4.z, l4.w}, dv[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float x = ex2(fmaf(__uint_as_float(pr[4 * q + e]), c, -lv[e]));
              pr[4 * q + e] = __float_as_uint(x);
              t[4 * q + e] = __float_as_uint(x * (__uint_as_float(t[4 * q + e]) - dv[e]));
            }
          }
          if (mask) {
            // KV: the row is the key; its queries are allowed from `first` on
            const int n_ok = (KV ? 0 : min(p.causal ? max(i + 1, pf) : p.L, p.L)) - c0;
            const int first = (KV && p.causal && i >= pf ? i : 0) - c0;
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (KV ? e < first : e >= n_ok) pr[e] = t[e] = 0u;
            if (doc) {
              const int4* dd = reinterpret_cast<const int4*>(doc + c0);
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const int4 v = __ldg(dd + e);
                if (v.x != id) pr[4 * e] = t[4 * e] = 0u;
                if (v.y != id) pr[4 * e + 1] = t[4 * e + 1] = 0u;
                if (v.z != id) pr[4 * e + 2] = t[4 * e + 2] = 0u;
                if (v.w != id) pr[4 * e + 3] = t[4 * e + 3] = 0u;
              }
            }
          }
          if (grad) {
            const int base = c0 - i0;                    // distance of the patch's corner
            if (base - 31 >= reach || base + 31 <= -reach) {
              float z = 0.f;
#pragma unroll
              for (int e = 0; e < 32; ++e) z += __uint_as_float(t[e]);
              if (base > 0) hi_sum += z;
              else lo_sum += z;
            } else {
              __syncwarp();
#pragma unroll
              for (int e = 0; e < 32; ++e) my_patch[lane * 33 + e] = __uint_as_float(t[e]);
              __syncwarp();
              // lane: the diagonals of distance base + lane (columns from
              // `lane` on) and base + lane - 32 (the wrapped rest)
              float up = 0.f, down = 0.f;
#pragma unroll 8
              for (int e = 0; e < 32; ++e) {
                const float z = my_patch[e * 33 + ((e + lane) & 31)];
                if (e + lane < 32) up += z;
                else down += z;
              }
              const int du = base + lane, dn = du - 32;
              if (du >= reach) hi_sum += up;
              else if (du <= -reach) lo_sum += up;
              else my_dist[du + reach] += up;
              __syncwarp();
              if (dn >= reach) hi_sum += down;
              else if (dn <= -reach) lo_sum += down;
              else my_dist[dn + reach] += down;
            }
          }
          if (cap > 0.f) {     // 1 - tanh^2 = 4 q (1 - q)
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const float q = __uint_as_float(s[e]);
              t[e] = __float_as_uint(__uint_as_float(t[e]) * (4.f * q * (1.f - q)));
            }
            if (mask) {        // a masked score may have been NaN
#pragma unroll
              for (int e = 0; e < 32; ++e)
                if (pr[e] == 0u) t[e] = 0u;
            }
          }
          uint32_t w[16];
          if (KV) {
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = bf16_pair(__uint_as_float(pr[2 * e]), __uint_as_float(pr[2 * e + 1]));
            tmem_st16(s_col + 16 * half, w);
          }
#pragma unroll
          for (int e = 0; e < 16; ++e) w[e] = bf16_pair(__uint_as_float(t[2 * e]), __uint_as_float(t[2 * e + 1]));
          tmem_st16(d_col + 16 * half, w);
        }
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(&pfull[wg]);
      }
    }
    if (n > 0) {
      wait.on_warp(afull, 0, 37);
      tc_fence_after();
    }
    // each warpgroup stores half of the columns of each sum
#pragma unroll 1
    for (int o = 0; o < (KV ? 2 : 1); ++o) {
      const Strided& out = !KV ? p.dq : o ? p.dk : p.dv;
      const float mul = KV && !o ? 1.f : p.scale;
      bf16* row = static_cast<bf16*>(out.p) + b * out.sb + int64_t(i) * out.sl + (KV ? kh : h0) * out.sh;
#pragma unroll 1
      for (int g = 0; g < DP / 64; ++g) {
        const int col = 32 * (wg * (DP / 64) + g);
        uint32_t a[32];
        if (n > 0) {
          tmem_ld32(tmem + lanes + 256 + o * DP + col, a);
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) a[e] = 0u;
        }
        if (i >= p.L) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (col + 8 * e >= p.D) break;
          uint32_t w[4];
#pragma unroll
          for (int k = 0; k < 4; ++k)
            w[k] = bf16_pair(__uint_as_float(a[8 * e + 2 * k]) * mul, __uint_as_float(a[8 * e + 2 * k + 1]) * mul);
          reinterpret_cast<uint4*>(row + col)[e] = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
    }
    if (grad) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        lo_sum += __shfl_xor_sync(0xffffffffu, lo_sum, o);
        hi_sum += __shfl_xor_sync(0xffffffffu, hi_sum, o);
      }
      __syncwarp();
      if (lane == 0) {
        my_dist[0] += lo_sum;
        my_dist[2 * reach] += hi_sum;
      }
      asm volatile("bar.sync 3, 256;" ::: "memory");
      const int64_t parts = int64_t(p.B) * tiles;
      for (int k = warp; k < p.buckets; k += 8) {
        float z = 0.f;
        for (int e = lane; e < 2 * reach + 1; e += 32)
          if (map[e] == k)
#pragma unroll
            for (int w = 0; w < 8; ++w) z += dist[w * nd + e];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
        if (lane == 0) p.part[(int64_t(h0) * p.buckets + k) * parts + int64_t(b) * tiles + tile] = z;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kMma) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

constexpr size_t kSmemLimit = 232448;

template <int DP, bool KV>
cudaError_t launch(BwdParams bp, cudaStream_t st) {
  using F = Bwd<DP, KV>;
  const bool grad = !KV && bp.s.dtable;
  int stages = kMaxStages;
  auto need = [&](int n) { return F::smem(bp.s.L, n, bp.s.table != nullptr, grad, bp.s.reach); };
  while (stages > 2 && need(stages) > kSmemLimit) --stages;
  bp.s.stages = stages;
  const size_t smem = need(stages);
  auto k = scored_bwd_tc_k<DP, KV>;
  cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem));
  if (e != cudaSuccess) return e;
  const int64_t tiles = ceil_div(bp.s.L, 128);
  return launch_k(k, dim3(unsigned(tiles * bp.s.B * (KV ? bp.s.KV : bp.s.H))), dim3(kThreads), smem, st, bp);
}

}  // namespace

cudaError_t scored_bwd_tc(const ScoredParams& p, cudaStream_t st, bool* ok) {
  BwdParams q, k;
  q.s = k.s = p;
  *ok = scored_map(&q.x, p.q, p, p.H, 128) && scored_map(&q.y, p.dout, p, p.H, 128) &&
        scored_map(&q.u, p.k, p, p.KV, 64) && scored_map(&q.w, p.v, p, p.KV, 64) &&
        scored_map(&k.x, p.k, p, p.KV, 128) && scored_map(&k.y, p.v, p, p.KV, 128) &&
        scored_map(&k.u, p.q, p, p.H, 64) && scored_map(&k.w, p.dout, p, p.H, 64);
  if (!*ok) return cudaSuccess;
  cudaError_t e = p.D <= 64 ? launch<64, true>(k, st) : launch<128, true>(k, st);
  if (e != cudaSuccess) return e;
  return p.D <= 64 ? launch<64, false>(q, st) : launch<128, false>(q, st);
}

cudaError_t scored_bwd_error(int* word) { return cudaMemcpyFromSymbol(word, g_err, sizeof(int)); }

}  // namespace fo
