// Scored attention backward on the tensor cores (fo_scored.h): bf16, head
// width a multiple of 8 up to 128.
//
// One kernel body, launched twice.  A CTA keeps a tile of 128 rows of X and Y
// in shared memory and walks blocks of 64 rows of U and W:
//   KV = false  rows are queries:  X = Q, Y = dO, U = K, W = V
//               S = X U^T, dP = Y W^T,  dQ += dS U, and P U
//   KV = true   rows are keys:     X = K, Y = V, U = Q, W = dO, over every
//               query head of the group
//               S^T = X U^T, dP^T = Y W^T,  dV += P^T W, dK += dS^T U, and the
//               table gradient
// so each gradient is a sum in one CTA (or cluster), in a fixed order, without atomics; the
// price is that S and dP are formed twice, and P U (8 products instead of 5).  An
// alternative that adds dQ in global memory would save three products and lose
// reproducibility.
// S and dP take 64 TMEM columns each, in three buffers where the sums leave
// room (two for head widths above 64): two groups of 256 threads
// process alternate blocks, so that one's arithmetic runs while the other's
// products do, and a third buffer keeps the scores one block ahead.  A row is
// shared by two threads, 32 columns each, which form P from all 32 at once and
// dS in two passes of 16.  S is handed over before dP, whose products run
// while P is formed; P is handed over before dS where there are only two
// buffers (capped 2048: 294 -> 275 us, causal 16384 of width 128: 1510 ->
// 1400; with three the extra wait cost what it gained; so it did for queries
// under a cap, whose P is formed with dS).  P and dS go back to
// TMEM as bf16 over the scores they came from, as A operands of the
// accumulating products; no score touches shared memory.  Row statistics
// (scored_delta_k) are per column where rows are keys and ride along in each
// stage.
// D = dO . O carries the rounding of O (and the truncating sums of the tensor
// cores that formed it), which would leave each row's dS with a sum of -dD
// instead of 0, most of it in whichever bucket holds most keys, and dQ with
// -dD P K.  The query pass, launched first, sums its dS rows in fp32.  The sum
// goes into D for the second launch, so that dK and the table gradient come
// from the exact D, and sum * P K (under a cap each pair with its derivative,
// like dS) is taken off dQ at the end, which costs the product P U.  Without it
// dQ was off by 0.3% beside the roundings' 0.24% with values of mean 0, and with
// values of mean 1 by 1.6% at 16384 keys and 13% at 131072, where the gradients
// that are left are small beside D; it takes 2 to 8% of the backward pass (16384
// tokens 1369 -> 1455 us, 4 x 2048 capped tokens 275 -> 297).
// The table gradient sums dS in fp32 by distance: each warp turns 32 x 16
// patches through shared memory so that a lane sums a diagonal, into arrays by
// distance shared by the two warps of a row group, one after the other;
// patches beyond the reach are one sum per thread.
// Where the key tiles are fewer than the SMs can take, a cluster of blocks
// shares one: each walks every n-th block of queries, and the first two add up
// dV and dK through distributed shared memory, in the order of the ranks.
// Rounding: P and dS to bf16 before their products, each gradient once (the
// table's in the table's type).
#include "fo_scored_tc.cuh"

namespace fo {

namespace {

__device__ GaveUp g_err;

struct BwdParams {
  ScoredParams s;
  CUtensorMap x, y, u, w;
};

constexpr int kThreads = 608;           // sixteen warps of arithmetic; TMA, MMA and padding warps
constexpr int kTma = 16, kMma = 17, kClean = 18;
constexpr int kMaxStages = 6;
constexpr int kBlock = 0x3fff, kMasked = 0x4000, kPadded = 0x8000;   // entries of the list of blocks: kMaxLen / 64 = 2^14
constexpr int kPatch = 32 * 17;         // floats of a warp's 32 x 16 patch, rows 17 apart

template <int DP, bool KV>
struct Bwd {
  static constexpr int kX = DP / 64 * 16384;        // 128 rows
  static constexpr int kU = DP / 64 * 8192;         // 64 rows
  static constexpr int kStats = KV ? 512 : 0;       // lse and D of 64 queries
  static constexpr int kStage = 2 * kU + (KV ? 1024 : 0);
  static constexpr int kBufs = DP == 128 ? 2 : 3;          // TMEM buffers of S and dP; the sums follow
  static constexpr int kBars = 1 + 3 * kMaxStages + 4 * kBufs + 2;
  // X, Y, stages, barriers (and the TMEM slot and the number of blocks), the
  // list of blocks, row sums of dS, bias, table-gradient arrays
  // (of one of `share` blocks that divide the list)
  __host__ __device__ static int list_bytes(int L, int share) {
    const int steps = (L + 63) / 64;
    return ((steps + share - 1) / share + 7) / 8 * 16;
  }
  static size_t smem(int L, int share, int stages, bool table, bool grad, int reach) {
    size_t n = 1024 + 2 * kX + size_t(stages) * kStage + 8 * (kBars + 1) + list_bytes(L, share);
    if (!KV) n += 4 * 4 * 128;
    if (table) n += 4 * kBiasFloats;
    if (grad) n += 4 * (16 * kPatch + 8 * dist_floats(reach)) + 2 * kMaxReach + 4;
    return n;
  }
  // Stages that fit in shared memory, 0 where too few do: kBufs steps are in
  // flight.  Only the keys of widths above 64 with the gradient of a table whose
  // reach is above about 380 can be too large, because of the list of a sequence
  // of 780,000 tokens (reach 512) and more.
  static int stages(const ScoredParams& p) {
    const int share = KV ? p.share : 1;
    int n = kMaxStages;
    while (n >= kBufs && smem(p.L, share, n, p.table, KV && p.dtable, p.reach) > kSmemLimit) --n;
    return n < kBufs ? 0 : n;
  }
  __host__ __device__ static int dist_floats(int reach) { return (2 * reach + 1 + 3) / 4 * 4; }
};

template <int DP, bool KV, int BIAS, int CAP>
__global__ void __launch_bounds__(kThreads, 1) scored_bwd_tc_k(const __grid_constant__ BwdParams bp) {
  using F = Bwd<DP, KV>;
  // the cap's derivative multiplies P as well (rows are queries)
  constexpr bool kChained = !KV && CAP;
  constexpr bool kSplit = DP == 128 && !kChained;            // P handed over before dS
  const ScoredParams& p = bp.s;
  extern __shared__ __align__(1024) char smem_raw[];
  char* sm = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);    // 1024-byte aligned
  char *sX = sm, *sY = sm + F::kX, *ring = sm + 2 * F::kX;
  const int stages = p.stages;
  uint64_t* bars = reinterpret_cast<uint64_t*>(ring + stages * F::kStage);
  uint64_t *xfull = bars, *full = bars + 1, *empty = full + kMaxStages, *clean = empty + kMaxStages,
           *sfull = clean + kMaxStages, *pfull = sfull + F::kBufs, *dfull = pfull + F::kBufs,
           *tfull = dfull + F::kBufs, *afull = tfull + F::kBufs, *done = afull + 1;
  uint32_t* tslot = reinterpret_cast<uint32_t*>(bars + F::kBars);
  // blocks of 64 columns with allowed pairs, in ascending order: the index,
  // with kMasked where some pairs are not allowed and kPadded where there is
  // padding
  uint16_t* list = reinterpret_cast<uint16_t*>(bars + F::kBars + 1);
  float* rowsum = reinterpret_cast<float*>(reinterpret_cast<char*>(list) +
                                             F::list_bytes(p.L, KV ? p.share : 1));   // KV false: [4][128]
  float* bias = rowsum + (KV ? 0 : 512);
  const bool grad = KV && BIAS == kBiasTable && p.dtable;
  float* patch = bias + (BIAS == kBiasTable ? kBiasFloats : 0);
  float* dist = patch + 16 * kPatch;
  const int nd = F::dist_floats(p.reach);
  uint8_t* map = reinterpret_cast<uint8_t*>(dist + 8 * nd);

  const int warp = __shfl_sync(0xffffffffu, int(threadIdx.x) / 32, 0), lane = threadIdx.x % 32;
  const int heads = KV ? p.KV : p.H, tiles = (p.L + 127) / 128, share = KV ? p.share : 1,
            rank = KV ? int(blockIdx.x) % share : 0, work = int(blockIdx.x) / share, bh = work % (p.B * heads);
  const int slot0 = work / (p.B * heads), tile = KV ? slot0 : tiles - 1 - slot0;   // longest causal first
  const int r0 = tile * 128, b = bh / heads, h0 = KV ? (bh % heads) * p.G : bh % heads, kh = h0 / p.G;
  const int groups = KV ? p.G : 1;
  if (threadIdx.x == 0) {
    mbar_init(xfull, 1);
    for (int e = 0; e < stages; ++e) {
      mbar_init(&full[e], 1);
      mbar_init(&empty[e], 1);
      mbar_init(&clean[e], 1);
    }
    for (int e = 0; e < F::kBufs; ++e) {
      mbar_init(&sfull[e], 1);
      mbar_init(&pfull[e], 8);           // P written (one arrival per warp)
      mbar_init(&dfull[e], 1);
      mbar_init(&tfull[e], 8);           // dS written
    }
    mbar_init(afull, 1);
    mbar_init(done, 1);
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
  const float unit = CAP ? 1.f : p.scale, c = unit * kLog2e;
  const int pf = p.prefix ? p.prefix[b] : 0;
  const int2* blk = p.blk ? p.blk + int64_t(b) * (p.Lp / kScoredBlock) : nullptr;
  if (BIAS == kBiasTable && !KV) load_bias(bias, p, h0, 1.f / unit, threadIdx.x, kThreads);
  if (grad) {
    for (int e = threadIdx.x; e < 8 * nd; e += kThreads) dist[e] = 0.f;
    for (int e = threadIdx.x; e < 2 * p.reach + 1; e += kThreads) map[e] = p.map[e];
  }
  if (warp == kClean) {
    int2 rd = make_int2(0, 0);
    if (blk) rd = doc_join(blk[r0 / 64], blk[r0 / 64 + 1]);
    uint32_t n = 0, pads = 0;
    for (int first = 0; first * 64 < p.L; first += 32) {
      const int c0 = (first + lane) * 64;
      int cls = kScoredNone;
      bool pad = false;
      if (c0 < p.L) {
        int2 cd = make_int2(0, 0);
        if (blk) cd = blk[c0 / 64];
        cls = KV ? scored_class(p, pf, c0, c0 + 64, r0, r0 + 128, blk != nullptr, cd, rd)
                 : scored_class(p, pf, r0, r0 + 128, c0, c0 + 64, blk != nullptr, rd, cd);
        // keys past the end are zeros in shared memory, not absent: as columns
        // they would enter dQ, as rows the table gradient; queries past the
        // end have P = 0
        if (cls == kScoredAll && (KV ? grad && r0 + 128 > p.L : c0 + 64 > p.L)) cls = kScoredSome;
        pad = cd.x < 0 && cls != kScoredNone;
      }
      const uint32_t on = __ballot_sync(0xffffffffu, cls != kScoredNone);
      pads |= __ballot_sync(0xffffffffu, pad);
      const uint32_t at = n + __popc(on & ((1u << lane) - 1));
      if (cls != kScoredNone && int(at) % share == rank)
        list[int(at) / share] = uint16_t((first + lane) | (cls == kScoredSome ? kMasked : 0) | (pad ? kPadded : 0));
      n += __popc(on);
    }
    n = (n + uint32_t(share - 1 - rank)) / uint32_t(share);          // of this block
    if (lane == 0) tslot[1] = n | (pads ? 0x80000000u : 0u);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // S and dP of buffer k: columns 128 k and 128 k + 64; sums at `acc` and acc + DP
  const uint32_t tmem = *tslot, acc = tmem + 128 * F::kBufs;
  const int count = int(tslot[1] & 0x7fffffffu);
  const bool any_padding = tslot[1] >> 31;
  pdl_trigger();
  Waits wait(&g_err);
  // Warps of arithmetic: 16 columns g of output o, of the sums of this
  // thread's row that it stores (each of the four warps of a row group has a
  // quarter of the columns).
  auto sums_of = [&](int o, int g, uint32_t (&a)[16]) {
    if (count > 0) {
      tmem_ld16_issue(acc + (uint32_t(32 * (warp % 4)) << 16) + o * DP + DP / 4 * (warp / 4) + 16 * g, a);
      tmem_ld16_wait(a);
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) a[e] = 0u;
    }
  };
  auto store = [&](int o, int g, const uint32_t (&a)[16]) {
    const Strided& out = !KV ? p.dq : o ? p.dk : p.dv;
    const float mul = KV && !o ? 1.f : CAP ? p.scale / kChainUp : p.scale;      // ch holds kChainUp derivatives
    const int i = r0 + 32 * (warp % 4) + lane, col = DP / 4 * (warp / 4) + 16 * g;
    if (i >= p.L) return;
    bf16* row = static_cast<bf16*>(out.p) + b * out.sb + int64_t(i) * out.sl + (KV ? kh : h0) * out.sh;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if (col + 8 * e >= p.D) break;
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        w[k] = bf16_pair(__uint_as_float(a[8 * e + 2 * k]) * mul, __uint_as_float(a[8 * e + 2 * k + 1]) * mul);
      reinterpret_cast<uint4*>(row + col)[e] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  };
  // Where blocks share a tile: output o is added up by block o; the others
  // leave theirs where X, Y and the stages were, four values of each thread
  // together (16 DP / 64 vectors of 512 threads: 64 KB per 64 columns).
  auto left = [&](int o, int g, int e) { return sm + ((o * (DP / 64) + g) * 4 + e) * 8192 + 16 * int(threadIdx.x); };

  if (warp == kTma) {
    if (lane == 0) {
      mbar_expect_tx(xfull, 2 * F::kX);
      for (int s = 0; s < DP / 64; ++s) {
        tma_4d(sX + s * 16384, &bp.x, xfull, 64 * s, r0, KV ? kh : h0, b);
        tma_4d(sY + s * 16384, &bp.y, xfull, 64 * s, r0, KV ? kh : h0, b);
      }
      int it = 0;
      for (int g = 0; g < groups && !wait.dead; ++g) {
        const int64_t stat = (int64_t(b) * p.H + h0 + g) * p.Lp;
        for (int k = 0; k < count; ++k, ++it) {
          const int cb = list[k] & kBlock;
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
      // every copy has landed before the block ends, whichever role gave up
      mbar_wait(xfull, 0);
      for (int e = max(0, it - stages); e < it; ++e) mbar_wait(&full[e % stages], (e / stages) & 1);
    }
  } else if (warp == kMma) {
    constexpr uint32_t id_s = instr_desc(64, false, false), id_a = instr_desc(DP, false, true);
    const uint32_t ring_at = smem_u32(ring);
    const Operand<16> x(smem_u32(sX)), y(smem_u32(sY));
    uint64_t* landed = any_padding ? clean : full;      // U and W have landed, without padding
    const int total = count * groups;
    int in = 0, in_slot = 0, in_phase = 0;           // the next step whose scores are formed
    Ring<F::kBufs> in_buf, buf;
    wait.on_lanes(xfull, 0, 33);
    int slot = 0;
    // one loop with one place for each product: kBufs steps of scores ahead
    for (int n = -F::kBufs; n < total; ++n) {
      if (n >= 0) {
        const uint32_t a = tmem + 128 * buf.at;
        const Operand<8192> u(ring_at + slot * F::kStage), w(ring_at + slot * F::kStage + F::kU);
        wait.on_lanes(kSplit ? &pfull[buf.at] : &tfull[buf.at], buf.phase, 34);
        tc_fence_after();
#pragma unroll
        for (int e = 0; e < 4; ++e)
          mma_ts(acc, a + 32 * (e >> 1) + 8 * (e & 1), (KV ? w : u).at(2048 * e), id_a, e > 0 ? 1u : uint32_t(n));
        if (kSplit) {
          wait.on_lanes(&tfull[buf.at], buf.phase, 39);
          tc_fence_after();
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
          mma_ts(acc + DP, a + 64 + 32 * (e >> 1) + 8 * (e & 1), u.at(2048 * e), id_a,
                 e > 0 ? 1u : uint32_t(n));
        commit_to(&empty[slot]);
        if (n + 1 == total) commit_to(afull);
        if (++slot == stages) slot = 0;
        buf.step();
      }
      if (in < total) {
        // after the commit above: with kBufs stages, this is the one it frees
        wait.on_lanes(&landed[in_slot], in_phase, 32);
        tc_fence_after();
        const uint32_t d = tmem + 128 * in_buf.at;
        const Operand<16> u(ring_at + in_slot * F::kStage), w(ring_at + in_slot * F::kStage + F::kU);
#pragma unroll
        for (int e = 0; e < DP / 16; ++e)
          mma_ss(d, x.at((e >> 2) * 16384 + 32 * (e & 3)), u.at((e >> 2) * 8192 + 32 * (e & 3)), id_s, e > 0 ? 1u : 0u);
        commit_to(&sfull[in_buf.at]);
#pragma unroll
        for (int e = 0; e < DP / 16; ++e)
          mma_ss(d + 64, y.at((e >> 2) * 16384 + 32 * (e & 3)), w.at((e >> 2) * 8192 + 32 * (e & 3)), id_s,
                 e > 0 ? 1u : 0u);
        commit_to(&dfull[in_buf.at]);
        ++in;
        in_buf.step();
        if (++in_slot == stages) in_slot = 0, in_phase ^= 1;
      }
      // off the waits' path; what was issued after one gave up is void anyway
      if (__any_sync(0xffffffffu, wait.dead)) break;
    }
    // no product is in flight when the block ends and its memory is another's
    commit_to(done);
    mbar_wait(done, 0);
    __syncwarp();
  } else if (warp == kClean) {
    if (any_padding) {
      const int32_t* doc = p.doc + int64_t(b) * p.Lp;
      int slot = 0, phase = 0;
      for (int g = 0; g < groups; ++g) {
        for (int k = 0; k < count && !wait.dead; ++k) {
          const int cb = list[k] & kBlock;
          wait.on_warp(&full[slot], phase, 38);
          if (list[k] & kPadded) {
            clear_padding(ring + slot * F::kStage, 64, DP / 64, doc + cb * 64);
            if (KV) clear_padding(ring + slot * F::kStage + F::kU, 64, DP / 64, doc + cb * 64);
          }
          arrive_warp(&clean[slot]);
          if (++slot == stages) slot = 0, phase ^= 1;
        }
      }
    }
  } else {
    const int side = warp / 8, half = warp / 4 % 2, quarter = warp % 4, i0 = r0 + 32 * quarter, i = i0 + lane;
    const uint32_t lanes = uint32_t(32 * quarter) << 16;
    const int32_t* doc = p.doc ? p.doc + int64_t(b) * p.Lp : nullptr;
    int id = doc && i < p.L ? doc[i] : 0;
    if (id < 0) id = INT32_MIN;            // padding equals nothing, itself included
    // position mask: rows that are queries allow columns below `edge`, rows
    // that are keys allow columns from `edge` on (none past the end)
    const int edge = KV ? (i >= p.L ? INT32_MAX : p.causal && i >= pf ? i : 0) : min(p.causal ? max(i + 1, pf) : p.L, p.L);
    const int64_t stat = (int64_t(b) * p.H + h0) * p.Lp + i;
    const float row_lse = KV ? 0.f : p.lse2[stat];
    const float row_d = KV ? 0.f : p.delta[stat];
    const F2 c2 = f2(c, c);
    F2 eps = f2(0.f, 0.f);                 // KV false: sum of this thread's dS
    float lo_sum = 0.f, hi_sum = 0.f;      // table gradient beyond the reach
    float* my_patch = patch + warp * kPatch;
    float* my_dist = dist + (4 * side + quarter) * nd;
    const int pair = 1 + 4 * side + quarter;
    int slot = side, phase = 0;              // this side's stage in shared memory
    Ring<F::kBufs, 2> buf(side);             // this side's buffer
    for (int g = 0; g < groups; ++g) {
      const Shape a = shape_of(p, h0 + g, unit, bias);
      if (KV && BIAS == kBiasTable) {
        asm volatile("bar.sync 9, 512;" ::: "memory");
        load_bias(bias, p, h0 + g, 1.f / unit, threadIdx.x, 512);
        asm volatile("bar.sync 9, 512;" ::: "memory");
      }
      for (int k = (side + g * count) & 1; k < count; k += 2) {      // every other step of the whole walk
        const uint32_t entry = list[k];
        const int cb = entry & kBlock;
        const bool mask = entry & kMasked;
        const uint32_t s_col = tmem + lanes + 128 * buf.at + 32 * half, d_col = s_col + 64;
        if (KV) wait.on_lanes(&full[slot], phase, 35);              // its statistics
        wait.on_lanes(&sfull[buf.at], buf.phase, 36);
        tc_fence_after();
        const uint32_t stats = smem_u32(ring + slot * F::kStage + 2 * F::kU) + 128 * half;
        const int c0 = cb * 64 + 32 * half;
        // P = 2^(c x - lse)
        uint32_t s[32], ch[16];                 // ch: kChainUp (1 - tanh^2) of the cap, pairs of fp16
        tmem_ld32_issue(s_col, s);
        tmem_ld32_wait(s);
        {
          // distance j - i: c0 + e - i (rows are queries) or i - c0 - e
          const int lo = KV ? i0 - c0 - 31 : c0 - i0 - 31;
          shape_scores<32, BIAS, CAP, KV ? -1 : 1, true>(s, ch, a, KV ? i - c0 : c0 - i, lo, lo + 62);
        }
#pragma unroll
        for (int e = 0; e < 32; e += 4) {
          F2 l0 = f2(row_lse, row_lse), l1 = l0;
          if (KV) ld_pairs(stats + 4 * e, l0, l1);
          float x, y;
          split(fma2(f2u(s[e], s[e + 1]), c2, l0), x, y);
          s[e] = __float_as_uint(ex2(x)), s[e + 1] = __float_as_uint(ex2(y));
          split(fma2(f2u(s[e + 2], s[e + 3]), c2, l1), x, y);
          s[e + 2] = __float_as_uint(ex2(x)), s[e + 3] = __float_as_uint(ex2(y));
        }
        if (mask) {
          const int first = edge - c0;
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (KV ? e < first : e >= first) s[e] = 0u;
          if (doc) {
            const int4* dd = reinterpret_cast<const int4*>(doc + c0);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int4 v = __ldg(dd + e);
              if (v.x != id) s[4 * e] = 0u;
              if (v.y != id) s[4 * e + 1] = 0u;
              if (v.z != id) s[4 * e + 2] = 0u;
              if (v.w != id) s[4 * e + 3] = 0u;
            }
          }
        }
        if (!kChained) {
          uint32_t w[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) w[e] = bf16_pair(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1]));
          tmem_st16(s_col, w);
          if (kSplit) {
            tmem_st_wait();
            tc_fence_before();
            arrive_warp(&pfull[buf.at]);
          }
        }
        // dS = P (dP - D)
        wait.on_lanes(&dfull[buf.at], buf.phase, 40);
        tc_fence_after();
#pragma unroll
        for (int pass = 0; pass < 2; ++pass) {
          uint32_t t[16];
          tmem_ld16_issue(d_col + 16 * pass, t);
          tmem_ld16_wait(t);
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            F2 d0 = f2(row_d, row_d), d1 = d0;
            if (KV) ld_pairs(stats + 256 + 64 * pass + 4 * e, d0, d1);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int at = e + 2 * k, sat = 16 * pass + at;
              float x, y;
              split(mul2(f2u(s[sat], s[sat + 1]), add2(f2u(t[at], t[at + 1]), k ? d1 : d0)), x, y);
              t[at] = __float_as_uint(x), t[at + 1] = __float_as_uint(y);
            }
          }
          if (mask) {                          // what stands in a masked place may have been NaN
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (s[16 * pass + e] == 0u) t[e] = 0u;
          }
          if (!KV) {
#pragma unroll
            for (int e = 0; e < 16; e += 2) eps = add2(eps, f2u(t[e], t[e + 1]));
          }
          if (KV && BIAS == kBiasTable && grad) {
            // the patch's distances: base + row - column; whether any of the
            // block's is within the reach is the same for the warps of a row
            // group, which meet at barriers below
            const int base = i0 - c0 - 16 * pass, corner = i0 - cb * 64;
            if (corner - 63 >= a.reach || corner + 31 <= -a.reach) {
              F2 z = f2u(t[0], t[1]);
#pragma unroll
              for (int e = 2; e < 16; e += 2) z = add2(z, f2u(t[e], t[e + 1]));
              float x, y;
              split(z, x, y);
              if (corner > 0) hi_sum += x + y;
              else lo_sum += x + y;
            } else {
              __syncwarp();
#pragma unroll
              for (int e = 0; e < 16; ++e) my_patch[lane * 17 + e] = __uint_as_float(t[e]);
              __syncwarp();
              // lane: distance base + lane (rows lane + e) and, where the rows
              // wrap, base + lane - 32
              float up = 0.f, down = 0.f;
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const float z = my_patch[((lane + e) & 31) * 17 + e];
                if (lane + e < 32) up += z;
                else down += z;
              }
              // the two warps of these rows write one after the other
              const int du = base + lane, dn = du - 32;
              auto put = [&](int d, float z) {
                if (d >= a.reach) hi_sum += z;
                else if (d <= -a.reach) lo_sum += z;
                else my_dist[d + a.reach] += z;
              };
              if (half) asm volatile("bar.sync %0, 64;" ::"r"(pair) : "memory");
              put(du, up);
              __syncwarp();
              if (lane >= 17) put(dn, down);
              if (!half) asm volatile("bar.sync %0, 64;" ::"r"(pair) : "memory");
              asm volatile("bar.sync %0, 64;" ::"r"(pair) : "memory");
            }
          }
          if (CAP) {
            uint32_t pc[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&ch[8 * pass + e]));
              float x, y;
              split(mul2(f2u(t[2 * e], t[2 * e + 1]), f2(f.x, f.y)), x, y);
              t[2 * e] = __float_as_uint(x), t[2 * e + 1] = __float_as_uint(y);
              if (kChained) {
                split(mul2(f2u(s[16 * pass + 2 * e], s[16 * pass + 2 * e + 1]), f2(f.x, f.y)), x, y);
                pc[e] = bf16_pair(x, y);
              }
            }
            if (mask) {
#pragma unroll
              for (int e = 0; e < 16; ++e)
                if (s[16 * pass + e] == 0u) {
                  t[e] = 0u;
                  if (kChained) pc[e / 2] &= e & 1 ? 0x0000ffffu : 0xffff0000u;
                }
            }
            if (kChained) tmem_st8(s_col + 8 * pass, pc);
          }
          uint32_t w[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e] = bf16_pair(__uint_as_float(t[2 * e]), __uint_as_float(t[2 * e + 1]));
          tmem_st8(d_col + 8 * pass, w);
        }
        tmem_st_wait();
        tc_fence_before();
        arrive_warp(&tfull[buf.at]);
        buf.step();
        slot += 2;
        if (slot >= stages) slot -= stages, phase ^= 1;
      }
      if (grad) {
        // this head's sums by distance -> buckets -> its partial gradient
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
          lo_sum += __shfl_xor_sync(0xffffffffu, lo_sum, o);
          hi_sum += __shfl_xor_sync(0xffffffffu, hi_sum, o);
        }
        for (int turn = 0; turn < 2; ++turn) {
          __syncwarp();
          if (turn == half && lane == 0) {
            my_dist[0] += lo_sum;
            my_dist[2 * a.reach] += hi_sum;
          }
          asm volatile("bar.sync 9, 512;" ::: "memory");
        }
        const int64_t parts = int64_t(p.B) * tiles * share;
        for (int k = warp; k < p.buckets; k += 16) {
          float z = 0.f;
          for (int e = lane; e < 2 * a.reach + 1; e += 32)
            if (map[e] == k)
#pragma unroll
              for (int w = 0; w < 8; ++w) z += dist[w * nd + e];
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
          if (lane == 0) p.part[(int64_t(h0 + g) * p.buckets + k) * parts + (int64_t(b) * tiles + tile) * share + rank] = z;
        }
        if (g + 1 < groups) {
          asm volatile("bar.sync 9, 512;" ::: "memory");
          for (int e = threadIdx.x; e < 8 * nd; e += 512) dist[e] = 0.f;
          lo_sum = hi_sum = 0.f;       // the next head's bias load synchronises
        }
      }
    }
    float off = 0.f;                       // KV false: the row's sum of dS, what D is off by
    if (!KV) {
      float x, y;
      split(eps, x, y);
      float* z = rowsum + 32 * quarter + lane;
      z[(2 * side + half) * 128] = x + y;
      asm volatile("bar.sync 9, 512;" ::: "memory");
      off = (z[0] + z[128]) + (z[256] + z[384]);
      if (warp < 4 && i < p.L) p.delta[stat] = row_d - off;
    }
    if (count > 0) {
      wait.on_lanes(afull, 0, 37);
      tc_fence_after();
    }
    if (share > 1 && count == 0) wait.on_lanes(xfull, 0, 41);     // before X and Y are written over
    if (!KV) {
#pragma unroll 1
      for (int g = 0; g < DP / 64; ++g) {
        uint32_t a[16], pu[16];
        sums_of(1, g, a);
        sums_of(0, g, pu);
#pragma unroll
        for (int e = 0; e < 16; ++e)
          a[e] = __float_as_uint(fmaf(-off, __uint_as_float(pu[e]), __uint_as_float(a[e])));
        store(1, g, a);
      }
    }
#pragma unroll 1
    for (int o = 0; o < (KV ? 2 : 0); ++o)
#pragma unroll 1
      for (int g = 0; g < DP / 64; ++g) {
        uint32_t a[16];
        if (share > 1 && o == rank) break;
        sums_of(o, g, a);
        if (share == 1) {
          store(o, g, a);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<uint4*>(left(o, g, e)) = make_uint4(a[4 * e], a[4 * e + 1], a[4 * e + 2], a[4 * e + 3]);
        }
      }
  }
  if (KV && share > 1) {
    __syncwarp();
    cluster_sync();
    if (warp < kTma && rank < 2) {
#pragma unroll 1
      for (int g = 0; g < DP / 64; ++g) {
        uint32_t a[16];
        sums_of(rank, g, a);
#pragma unroll 1
        for (int r = 0; r < share; ++r) {
          if (r == rank) continue;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint32_t at, v[4];
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(left(rank, g, e))), "r"(r));
            asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                         : "r"(at)
                         : "memory");
#pragma unroll
            for (int k = 0; k < 4; ++k)
              a[4 * e + k] = __float_as_uint(__uint_as_float(a[4 * e + k]) + __uint_as_float(v[k]));
          }
        }
        store(rank, g, a);
      }
    }
    __syncwarp();
    cluster_sync();                    // the others' memory has been read
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kMma) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

template <int DP, bool KV>
struct Launch {
  BwdParams& bp;
  cudaStream_t st;
  template <int BIAS, int CAP>
  cudaError_t operator()() const {
    using F = Bwd<DP, KV>;
    const ScoredParams& s = bp.s;
    const size_t smem = F::smem(s.L, KV ? s.share : 1, s.stages, BIAS == kBiasTable, KV && s.dtable, s.reach);
    auto k = scored_bwd_tc_k<DP, KV, BIAS, CAP>;
    static std::atomic<bool> allowed[kMaxDevices];
    const cudaError_t e = allow_smem(k, allowed);
    if (e != cudaSuccess) return e;
    const int64_t tiles = ceil_div(s.L, 128);
    if (KV) return launch_cluster(k, tiles * s.B * s.KV, kThreads, smem, s.share, st, bp);
    return launch_k(k, dim3(unsigned(tiles * s.B * s.H)), dim3(kThreads), smem, st, bp);
  }
};
// Both launches, or none where one does not fit.
template <int DP>
cudaError_t launch_both(BwdParams& queries, BwdParams& keys, cudaStream_t st, bool* ok) {
  queries.s.stages = Bwd<DP, false>::stages(queries.s);
  keys.s.stages = Bwd<DP, true>::stages(keys.s);
  *ok = queries.s.stages > 0 && keys.s.stages > 0;
  if (!*ok) return cudaSuccess;
  const cudaError_t e = with_shape(queries.s, Launch<DP, false>{queries, st});
  return e != cudaSuccess ? e : with_shape(keys.s, Launch<DP, true>{keys, st});
}

// How many blocks (a cluster) share a tile of keys: twice as many while each
// keeps enough steps of 64 queries to pay for its start and for adding up.
// Eight will do while every block has an SM of its own (8192 causal tokens, 4
// heads of 128 on 1: 488 -> 305 us; 2048 tokens of one head of 64: 46 -> 36,
// and 48 with four steps each).  With a causal mask a second block per SM
// evens out the tiles' lengths from 32 steps on (the same 305 -> 216; 8 steps,
// 2 x 1024 tokens, 8 heads of 64 on 2, took 56 us against 36), and up to four
// from 512 on (16384 tokens, 16 heads of 128 on 2: 2.87 -> 2.75 ms; 64 steps,
// 4 x 2048 tokens, 16 heads of 128 on 4, 308 us against 289).
int shared_by(const ScoredParams& p) {
  const int64_t sms = elementwise_blocks(INT64_MAX / 2, kThreads) / 8, blocks = ceil_div(p.L, 128) * p.B * p.KV;
  const int64_t steps = ceil_div(p.L, 64);
  int n = 1;
  while (n < kMaxShare && 2 * n <= steps) {
    const int64_t grid = 2 * n * blocks, each = steps * p.G / (2 * n);
    const int64_t room = !p.causal || each < 32 ? sms : each < 512 ? 2 * sms : 4 * sms;
    if (each < 8 || grid > room) break;
    n *= 2;
  }
  return n;
}

}  // namespace

cudaError_t scored_bwd_tc(ScoredParams& p, cudaStream_t st, bool* ok) {
  p.share = shared_by(p);
  BwdParams q, k;
  q.s = k.s = p;
  *ok = scored_map(&q.x, p.q, p, p.H, 128) && scored_map(&q.y, p.dout, p, p.H, 128) &&
        scored_map(&q.u, p.k, p, p.KV, 64) && scored_map(&q.w, p.v, p, p.KV, 64) &&
        scored_map(&k.x, p.k, p, p.KV, 128) && scored_map(&k.y, p.v, p, p.KV, 128) &&
        scored_map(&k.u, p.q, p, p.H, 64) && scored_map(&k.w, p.dout, p, p.H, 64);
  if (!*ok) return cudaSuccess;
  return p.D <= 64 ? launch_both<64>(q, k, st, ok) : launch_both<128>(q, k, st, ok);
}

cudaError_t scored_bwd_error(unsigned* told, int* code) { return gave_up_since(g_err, told, code); }

}  // namespace fo
