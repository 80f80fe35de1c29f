// gfx950 kernels of plain causal attention on packed sequences, forward and
// backward: the attention of Sec. 2.1 of the DMC paper, for layers that keep
// their full cache (and for the uncompressed model that DMC is measured
// against or taught by).  Query i of a sequence attends to its tokens j <= i:
//   S = Q K^T / sqrt(d),  P = softmax(S),  O = P V,  L = log sum exp(S)
//   dV = P^T dO,  dS = P (dO V^T - D),  D = sum(dO O),
//   dQ = dS K / sqrt(d),  dK = dS^T Q / sqrt(d)
// with dK and dV summed over the query heads of a kv head's group.
//
// Bound by the matrix cores and the vector work of the softmax beside them: 2
// products forward, 8 backward for the 5 of the formulas (dq: S, dP, dQ; the dV
// launch: S, dV; the dK launch: S, dP, dK).  One kernel for all of them would form
// S and dP once, but needs either atomics, whose order changes results, or the
// accumulators of all three; dV and dK in one launch, a product less, need 128
// accumulator and 64 operand registers, which leaves one wave per SIMD (not tried).
// Of the SIMD cycles of the large cases the matrix pipes are busy for 36 - 52 %
// (a large matrix product here reaches 47 % of its peak), vector instructions issue
// in 26 - 43 %; LDS moves data in 22 - 28 %, without bank conflicts.
//
// A workgroup owns a tile of one head (128 columns in bf16, 32 in fp32) of one
// sequence, whose other side streams past it in blocks of 32 rows.  Blocks and
// tiles start at the sequence's first token, so that a wave's 32 columns meet
// the diagonal in exactly one block.  Rows past a sequence's end are its last
// row again (in bounds whatever lies behind) with weight 0.
#include <algorithm>
#include <type_traits>

#include "dmc_mfma.h"

namespace dmc {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kTileShift = 7, kTile = 1 << kTileShift;     // bf16: tokens per workgroup
constexpr int kTileShift32 = 5, kTile32 = 1 << kTileShift32;   // fp32

// Head (of `heads`) and rank among the tiles of a workgroup.  Heads are dealt to
// the XCDs (workgroup i runs on XCD i mod 8) in runs where their count allows, so
// that a kv head's keys and values stay in one L2.
__device__ __forceinline__ void head_of_block(int heads, int &head, int &rank) {
  const int bid = blockIdx.x;
  if ((heads & 7) == 0) {
    const int per = heads >> 3, r = bid >> 3;
    rank = r / per;
    head = (bid & 7) * per + r - rank * per;
  } else {
    rank = bid / heads;
    head = bid - rank * heads;
  }
}

__device__ __forceinline__ float wave_sum(float x) {
  x = row_sum<32>(x);
  return x + __shfl_xor(x, 32, 64);
}

// The tile of a rank in descending order of length: tile k (from 1) of a query
// kernel's sequence takes k tiles' worth of blocks, in a key kernel (REVERSED)
// the k-th from its end does; heavy tiles that start last leave most of the chip
// idle.  With N(l) tiles of length l or more, found by bisection over l: the length
// of rank r is the largest l with N(l) > r, and the rank counts from N(l + 1) over
// the sequences that have such a tile.
constexpr int kSortSeqs = 256;   // sequences a wave holds the lengths of, four to a lane
template <bool REVERSED>
__device__ __forceinline__ PackedTile sorted_tile(const int32_t *cu, int seqs, int total, int rank, int shift) {
  constexpr int kPer = kSortSeqs / 64;
  const int lane = threadIdx.x & 63;
  int start[kPer], tiles[kPer], n[kPer];
  int most = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int b = j * 64 + lane;
    const bool here = b < seqs;
    start[j] = clamp_token(cu[here ? b : 0], total);
    const int end = clamp_token(cu[here ? b + 1 : 0], total);
    n[j] = here && end > start[j] ? end - start[j] : 0;
    tiles[j] = (n[j] + (1 << shift) - 1) >> shift;
    most = max(most, tiles[j]);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) most = max(most, __shfl_xor(most, o, 64));
  // (counts below 2^24: exact in floats)
  auto at_least = [&](int l) {
    int x = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) x += max(tiles[j] - l + 1, 0);
    return __builtin_amdgcn_readfirstlane(static_cast<int>(wave_sum(static_cast<float>(x))));
  };
  PackedTile t{0, 0, 0, -1};
  int lo = 1, hi = __builtin_amdgcn_readfirstlane(most) + 1;   // N(lo) > rank >= N(hi), if at all
  if (at_least(1) <= rank) return t;
  int above = 0;   // N(hi)
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1, c = at_least(mid);
    if (c > rank) {
      lo = mid;
    } else {
      hi = mid;
      above = c;
    }
  }
  int k = rank - above;   // among the sequences with a tile of length lo
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const unsigned long long has = __ballot(tiles[j] >= lo);
    const int c = __popcll(has);
    if (t.tile < 0 && k < c) {
      const bool mine = ((has >> lane) & 1) && __popcll(has & ((1ull << lane) - 1)) == k;
      const int src = 63 - __clzll(static_cast<long long>(__ballot(mine)));
      t.seq = j * 64 + src;
      t.start = __builtin_amdgcn_readlane(start[j], src);
      t.n = __builtin_amdgcn_readlane(n[j], src);
      t.tile = REVERSED ? __builtin_amdgcn_readlane(tiles[j], src) - lo : lo - 1;
    }
    k -= c;
  }
  t.seq = __builtin_amdgcn_readfirstlane(t.seq);
  t.start = __builtin_amdgcn_readfirstlane(t.start);
  t.n = __builtin_amdgcn_readfirstlane(t.n);
  t.tile = __builtin_amdgcn_readfirstlane(t.tile);
  return t;
}

// A workgroup's tile: by rank in descending length where the launch asks for it,
// else in the order of the sequences (last ones first for queries).
template <bool REVERSED>
__device__ __forceinline__ PackedTile tile_of_rank(const CausalParams &p, int rank, int ntiles, int shift) {
  if (p.sorted) return sorted_tile<REVERSED>(p.cu, p.seqs, p.total, rank, shift);
  return packed_tile(p.cu, p.seqs, p.total, REVERSED ? rank : ntiles - 1 - rank, shift);
}

// Parts that a query tile of `blocks` key blocks is cut into, four blocks or more
// each (of up to `most`).
__device__ __forceinline__ int tile_parts(int most, int blocks) { return max(1, min(most, blocks >> 2)); }

// Row `token`, head `h` of a strided tensor of ES-byte elements.
template <int ES>
__device__ __forceinline__ const char *row_at(const void *base, const int64_t (&st)[2], int64_t token, int h) {
  return static_cast<const char *>(base) + (token * st[0] + h * st[1]) * ES;
}

// ---------------------------------------------------------------------------
// bf16.  MODE 0 = forward, 1 = dq.  One workgroup = 4 waves = 128 queries of one
// head, a wave owning 32 (lane l: column l % 32, half l / 32).  Keys and values
// stream through LDS in blocks of 32 tokens (direct global -> LDS transfers, a
// ring of four blocks, three ahead):
//   S^T[key][col] = K . Q^T;   O^T[dim][col] += V^T P^T;   dQ^T[dim][col] += K^T dS^T
// Score row m is key pi(m) (bits 2 and 3 of m swapped), which makes a lane's
// score registers the operand of the second product.  Forward: block kb's
// exponentials run between the score products of block kb + 1.  5 sequences up to
// 8192, 32 heads, d 128: a forward pass 1045 us (952 TFLOP/s); 6 up to 4096, 32/8
// heads: forward 512 us, dq 657 us (medians of a trace).  dq at d = 128 holds queries,
// output gradients and accumulators in 192 registers and spills 10 of the rest.
// ---------------------------------------------------------------------------
template <int D, int MODE>
__global__ __launch_bounds__(kThreads, 2) void causal_query_kernel(CausalParams p, int ntiles) {
  constexpr int kSt = 4;               // ring slots
  constexpr int KS = D / 16, NTL = D / 32, RB = D * 2, CPR = D / 8, BLK = 32 * RB;
  constexpr int DPW = BLK / 16 / kThreads;
  constexpr int KSW = MODE == 0 ? 0 : 2;     // dq also reads keys transposed
  constexpr int VSW = MODE == 0 ? 1 : KSW;   // forward reads values transposed
  static_assert(DPW >= 1 && BLK % (16 * kThreads) == 0, "block split");
  static_assert(KS == 2 * NTL && KS > 3, "one transposed operand per score product");
  __shared__ __align__(16) unsigned char ring0[2 * BLK], ring1[2 * BLK], ring2[2 * BLK], ring3[2 * BLK];
  auto slot = [&](auto st_c) -> unsigned char * {
    constexpr int S = decltype(st_c)::value;
    if constexpr (S == 0) return ring0;
    else if constexpr (S == 1) return ring1;
    else if constexpr (S == 2) return ring2;
    else return ring3;
  };
  int h, rank;
  head_of_block(p.hq, h, rank);
  const PackedTile pt = tile_of_rank<false>(p, rank, ntiles, kTileShift);
  const int n = pt.n;
  if (pt.tile < 0 || pt.tile * kTile >= n) return;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, hb = lane >> 5;
  const int a = pt.tile * kTile + wave * 32;    // this wave's first token
  const int t = a + col;
  const bool colv = t < n;
  const int64_t token = pt.start + (colv ? t : 0);
  // The tile's key blocks; this workgroup's part of them.
  const int all = (min(n, pt.tile * kTile + kTile) + 31) >> 5, parts = tile_parts(p.query_parts, all), share = blockIdx.y;
  if (share >= parts) return;
  const int blk0 = all * share / parts, nblk = all * (share + 1) / parts;
  const int wave_hi = a < n ? min(min(a + 32, n), nblk * 32) : 0;   // keys < wave_hi feed this wave
  const int g = h / (p.hq / p.hkv);
  const uint4 zero4 = make_uint4(0, 0, 0, 0);
  const float sl2 = p.scale_log2;

  uint4 qop[KS], dop[MODE == 1 ? KS : 1];
  float Lc = 0.0f, Dc = 0.0f;
  {
    const char *qr = row_at<2>(p.q, p.qs, token, h);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qop[ks] = colv ? ld16(qr + ks * 32 + hb * 16) : zero4;
    if constexpr (MODE == 1) {
      const char *dr = row_at<2>(p.dout, p.dos, token, h), *orow = row_at<2>(p.out, p.os, token, h);
      float part = 0.0f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        dop[ks] = colv ? ld16(dr + ks * 32 + hb * 16) : zero4;
        const uint4 ov = colv ? ld16(orow + ks * 32 + hb * 16) : zero4;
        float df[8], of[8];
        V16<2>::unpack(dop[ks], df);
        V16<2>::unpack(ov, of);
#pragma unroll
        for (int e = 0; e < 8; ++e) part = fmaf(df[e], of[e], part);
      }
      Dc = part + __shfl_xor(part, 32, 64);
      if (colv) Lc = p.lse[token * p.hq + h] * kLog2e;
      // D from the rounded outputs is off by up to 2^-8 |dO . o|, which shows in the
      // gradients of rows of few keys (their outputs are as large as the values; over n
      // keys they average out to n^-1/2 of it).  As the probabilities of a row add up
      // to 1, sum dS is what D lacks: a sequence's first tile, at most four blocks,
      // takes it from there first.
      if (pt.tile == 0 && a < n) {
        float lack = 0.0f;
        const char *k0 = row_at<2>(p.k, p.ks, pt.start, g), *v0 = row_at<2>(p.v, p.vs, pt.start, g);
#pragma unroll 1
        for (int kb = 0; kb * 32 <= a; ++kb) {
          const int64_t row = min(kb * 32 + score_slot(col), n - 1);
          f32x16_t sc = f32x16_t{}, dp = f32x16_t{};
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            sc = mfma_32x32x16(ld16(k0 + row * p.ks[0] * 2 + ks * 32 + hb * 16), qop[ks], sc);
            dp = mfma_32x32x16(ld16(v0 + row * p.vs[0] * 2 + ks * 32 + hb * 16), dop[ks], dp);
          }
          const int tr = one_register(kb * 32 == a ? col - 8 * hb : 32);
#pragma unroll
          for (int rr = 0; rr < 16; ++rr)
            lack += score_row(rr) <= tr ? fast_exp2(fmaf(sc[rr], sl2, -Lc)) * (dp[rr] - Dc) : 0.0f;
        }
        Dc += lack + __shfl_xor(lack, 32, 64);
      }
      if (colv && hb == 0 && share == 0) {   // for the key kernels
        *reinterpret_cast<float2 *>(p.stats + (h * p.stat_stride + token) * 2) = make_float2(Lc, Dc);
      }
    }
  }

  // (the lowest finite value: no score may lie below the running maximum's start)
  float m = lowest(), ls = 0.0f;
  f32x16_t acc[NTL];
#pragma unroll
  for (int i = 0; i < NTL; ++i) acc[i] = f32x16_t{};

  // This thread's chunks of a block: row, byte offset within the row, and the
  // offset from the block's first row while the block lies inside the sequence.
  const uint32_t kst = static_cast<uint32_t>(p.ks[0] * 2), vst = static_cast<uint32_t>(p.vs[0] * 2);
  uint32_t krow[DPW], kchunk[DPW], vchunk[DPW];
#pragma unroll
  for (int i = 0; i < DPW; ++i) {
    const int c = (i * kWaves + wave) * 64 + lane;
    const int row = c / CPR, pc = c - row * CPR;
    krow[i] = row;
    kchunk[i] = (pc ^ block_swizzle<CPR, KSW>(row)) * 16;
    vchunk[i] = (pc ^ block_swizzle<CPR, VSW>(row)) * 16;
  }
  const char *kbase = row_at<2>(p.k, p.ks, pt.start, g), *vbase = row_at<2>(p.v, p.vs, pt.start, g);
  // Every call issues 2 DPW transfers per wave; those of blocks past the last
  // one are switched off.
  auto issue = [&](int kb, auto st_c) {
    const bool on = kb < nblk;
    const char *kp = uniform_ptr(kbase + int64_t(kb) * 32 * kst), *vp = uniform_ptr(vbase + int64_t(kb) * 32 * vst);
    const uint32_t last = static_cast<uint32_t>(max(n - 1 - kb * 32, 0));   // the block's last row inside the sequence
#pragma unroll
    for (int i = 0; i < DPW; ++i) {
      unsigned char *dst = slot(st_c) + (i * kWaves + wave) * 1024;
      const uint32_t row = min(krow[i], last);
      dma16_s(dst, kp, row * kst + kchunk[i], on);
      dma16_s(dst + BLK, vp, row * vst + vchunk[i], on);
    }
  };
  const int krow_s = score_slot(col);
  uint32_t kaddr[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) kaddr[ks] = row_offset<D, KSW>(krow_s, ks, hb);
  uint32_t traddr[NTL][2];
  tr_offsets<D, MODE == 0 ? VSW : KSW>(lane, traddr);
  bool left_out = false;

  issue(blk0, std::integral_constant<int, 0>{});
  issue(blk0 + 1, std::integral_constant<int, 1>{});
  issue(blk0 + 2, std::integral_constant<int, 2>{});
  if constexpr (MODE == 0) {
    f32x16_t scn = f32x16_t{};
    wait_vmcnt<(kSt - 2) * 2 * DPW>();   // the first block has landed
    ring_barrier();
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      scn = mfma_32x32x16(*reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(ring0) + kaddr[ks]),
                          qop[ks], scn);
    auto step = [&](auto stage_c, int kb) {
      constexpr int ST = decltype(stage_c)::value, SN = (ST + 1) % kSt;
      wait_vmcnt<(kSt - 3) * 2 * DPW>();   // block kb + 1 has landed
      ring_barrier();   // every wave is past step kb - 1: the slot of kb - 1 is free
      issue(kb + kSt - 1, std::integral_constant<int, (ST + kSt - 1) % kSt>{});
      if (kb * 32 >= wave_hi) return;
      const bool diagonal = kb * 32 == a;
      const char *vd = reinterpret_cast<const char *>(slot(stage_c)) + BLK;
      const char *kn = reinterpret_cast<const char *>(slot(std::integral_constant<int, SN>{}));   // block kb + 1's keys
      // (past the last block the next scores are not used)
      uint4 kr[4], va[NTL][2];
#pragma unroll
      for (int i = 0; i < 3; ++i) kr[i] = *reinterpret_cast<const uint4 *>(kn + kaddr[i]);
      float sv[16];
#pragma unroll
      for (int rr = 0; rr < 16; ++rr) sv[rr] = scn[rr];
      if (diagonal) {
        const int tr = one_register(col - 8 * hb);
#pragma unroll
        for (int rr = 0; rr < 16; ++rr)
          if (score_row(rr) > tr) sv[rr] = neg_inf();
      }
      float mx = fmaxf(fmaxf(sv[0], sv[1]), sv[2]);
#pragma unroll
      for (int rr = 3; rr < 15; rr += 2) mx = fmaxf(fmaxf(mx, sv[rr]), sv[rr + 1]);
      mx = fmaxf(mx, sv[15]);
      mx = max_halves(mx) * sl2;
      if (__any(mx > m + kLazyRescale)) {
        const float mn = fmaxf(m, mx);
        const float f = fast_exp2(m - mn);
        m = mn;
        ls *= f;
#pragma unroll
        for (int i = 0; i < NTL; ++i) acc[i] *= f;
      }
      f32x16_t sc = f32x16_t{};
      float ev[16];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        if (ks + 3 < KS) kr[(ks + 3) & 3] = *reinterpret_cast<const uint4 *>(kn + kaddr[ks + 3]);
        sc = mfma_32x32x16(kr[ks & 3], qop[ks], sc);
#pragma unroll
        for (int e = 0; e < 16 / KS; ++e) {
          const int i = ks * (16 / KS) + e;
          ev[i] = fast_exp2(fmaf(sv[i], sl2, -m));
          computed_here(ev[i]);
        }
        va[ks >> 1][ks & 1] = tr_operand<RB>(vd, traddr[ks >> 1], ks & 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      scn = sc;
      // P enters the value product rounded to bf16 (off by at most 2^-8 of a
      // probability, at random); its sum is taken in fp32 before that, which L is
      // the logarithm of (over the rounded values L was off by 1e-3).
      uint4 pb[2];
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float e0 = ev[8 * kk + 2 * q], e1 = ev[8 * kk + 2 * q + 1];
          w[q] = cvt_pk_bf16(e0, e1);
          ls += e0 + e1;
        }
        pb[kk] = make_uint4(w[0], w[1], w[2], w[3]);
      }
      if (diagonal) {
#pragma unroll
        for (int i = 0; i < NTL; ++i) left_out |= leave_out_nonfinite(va[i]);
      }
#pragma unroll
      for (int i = 0; i < NTL; ++i)
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) acc[i] = mfma_32x32x16(va[i][kk], pb[kk], acc[i]);
    };
    // Whole rounds of four steps (a step past the last block only keeps the
    // barriers and transfer counts in step).
    for (int kb = blk0; kb < nblk; kb += kSt) {
      step(std::integral_constant<int, 0>{}, kb);
      step(std::integral_constant<int, 1>{}, kb + 1);
      step(std::integral_constant<int, 2>{}, kb + 2);
      step(std::integral_constant<int, 3>{}, kb + 3);
    }
  } else {
    auto step = [&](auto stage_c, int kb) {
      constexpr int ST = decltype(stage_c)::value;
      wait_vmcnt<(kSt - 2) * 2 * DPW>();   // block kb has landed
      ring_barrier();   // block kb is in LDS for every wave; the slot of kb - 1 is free
      issue(kb + kSt - 1, std::integral_constant<int, (ST + kSt - 1) % kSt>{});
      if (kb * 32 >= wave_hi) return;
      const bool diagonal = kb * 32 == a;
      const char *kd = reinterpret_cast<const char *>(slot(stage_c));
      const char *vd = kd + BLK;
      // Row operands are read three products ahead (order pinned).
      f32x16_t sc = f32x16_t{};
      uint4 kr[4];
#pragma unroll
      for (int i = 0; i < 3; ++i) kr[i] = *reinterpret_cast<const uint4 *>(kd + kaddr[i]);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        if (ks + 3 < KS) kr[(ks + 3) & 3] = *reinterpret_cast<const uint4 *>(kd + kaddr[ks + 3]);
        sc = mfma_32x32x16(kr[ks & 3], qop[ks], sc);
        __builtin_amdgcn_sched_barrier(0);
      }
      uint4 vr[4];
#pragma unroll
      for (int i = 0; i < 3; ++i) vr[i] = *reinterpret_cast<const uint4 *>(vd + kaddr[i]);
      float sv[16];
#pragma unroll
      for (int rr = 0; rr < 16; ++rr) sv[rr] = sc[rr];
      const int tr = one_register(diagonal ? col - 8 * hb : 32);
      if (diagonal) {
#pragma unroll
        for (int rr = 0; rr < 16; ++rr)
          if (score_row(rr) > tr) sv[rr] = neg_inf();
      }
      // dP^T = V . dO^T, with P = exp2(S - L) formed between its products, then
      // dS^T = P^T (dP^T - D).
      f32x16_t dp = f32x16_t{};
      float pe[16];
      uint4 kt[KS];   // transposed keys
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        if (ks + 3 < KS) vr[(ks + 3) & 3] = *reinterpret_cast<const uint4 *>(vd + kaddr[ks + 3]);
        dp = mfma_32x32x16(vr[ks & 3], dop[ks], dp);
#pragma unroll
        for (int e = 0; e < 16 / KS; ++e) {
          const int i = ks * (16 / KS) + e;
          pe[i] = fast_exp2(fmaf(sv[i], sl2, -Lc));
          computed_here(pe[i]);
        }
        kt[ks] = tr_operand<RB>(kd, traddr[ks >> 1], ks & 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (diagonal) {   // (a masked row's dP may be anything)
#pragma unroll
        for (int rr = 0; rr < 16; ++rr)
          if (score_row(rr) > tr) dp[rr] = Dc;
      }
      uint4 sb[2];
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int r0 = 8 * kk + 2 * q;
          w[q] = cvt_pk_bf16(pe[r0] * (dp[r0] - Dc), pe[r0 + 1] * (dp[r0 + 1] - Dc));
        }
        sb[kk] = make_uint4(w[0], w[1], w[2], w[3]);
      }
      if (diagonal) {   // (one by one: the check of all at once spills fifty registers here)
#pragma unroll
        for (int j = 0; j < 2 * NTL; ++j) left_out |= leave_out_nonfinite(kt[j]);
      }
#pragma unroll
      for (int j = 0; j < 2 * NTL; ++j) acc[j >> 1] = mfma_32x32x16(kt[j], sb[j & 1], acc[j >> 1]);
    };
    for (int kb = blk0; kb < nblk; kb += kSt) {
      step(std::integral_constant<int, 0>{}, kb);
      step(std::integral_constant<int, 1>{}, kb + 1);
      step(std::integral_constant<int, 2>{}, kb + 2);
      step(std::integral_constant<int, 3>{}, kb + 3);
    }
  }
  if (__any(left_out)) {
    const char *base = MODE == 0 ? vbase : kbase;
    const uint32_t st = MODE == 0 ? vst : kst;
    add_nonfinite<D, MODE != 0>(acc, [&](int i, int e) { return row4(base + int64_t(min(a + i, n - 1)) * st, e); },
                                [&](int i) { return colv && i <= col; }, hb);
  }

  // Lane holds dims 32 i + 8 j + 4 hb .. + 4 of its column.
  const float lt = ls + __shfl_xor(ls, 32, 64);
  if (!colv) return;
  if (parts > 1) {   // this part's record: the sums, and in the forward the maximum and sum of the weights
    float *rec = p.part_q + ((int64_t(share) * p.total + token) * p.hq + h) * (D + 4);
    if (MODE == 0 && hb == 0) {
      rec[0] = m;
      rec[1] = lt;
    }
#pragma unroll
    for (int i = 0; i < NTL; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<float4 *>(rec + 4 + 32 * i + 8 * j + 4 * hb) =
            make_float4(acc[i][4 * j], acc[i][4 * j + 1], acc[i][4 * j + 2], acc[i][4 * j + 3]);
    return;
  }
  char *orow = const_cast<char *>(MODE == 0 ? row_at<2>(p.out, p.os, token, h) : row_at<2>(p.dq, p.dqs, token, h));
  float scale;
  if constexpr (MODE == 0) {
    scale = 1.0f / lt;
    if (hb == 0) p.lse[token * p.hq + h] = (m + __log2f(lt)) * kLn2;
  } else {
    scale = sl2 / kLog2e;   // 1 / sqrt(d)
  }
#pragma unroll
  for (int i = 0; i < NTL; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t lo = cvt_pk_bf16(acc[i][4 * j] * scale, acc[i][4 * j + 1] * scale);
      const uint32_t hi = cvt_pk_bf16(acc[i][4 * j + 2] * scale, acc[i][4 * j + 3] * scale);
      *reinterpret_cast<uint2 *>(orow + (32 * i + 8 * j + 4 * hb) * 2) = make_uint2(lo, hi);
    }
}

// dV (PART 1: S, P) and dK (PART 2: S, dP, dS) of 128 keys of one kv head, 32
// per wave (its K and V rows are operands in registers); the queries of the
// group's heads, one head after another, stream through LDS in blocks of 32
// rows with their statistics (a ring of three blocks, two ahead).  In two parts,
// each holds half the accumulators and runs two waves per SIMD.
//   S[row][key] = Q . K^T,  dP[row][key] = dO . V^T   (rows pi-permuted)
//   dV^T[dim][key] += dO^T P,  dK^T[dim][key] += Q^T dS
// 6 sequences up to 4096, 32/8 heads, d 128: dV 580 us, dK 757 us (medians of a trace).
// P and dS enter the products rounded to bf16, the operands' type: off by at most
// 2^-8 of each, at random, where the gradients are rounded by as much in the end.
template <int D, int PART>
__global__ __launch_bounds__(kThreads, 2) void causal_key_kernel(CausalParams p) {
  static_assert(PART == 1 || PART == 2, "dV part or dK part");
  constexpr int kSt = 3;
  constexpr int KS = D / 16, NTL = D / 32, RB = D * 2, CPR = D / 8, BLK = 32 * RB;
  constexpr int DPW = BLK / 16 / kThreads;
  // One ring slot: query rows, dO rows, then per wave its own copy of the
  // block's statistics (32 L, then 32 D).
  constexpr int SLOT = 2 * BLK + kWaves * 256;
  static_assert(DPW >= 1, "block split");
  __shared__ __align__(16) unsigned char ring0[SLOT], ring1[SLOT], ring2[SLOT];
  auto slot = [&](auto st_c) -> unsigned char * {
    constexpr int S = decltype(st_c)::value;
    if constexpr (S == 0) return ring0;
    else if constexpr (S == 1) return ring1;
    else return ring2;
  };
  int g, rank;
  head_of_block(p.hkv, g, rank);
  const PackedTile pt = tile_of_rank<true>(p, rank, 0, kTileShift);
  const int n = pt.n;
  if (pt.tile < 0 || pt.tile * kTile >= n) return;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, hb = lane >> 5;
  const int s0 = pt.tile * kTile + wave * 32;        // this wave's first key
  const int js = s0 + col;                           // this lane's key (column)
  const bool kv_ok = js < n;
  const uint4 zero4 = make_uint4(0, 0, 0, 0);
  const float sl2 = p.scale_log2;
  const int G = p.hq / p.hkv;

  uint4 kop[KS], vop[PART == 2 ? KS : 1];
  {
    const int64_t token = pt.start + (kv_ok ? js : 0);
    const char *kr = row_at<2>(p.k, p.ks, token, g), *vr = row_at<2>(p.v, p.vs, token, g);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      kop[ks] = kv_ok ? ld16(kr + ks * 32 + hb * 16) : zero4;
      if constexpr (PART == 2) vop[ks] = kv_ok ? ld16(vr + ks * 32 + hb * 16) : zero4;
    }
  }

  // Row blocks that see the tile, of every head in turn; this workgroup's part of them.
  const int qb0 = pt.tile * (kTile / 32), qb1 = (n + 31) >> 5, per_head = qb1 - qb0;
  const int part = blockIdx.y, lo = G * per_head * part / p.parts, nblk = G * per_head * (part + 1) / p.parts - lo;
  const uint32_t qst = static_cast<uint32_t>(p.qs[0] * 2), dst_ = static_cast<uint32_t>(p.dos[0] * 2);
  uint32_t qrow[DPW], qchunk[DPW];
#pragma unroll
  for (int i = 0; i < DPW; ++i) {
    const int c = (i * kWaves + wave) * 64 + lane;
    const int row = c / CPR, pc = c - row * CPR;
    qrow[i] = row;
    qchunk[i] = (pc ^ dual_swizzle<CPR>(row)) * 16;
  }
  // Statistics, one 4-byte transfer per wave into its own area: lanes 0..31 the
  // rows' L, lanes 32..63 their D (rows past the sequence: the next one's, or
  // the workspace's padding, not used).
  const uint32_t soff = uint32_t(col) * 8 + uint32_t(hb) * 4;
  int ih = g * G + lo / per_head, iq = qb0 + lo % per_head, left = nblk;   // next block to issue: head, row block
  // Every call issues 2 DPW + 1 transfers per wave; those past the last block
  // are switched off.
  auto issue = [&](auto st_c) {
    const bool on = left-- > 0;
    const int hh = min(ih, g * G + G - 1);
    unsigned char *dst = slot(st_c);
    const char *qp = uniform_ptr(row_at<2>(p.q, p.qs, pt.start + iq * 32, hh));
    const char *dp = uniform_ptr(row_at<2>(p.dout, p.dos, pt.start + iq * 32, hh));
    const char *sp = uniform_ptr(reinterpret_cast<const char *>(p.stats + (hh * p.stat_stride + pt.start + iq * 32) * 2));
    const uint32_t last = static_cast<uint32_t>(n - 1 - iq * 32);   // the block's last row inside the sequence
#pragma unroll
    for (int i = 0; i < DPW; ++i) {
      unsigned char *cdst = dst + (i * kWaves + wave) * 1024;
      const uint32_t row = min(qrow[i], last);
      dma16_s(cdst, qp, row * qst + qchunk[i], on);
      dma16_s(cdst + BLK, dp, row * dst_ + qchunk[i], on);
    }
    dma_so<kCachePolicyDefault, 4>(dst + 2 * BLK + wave * 256, sp, soff, on);
    if (++iq == qb1) {
      iq = qb0;
      ++ih;
    }
  };
  const int qrow_s = score_slot(col);
  uint32_t raddr[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) raddr[ks] = row_offset<D, 2>(qrow_s, ks, hb);
  uint32_t traddr[NTL][2];
  tr_offsets<D, 2>(lane, traddr);

  f32x16_t acc[NTL];
#pragma unroll
  for (int i = 0; i < NTL; ++i) acc[i] = f32x16_t{};
  bool left_out = false;
  int cq = iq;   // row block of the next step

  auto step = [&](auto stage_c, int kb) {
    constexpr int ST = decltype(stage_c)::value;
    wait_vmcnt<(kSt - 2) * (2 * DPW + 1)>();   // block kb has landed
    ring_barrier();   // block kb is in LDS for every wave; the slot of kb - 1 is free
    issue(std::integral_constant<int, (ST + kSt - 1) % kSt>{});
    const int rb = cq * 32;                    // first row of the block
    if (++cq == qb1) cq = qb0;
    if (kb >= nblk || rb < s0) return;         // past the last block, or every row precedes this wave's keys
    const char *qd = reinterpret_cast<const char *>(slot(stage_c));
    const char *dd = qd + BLK;
    const bool masked = rb == s0 || rb + 32 > n;   // the diagonal, or rows past the sequence
    // Register 8 kk + q of this lane: row rb + 16 kk + 8 hb + q.
    const float *sl = reinterpret_cast<const float *>(qd + 2 * BLK + wave * 256) + 8 * hb;
    float Lr[16], Dr[PART == 2 ? 16 : 1];
    auto statistics = [&](const float *e8, float *x) {
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const float4 f = *reinterpret_cast<const float4 *>(e8 + 16 * (c >> 1) + 4 * (c & 1));
        x[4 * c + 0] = f.x; x[4 * c + 1] = f.y; x[4 * c + 2] = f.z; x[4 * c + 3] = f.w;
      }
    };
    f32x16_t sc = f32x16_t{};
    uint4 qr[4];
#pragma unroll
    for (int i = 0; i < 3; ++i) qr[i] = *reinterpret_cast<const uint4 *>(qd + raddr[i]);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (ks + 3 < KS) qr[(ks + 3) & 3] = *reinterpret_cast<const uint4 *>(qd + raddr[ks + 3]);
      sc = mfma_32x32x16(qr[ks & 3], kop[ks], sc);
      if (ks == 0) statistics(sl, Lr);
      __builtin_amdgcn_sched_barrier(0);
    }
    float pe[16];
    const char *xd = PART == 1 ? dd : qd;   // rows of the last product: dO (dV), Q (dK)
    uint4 xt[4];                            // them transposed, read three products ahead
    f32x16_t dp = f32x16_t{};
    if constexpr (PART == 2) {
      uint4 dr[4];
#pragma unroll
      for (int i = 0; i < 3; ++i) dr[i] = *reinterpret_cast<const uint4 *>(dd + raddr[i]);
      // dP's products with P's exponentials between them (order pinned).
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        if (ks + 3 < KS) dr[(ks + 3) & 3] = *reinterpret_cast<const uint4 *>(dd + raddr[ks + 3]);
        dp = mfma_32x32x16(dr[ks & 3], vop[ks], dp);
#pragma unroll
        for (int e = 0; e < 16 / KS; ++e) {
          const int i = ks * (16 / KS) + e;
          pe[i] = fast_exp2(fmaf(sc[i], sl2, -Lr[i]));
          computed_here(pe[i]);
        }
        if (ks == KS - 4) statistics(sl + 32, Dr);
        if (ks >= KS - 3) xt[ks - (KS - 3)] = tr_operand<RB>(xd, traddr[(ks - (KS - 3)) >> 1], (ks - (KS - 3)) & 1);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 3; ++j) xt[j] = tr_operand<RB>(xd, traddr[j >> 1], j & 1);
#pragma unroll
      for (int i = 0; i < 16; ++i) pe[i] = fast_exp2(fmaf(sc[i], sl2, -Lr[i]));
    }
    if (masked) {
      // row 16 kk + 8 hb + q is seen from key col on, and up to the sequence's end
      const int from = one_register(rb == s0 ? col - 8 * hb : -8), to = one_register(n - rb - 8 * hb);
#pragma unroll
      for (int rr = 0; rr < 16; ++rr) {
        const bool vis = score_row(rr) >= from && score_row(rr) < to;
        pe[rr] = vis ? pe[rr] : 0.0f;
        if constexpr (PART == 2) dp[rr] = vis ? dp[rr] - Dr[rr] : 0.0f;
      }
    } else if constexpr (PART == 2) {
#pragma unroll
      for (int rr = 0; rr < 16; ++rr) dp[rr] -= Dr[rr];
    }
    uint4 wb[2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      uint32_t w[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int i = 8 * kk + 2 * q;
        if constexpr (PART == 1) w[q] = cvt_pk_bf16(pe[i], pe[i + 1]);
        else w[q] = cvt_pk_bf16(pe[i] * dp[i], pe[i + 1] * dp[i + 1]);
      }
      wb[kk] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    auto product = [&](auto masked_c) {
#pragma unroll
      for (int j = 0; j < 2 * NTL; ++j) {
        if (j + 3 < 2 * NTL) xt[(j + 3) & 3] = tr_operand<RB>(xd, traddr[(j + 3) >> 1], (j + 3) & 1);
        if constexpr (decltype(masked_c)::value) left_out |= leave_out_nonfinite(xt[j & 3]);
        acc[j >> 1] = mfma_32x32x16(xt[j & 3], wb[j & 1], acc[j >> 1]);
      }
    };
    if (masked) product(std::true_type{});
    else product(std::false_type{});
  };

  issue(std::integral_constant<int, 0>{});
  issue(std::integral_constant<int, 1>{});
  // Whole rounds of three steps (a step past the last block only keeps the
  // barriers and transfer counts in step).
  for (int kb = 0; kb < nblk; kb += kSt) {
    step(std::integral_constant<int, 0>{}, kb);
    step(std::integral_constant<int, 1>{}, kb + 1);
    step(std::integral_constant<int, 2>{}, kb + 2);
  }
  if (__any(left_out)) {   // the masked blocks of every head again
    const void *base = PART == 1 ? p.dout : p.q;
    for (int i = lo; i < lo + nblk; ++i) {
      const int hh = g * G + i / per_head, rb = (qb0 + i % per_head) * 32;
      if (rb < s0 || (rb != s0 && rb + 32 <= n)) continue;
      add_nonfinite<D, PART == 2>(
            acc,
          [&](int r, int e) {
            return row4(row_at<2>(base, PART == 1 ? p.dos : p.qs, pt.start + min(rb + r, n - 1), hh), e);
          },
          [&](int r) { return kv_ok && rb + r >= js && rb + r < n; }, hb);
    }
  }
  if (!kv_ok) return;
  const float scale = PART == 1 ? 1.0f : sl2 / kLog2e;
  if (p.parts > 1) {   // this part's share, in fp32
    float *rec = (PART == 1 ? p.part_v : p.part_k) + ((int64_t(part) * p.total + pt.start + js) * p.hkv + g) * D;
#pragma unroll
    for (int i = 0; i < NTL; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<float4 *>(rec + 32 * i + 8 * j + 4 * hb) =
            make_float4(acc[i][4 * j] * scale, acc[i][4 * j + 1] * scale, acc[i][4 * j + 2] * scale,
                        acc[i][4 * j + 3] * scale);
    return;
  }
  char *orow = const_cast<char *>(PART == 1 ? row_at<2>(p.dv, p.dvs, pt.start + js, g)
                                            : row_at<2>(p.dk, p.dks, pt.start + js, g));
#pragma unroll
  for (int i = 0; i < NTL; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t lo = cvt_pk_bf16(acc[i][4 * j] * scale, acc[i][4 * j + 1] * scale);
      const uint32_t hi = cvt_pk_bf16(acc[i][4 * j + 2] * scale, acc[i][4 * j + 3] * scale);
      *reinterpret_cast<uint2 *>(orow + (32 * i + 8 * j + 4 * hb) * 2) = make_uint2(lo, hi);
    }
}

// The parts of a query row put together, in their order, one wave per row and head:
// outputs (MODE 0: with the weights 2^(m - M) of their maxima, and the row's log
// sum exp) or dQ.
template <int D, int MODE>
__global__ __launch_bounds__(kThreads) void causal_query_parts_kernel(CausalParams p, int ntiles) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63;
  const int wid = blockIdx.x * kWaves + (threadIdx.x >> 6);
  const int h = wid % p.hq, row = wid / p.hq;   // (tile index, row of the tile)
  const PackedTile pt = packed_tile(p.cu, p.seqs, p.total, row >> kTileShift, kTileShift);
  const int t = pt.tile * kTile + (row & (kTile - 1));
  if (row >= ntiles * kTile || pt.tile < 0 || t >= pt.n) return;
  const int parts = tile_parts(p.query_parts, (min(pt.n, pt.tile * kTile + kTile) + 31) >> 5);
  if (parts == 1) return;
  const int64_t token = pt.start + t, step = int64_t(p.total) * p.hq * (D + 4);
  const float *rec = p.part_q + (token * p.hq + h) * (D + 4);
  float M = lowest(), L = 0.0f, A[E];
#pragma unroll
  for (int e = 0; e < E; ++e) A[e] = 0.0f;
  float m[kMaxQueryParts], l[kMaxQueryParts], a[kMaxQueryParts][E];
#pragma unroll
  for (int i = 0; i < kMaxQueryParts; ++i) {   // (every load in flight; past the parts, the last one again)
    const float *r = rec + min(i, parts - 1) * step;
    m[i] = r[0];
    l[i] = r[1];
#pragma unroll
    for (int e = 0; e < E; ++e) a[i][e] = r[4 + lane * E + e];
  }
  if constexpr (MODE == 0) {
#pragma unroll
    for (int i = 0; i < kMaxQueryParts; ++i) M = fmaxf(M, m[i]);
  }
#pragma unroll
  for (int i = 0; i < kMaxQueryParts; ++i) {
    if (i < parts) {
      const float w = MODE == 0 ? fast_exp2(m[i] - M) : 1.0f;
      L = fmaf(w, l[i], L);
#pragma unroll
      for (int e = 0; e < E; ++e) A[e] = fmaf(w, a[i][e], A[e]);
    }
  }
  const float scale = MODE == 0 ? 1.0f / L : p.scale_log2 / kLog2e;
#pragma unroll
  for (int e = 0; e < E; ++e) A[e] *= scale;
  const char *o = MODE == 0 ? row_at<2>(p.out, p.os, token, h) : row_at<2>(p.dq, p.dqs, token, h);
  store_e<2, E>(const_cast<char *>(o) + lane * E * 2, A);
  if (MODE == 0 && lane == 0) p.lse[token * p.hq + h] = (M + __log2f(L)) * kLn2;
}

// The parts of dK and dV put together, in their order: one thread per 4 elements of
// a row of a kv head, for the tokens inside the sequences.
template <int ES, int D>
__global__ __launch_bounds__(kThreads) void causal_parts_kernel(CausalParams p) {
  const int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  const int first = clamp_token(p.cu[0], p.total), end = clamp_token(p.cu[p.seqs], p.total);
  const int64_t row = i / (D / 4);
  const int e = static_cast<int>(i - row * (D / 4)) * 4;
  const int64_t token = row / p.hkv;
  const int g = static_cast<int>(row - token * p.hkv);
  if (token < first || token >= end) return;
  const int64_t step = int64_t(p.total) * p.hkv * D;
  float4 k = make_float4(0, 0, 0, 0), v = k;
  for (int part = 0; part < p.parts; ++part) {
    const float4 a = *reinterpret_cast<const float4 *>(p.part_k + part * step + row * D + e);
    const float4 b = *reinterpret_cast<const float4 *>(p.part_v + part * step + row * D + e);
    k.x += a.x; k.y += a.y; k.z += a.z; k.w += a.w;
    v.x += b.x; v.y += b.y; v.z += b.z; v.w += b.w;
  }
  char *dk = const_cast<char *>(row_at<ES>(p.dk, p.dks, token, g)) + e * ES;
  char *dv = const_cast<char *>(row_at<ES>(p.dv, p.dvs, token, g)) + e * ES;
  if constexpr (ES == 2) {
    *reinterpret_cast<uint2 *>(dk) = make_uint2(cvt_pk_bf16(k.x, k.y), cvt_pk_bf16(k.z, k.w));
    *reinterpret_cast<uint2 *>(dv) = make_uint2(cvt_pk_bf16(v.x, v.y), cvt_pk_bf16(v.z, v.w));
  } else {
    *reinterpret_cast<float4 *>(dk) = k;
    *reinterpret_cast<float4 *>(dv) = v;
  }
}

// ---------------------------------------------------------------------------
// fp32, on v_mfma_f32_32x32x2_f32 (operand forms: F32).  One workgroup = 32
// columns of one head -- queries in the forward and dq, keys in the key kernel
// -- whose four waves share the column operands and take every fourth 32-row
// block of the other side straight from global memory; their results meet in
// LDS.  Bound by the fp32 matrix rate and by the longest tile's chain of blocks (4
// sequences up to 640, 8/4 heads, d 64: forward 30 us, dq 51, dK and dV 74).
// ---------------------------------------------------------------------------
template <int D, int MODE>
__global__ __launch_bounds__(kThreads) void causal_query_f32_kernel(CausalParams p, int ntiles) {
  using F = F32<D>;
  constexpr int NT = F::NT;
  __shared__ __align__(16) float s_acc[F::kArea];
  __shared__ float s_m[kWaves * 32], s_l[kWaves * 32];
  int h, rank;
  head_of_block(p.hq, h, rank);
  const PackedTile pt = tile_of_rank<false>(p, rank, ntiles, kTileShift32);
  const int n = pt.n, a = pt.tile * kTile32;
  if (pt.tile < 0 || a >= n) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 31, hb = lane >> 5;
  const int g = h / (p.hq / p.hkv);
  const int t = a + col;
  const bool colv = t < n;
  const int64_t token = pt.start + (colv ? t : 0);
  const int nblk = pt.tile + 1;   // the last one holds the diagonal

  auto col_row = [&](const void *base, const int64_t (&st)[2], int c) -> const float * {
    return a + c < n ? reinterpret_cast<const float *>(row_at<4>(base, st, pt.start + a + c, h)) : nullptr;
  };
  F::stage(s_acc, [&](int c) { return col_row(p.q, p.qs, c); }, false);
  if constexpr (MODE == 1) F::stage(s_acc + 32 * F::kCol, [&](int c) { return col_row(p.dout, p.dos, c); }, false);
  __syncthreads();
  const float *qs = F::staged(s_acc, lane), *dos = F::staged(s_acc + (MODE == 1 ? 32 * F::kCol : 0), lane);
  typename F::f4_t kr[F::NJ], vr[MODE == 1 ? F::NJ : 1];
  float Lc = 0.0f, Dc = 0.0f;
  if constexpr (MODE == 1) {
    if (colv) {
      F::load_row(kr, col_row(p.out, p.os, col), hb);
      Lc = p.lse[token * p.hq + h] * kLog2e;
#pragma unroll
      for (int j = 0; j < F::NJ; ++j) {
        const typename F::f4_t d4 = *reinterpret_cast<const typename F::f4_t *>(dos + 8 * j);
        float part = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) part = fmaf(d4[i], kr[j][i], part);
        Dc += part;
      }
    }
    Dc += __shfl_xor(Dc, 32, 64);
    if (tid < 32 && colv)
      *reinterpret_cast<float2 *>(p.stats + (h * p.stat_stride + token) * 2) = make_float2(Lc, Dc);
  }
  float m = lowest(), ls = 0.0f;
  f32x16_t acc[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) acc[i] = f32x16_t{};
  auto key_at = [&](int s) { return reinterpret_cast<const float *>(row_at<4>(p.k, p.ks, pt.start + min(s, n - 1), g)); };
  auto value_at = [&](int s) { return reinterpret_cast<const float *>(row_at<4>(p.v, p.vs, pt.start + min(s, n - 1), g)); };
  F::load_row(kr, key_at(wave * 32 + col), hb);
  bool left_out = false;
  auto block = [&](int kb, auto last_c) {
    constexpr bool LAST = decltype(last_c)::value;   // the diagonal's block
    if constexpr (MODE == 1) F::load_row(vr, value_at(kb * 32 + col), hb);   // lands while the scores run
    typename F::Cols xc;
    auto x_row = [&](int i) { return MODE == 0 ? value_at(kb * 32 + i) : key_at(kb * 32 + i); };
    xc.load(x_row, 0, lane);
    const f32x16_t sc = F::dots(kr, qs);
    f32x16_t dp = f32x16_t{};
    if constexpr (MODE == 1) dp = F::dots(vr, dos);
    if (!LAST) F::load_row(kr, key_at((kb + kWaves) * 32 + col), hb);
    float x[16];
    if constexpr (MODE == 0) {
      float mx = neg_inf();
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[r] = sc[r] * p.scale_log2;
        if (LAST && F::row(r, hb) > col) x[r] = neg_inf();
        mx = fmaxf(mx, x[r]);
      }
      const float mn = fmaxf(m, max_halves(mx));
      const float f = fast_exp2(m - mn);
      m = mn;
      ls *= f;
#pragma unroll
      for (int i = 0; i < NT; ++i) acc[i] *= f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[r] = fast_exp2(x[r] - mn);
        ls += x[r];
      }
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        x[r] = LAST && F::row(r, hb) > col ? 0.0f : fast_exp2(sc[r] * p.scale_log2 - Lc) * (dp[r] - Dc);
    }
    left_out |= F::template add_rows<LAST>(acc, xc, x_row, x, lane);
  };
#pragma unroll 1
  for (int kb = wave; kb < nblk - 1; kb += kWaves) block(kb, std::false_type{});
  if (((nblk - 1) & (kWaves - 1)) == wave) block(nblk - 1, std::true_type{});
  if (__any(left_out))
    F::add_nonfinite(acc, [&](int i) { return MODE == 0 ? value_at(a + i) : key_at(a + i); },
                     [&](int i) { return colv && i <= col; }, lane);
  if constexpr (MODE == 0) {
    ls += __shfl_xor(ls, 32, 64);
    if (hb == 0) {
      s_m[wave * 32 + col] = m;
      s_l[wave * 32 + col] = ls;
    }
    __syncthreads();   // (and the staged rows' last use)
    float M = s_m[col], L = 0.0f;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, s_m[w * 32 + col]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) L += s_l[w * 32 + col] * fast_exp2(s_m[w * 32 + col] - M);
    const float f = fast_exp2(m - M) / L;
#pragma unroll
    for (int i = 0; i < NT; ++i) acc[i] *= f;
    if (tid < 32 && colv) p.lse[token * p.hq + h] = (M + __log2f(L)) * kLn2;
  } else {
    const float scale = p.scale_log2 / kLog2e;   // 1 / sqrt(d)
#pragma unroll
    for (int i = 0; i < NT; ++i) acc[i] *= scale;
    __syncthreads();   // the staged rows' last use
  }
  F::put(s_acc, wave, lane, acc);
  __syncthreads();
  for (int i = tid; i < 32 * D / 4; i += kThreads) {
    const int c = i / (D / 4), e = i % (D / 4);
    if (a + c >= n) continue;
    const char *o = MODE == 0 ? row_at<4>(p.out, p.os, pt.start + a + c, h) : row_at<4>(p.dq, p.dqs, pt.start + a + c, h);
    *reinterpret_cast<typename F::f4_t *>(const_cast<char *>(o) + 16 * e) = F::sum(s_acc, c, e);
  }
}

// dK and dV of 32 keys.  PART 0 computes both; at d = 128, where both sets of
// operands exceed the register file, PART 1 is dV alone and PART 2 dK.
template <int D, int PART>
__global__ __launch_bounds__(kThreads) void causal_key_f32_kernel(CausalParams p) {
  using F = F32<D>;
  constexpr int NT = F::NT;
  constexpr bool DV = PART != 2, DK = PART != 1;
  __shared__ __align__(16) float s_acc[F::kArea];
  int g, rank;
  head_of_block(p.hkv, g, rank);
  const PackedTile pt = tile_of_rank<true>(p, rank, 0, kTileShift32);
  const int n = pt.n, s0 = pt.tile * kTile32;
  if (pt.tile < 0 || s0 >= n) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 31, hb = lane >> 5;
  const int G = p.hq / p.hkv;
  const int js = s0 + col;   // this lane's key
  const bool kv_ok = js < n;
  // Row blocks that see the tile, of every head in turn (the first of a head holds the
  // diagonal); this workgroup's part of them.
  const int qb0 = pt.tile, per_head = ((n + 31) >> 5) - qb0, part = blockIdx.y;
  const int blk0 = G * per_head * part / p.parts, nblk = G * per_head * (part + 1) / p.parts;

  auto key_row = [&](const void *base, const int64_t (&st)[2], int c) -> const float * {
    return s0 + c < n ? reinterpret_cast<const float *>(row_at<4>(base, st, pt.start + s0 + c, g)) : nullptr;
  };
  F::stage(s_acc, [&](int c) { return key_row(p.k, p.ks, c); }, false);
  if constexpr (DK) F::stage(s_acc + 32 * F::kCol, [&](int c) { return key_row(p.v, p.vs, c); }, false);
  __syncthreads();
  const float *kst = F::staged(s_acc, lane), *vst = F::staged(s_acc + (DK ? 32 * F::kCol : 0), lane);
  typename F::f4_t qr[F::NJ], dor[DK ? F::NJ : 1];
  f32x16_t dk[DK ? NT : 1], dv[DV ? NT : 1];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    if constexpr (DK) dk[i] = f32x16_t{};
    if constexpr (DV) dv[i] = f32x16_t{};
  }
  // block i: head, first row
  auto at = [&](int i, int &hh, int &rb) {
    const int q = i / per_head;
    hh = g * G + q;
    rb = (qb0 + i - q * per_head) * 32;
  };
  auto q_at = [&](int hh, int r) { return reinterpret_cast<const float *>(row_at<4>(p.q, p.qs, pt.start + min(r, n - 1), hh)); };
  auto do_at = [&](int hh, int r) { return reinterpret_cast<const float *>(row_at<4>(p.dout, p.dos, pt.start + min(r, n - 1), hh)); };
  int hh, rb;
  at(min(blk0 + wave, G * per_head - 1), hh, rb);
  F::load_row(qr, q_at(hh, rb + col), hb);
  bool out_v = false, out_k = false;
  auto block = [&](int i, auto masked_c, bool masked) {
    constexpr bool MASKED = decltype(masked_c)::value;
    if constexpr (DK) F::load_row(dor, do_at(hh, rb + col), hb);   // lands while the scores run
    typename F::Cols qc, oc;
    auto q_row = [&](int r) { return q_at(hh, rb + r); };
    auto do_row = [&](int r) { return do_at(hh, rb + r); };
    if constexpr (DV) oc.load(do_row, 0, lane);
    if constexpr (DK) qc.load(q_row, 0, lane);
    float Lr[16], Dr[16];
    const float *st = p.stats + (hh * p.stat_stride + pt.start + rb) * 2;   // (padded by 32 rows)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      float x[8];
      load4(st + (8 * c + 4 * hb) * 2, x);
      load4(st + (8 * c + 4 * hb) * 2 + 4, x + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        Lr[4 * c + e] = x[2 * e];
        Dr[4 * c + e] = x[2 * e + 1];
      }
    }
    const f32x16_t sc = F::dots(qr, kst);
    f32x16_t dp = f32x16_t{};
    if constexpr (DK) dp = F::dots(dor, vst);
    int hn, rn;
    at(min(i + kWaves, G * per_head - 1), hn, rn);
    F::load_row(qr, q_at(hn, rn + col), hb);
    float pv[16], ds[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = rb + F::row(r, hb);
      const bool vis = !MASKED || (row >= js && row < n);
      pv[r] = vis ? fast_exp2(sc[r] * p.scale_log2 - Lr[r]) : 0.0f;
      if constexpr (DK) ds[r] = vis ? pv[r] * (dp[r] - Dr[r]) : 0.0f;
    }
    if constexpr (DV) out_v |= F::template add_rows<MASKED>(dv, oc, do_row, pv, lane, masked);
    if constexpr (DK) out_k |= F::template add_rows<MASKED>(dk, qc, q_row, ds, lane, masked);
  };
#pragma unroll 1
  for (int i = blk0 + wave; i < nblk; i += kWaves) {
    at(i, hh, rb);
    const bool masked = rb == s0 || rb + 32 > n;
    // (PART 2: the masked sums in a body of their own -- beside the others they spilled two
    // hundred registers, 644 -> 270 us for 3 sequences up to 1000 tokens, 8/2 heads)
    if (PART != 2 || masked) block(i, std::true_type{}, masked);
    else block(i, std::false_type{}, false);
  }
  if (__any(out_v || out_k)) {
    for (int i = blk0 + wave; i < nblk; i += kWaves) {
      at(i, hh, rb);
      if (!(rb == s0 || rb + 32 > n)) continue;
      auto sees = [&](int r) { return kv_ok && rb + r >= js && rb + r < n; };
      if constexpr (DV) F::add_nonfinite(dv, [&](int r) { return do_at(hh, rb + r); }, sees, lane);
      if constexpr (DK) F::add_nonfinite(dk, [&](int r) { return q_at(hh, rb + r); }, sees, lane);
    }
  }
  auto emit = [&](void *out, const int64_t (&st)[2], float *share) {   // the merged rows of the tile's keys
    __syncthreads();
    for (int i = tid; i < 32 * D / 4; i += kThreads) {
      const int c = i / (D / 4), e = i % (D / 4);
      if (s0 + c >= n) continue;
      const int64_t token = pt.start + s0 + c;
      char *o = p.parts > 1 ? reinterpret_cast<char *>(share + ((int64_t(part) * p.total + token) * p.hkv + g) * D)
                            : const_cast<char *>(row_at<4>(out, st, token, g));
      *reinterpret_cast<typename F::f4_t *>(o + 16 * e) = F::sum(s_acc, c, e);
    }
  };
  __syncthreads();   // the staged rows' last use
  if constexpr (DV) {
    F::put(s_acc, wave, lane, dv);
    emit(p.dv, p.dvs, p.part_v);
    if constexpr (DK) __syncthreads();   // the merge area is reused
  }
  if constexpr (DK) {
    const float scale = p.scale_log2 / kLog2e;
#pragma unroll
    for (int i = 0; i < NT; ++i) dk[i] *= scale;
    F::put(s_acc, wave, lane, dk);
    emit(p.dk, p.dks, p.part_k);
  }
}

// Whether tiles go out in descending length: where there are more of them than run
// at once, two workgroups per compute unit (finding a rank's tile takes about a
// microsecond).  Query tiles only where an XCD's share of the keys and values fits
// its 4 MB L2: sequences then run side by side rather than one after another.  us,
// in the order of the sequences -> by length: backward, 6 sequences up to 4096
// tokens, 32/8 heads, dV 718 -> 616, dK 911 -> 766; forward of 16 x 500 tokens,
// 8 heads, d = 64, 20.7 -> 16.3, but of 4 x 4096, 32 heads, 582 -> 611.
bool sort_tiles(const CausalParams &p, int64_t workgroups) {
  return p.seqs <= kSortSeqs && workgroups > kPartPlaces / 2;
}
bool sort_queries(const CausalParams &p, int64_t workgroups, int row_bytes) {
  const int64_t heads = (p.hkv + 7) / 8;
  return sort_tiles(p, workgroups) && heads * p.total * 2 * row_bytes <= (4 << 20);
}

template <int D, int MODE>
void launch_query_parts(const CausalParams &p, int ntiles, hipStream_t s) {
  if (p.query_parts > 1)
    hipLaunchKernelGGL((causal_query_parts_kernel<D, MODE>),
                       dim3(unsigned((int64_t(ntiles) * kTile * p.hq + kWaves - 1) / kWaves)), dim3(kThreads), 0, s, p, ntiles);
}

template <int D>
hipError_t causal_forward(int elem_bytes, CausalParams p, hipStream_t s) {
  const int shift = elem_bytes == 2 ? kTileShift : kTileShift32;
  const int ntiles = (p.total >> shift) + p.seqs;
  const int64_t blocks = int64_t(ntiles) * p.hq;
  if (blocks > 0x7fffffff) return hipErrorInvalidConfiguration;
  p.sorted = sort_queries(p, blocks, D * elem_bytes);
  const dim3 grid(unsigned(blocks), elem_bytes == 2 ? p.query_parts : 1), threads(kThreads);
  if (elem_bytes == 2) {
    hipLaunchKernelGGL((causal_query_kernel<D, 0>), grid, threads, 0, s, p, ntiles);
    launch_query_parts<D, 0>(p, ntiles, s);
  } else {
    hipLaunchKernelGGL((causal_query_f32_kernel<D, 0>), grid, threads, 0, s, p, ntiles);
  }
  return hipGetLastError();
}

template <int D>
hipError_t causal_backward(int elem_bytes, CausalParams p, hipStream_t s) {
  const int shift = elem_bytes == 2 ? kTileShift : kTileShift32;
  const int ntiles = (p.total >> shift) + p.seqs;
  if (int64_t(ntiles) * p.hq > 0x7fffffff) return hipErrorInvalidConfiguration;
  const dim3 queries(unsigned(ntiles) * p.hq, elem_bytes == 2 ? p.query_parts : 1), threads(kThreads);
  const dim3 keys(unsigned(ntiles) * p.hkv, p.parts);
  const dim3 rows(unsigned((int64_t(p.total) * p.hkv * (D / 4) + kThreads - 1) / kThreads));
  p.sorted = sort_queries(p, queries.x, D * elem_bytes);
  if (elem_bytes == 2) {
    hipLaunchKernelGGL((causal_query_kernel<D, 1>), queries, threads, 0, s, p, ntiles);
    launch_query_parts<D, 1>(p, ntiles, s);
    p.sorted = sort_tiles(p, int64_t(keys.x) * keys.y);
    hipLaunchKernelGGL((causal_key_kernel<D, 1>), keys, threads, 0, s, p);
    hipLaunchKernelGGL((causal_key_kernel<D, 2>), keys, threads, 0, s, p);
    if (p.parts > 1) hipLaunchKernelGGL((causal_parts_kernel<2, D>), rows, threads, 0, s, p);
  } else {
    hipLaunchKernelGGL((causal_query_f32_kernel<D, 1>), queries, threads, 0, s, p, ntiles);
    p.sorted = sort_tiles(p, int64_t(keys.x) * keys.y);
    if constexpr (D == 64) {
      hipLaunchKernelGGL((causal_key_f32_kernel<D, 0>), keys, threads, 0, s, p);
    } else {
      hipLaunchKernelGGL((causal_key_f32_kernel<D, 1>), keys, threads, 0, s, p);
      hipLaunchKernelGGL((causal_key_f32_kernel<D, 2>), keys, threads, 0, s, p);
    }
    if (p.parts > 1) hipLaunchKernelGGL((causal_parts_kernel<4, D>), rows, threads, 0, s, p);
  }
  return hipGetLastError();
}

}  // namespace

CausalParts causal_parts(int elem_bytes, int hq, int hkv, int seqs, int64_t total) {
  CausalParts x{1, 1};
  if (seqs < 1) return x;
  const int64_t tiles = (total >> (elem_bytes == 2 ? kTileShift : kTileShift32)) + 1;   // of one head
  const int64_t blocks = total / seqs / 32;                                              // of the average sequence
  const int64_t keys = std::min<int64_t>(kPartPlaces / (tiles * hkv), (hq / hkv) * blocks / (elem_bytes == 2 ? 8 : 4));
  const int64_t queries = std::min<int64_t>(kQueryPartPlaces / (tiles * hq), blocks / 8);
  x.keys = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(keys, kMaxKeyParts)));
  if (elem_bytes == 2) x.queries = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(queries, kMaxQueryParts)));
  return x;
}

hipError_t launch_causal_forward(int elem_bytes, int head_dim, const CausalParams &p, hipStream_t s) {
  return head_dim == 128 ? causal_forward<128>(elem_bytes, p, s) : causal_forward<64>(elem_bytes, p, s);
}

hipError_t launch_causal_backward(int elem_bytes, int head_dim, const CausalParams &p, hipStream_t s) {
  return head_dim == 128 ? causal_backward<128>(elem_bytes, p, s) : causal_backward<64>(elem_bytes, p, s);
}

}  // namespace dmc
