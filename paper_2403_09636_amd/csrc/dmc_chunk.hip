// gfx950 kernels for a chunk of new tokens per row on top of a layer's paged
// cache: attention that leaves the cache as it is (dmc_chunk_attend), and the
// commit of the chunk or its accepted part (dmc_chunk_append).
//
// Method: Nawrot et al., "Dynamic Memory Compression" (ICML 2024), Algorithm 1
// applied to the chunk's tokens in order.  With the open slot (z, K, V) of a unit
// before the chunk as token -1, alpha_t = (k_t[0] > c) and omega_t:
//   z_t = alpha_t z_{t-1} + omega_t,   K~_t = (alpha_t z_{t-1} K~_{t-1} + omega_t k_t) / z_t,  V~ likewise.
// A state is closed when the next token opens a slot (alpha = 0).  Query t sees
// the closed cached slots, the closed states before t, and state t.
//
// Both run on the states, a segmented sum over the tokens: rows of up to 64
// tokens in one pass, longer ones from the sums of 64-token blocks.  The append
// writes closed states and the last one into pages; the attention writes every
// state (each query's own) and the closed ones by themselves, in order, so that
// they are blocks of rows like the cache's.
#include <type_traits>

#include "dmc_mfma.h"

namespace dmc {
namespace {

constexpr int kBlockShift = 6, kBlock = 1 << kBlockShift;   // tokens of a workgroup of the state kernels
constexpr int kStateThreads = 512, kStateWaves = kStateThreads / 64;
constexpr int kWaveTokens = kBlock / kStateWaves;

// The E elements of a row at `p` as floats (one access).
template <int ES, int E>
struct Elems {
  float f[E];
  __device__ __forceinline__ void load(const char *p) {
    if constexpr (ES == 2 && E == 4) {
      const uint2 w = *reinterpret_cast<const uint2 *>(p);
      f[0] = bf16_lo(w.x); f[1] = bf16_hi(w.x); f[2] = bf16_lo(w.y); f[3] = bf16_hi(w.y);
    } else if constexpr (ES == 4 && E == 4) {
      const float4 w = *reinterpret_cast<const float4 *>(p);
      f[0] = w.x; f[1] = w.y; f[2] = w.z; f[3] = w.w;
    } else {
      load_e<ES, E>(p, f);
    }
  }
  __device__ __forceinline__ void store(char *p) const {
    if constexpr (ES == 2 && E == 4) {
      *reinterpret_cast<uint2 *>(p) = make_uint2(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]));
    } else if constexpr (ES == 4 && E == 4) {
      *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
    } else {
      store_e<ES, E>(p, f);
    }
  }
};

// Tokens of a row that count: at most max_chunk, and for an append the accepted
// ones (out-of-range values are clamped).
__device__ __forceinline__ int row_tokens(const ChunkParams &p, int b, int n) {
  n = min(n, p.max_chunk);
  if (p.accepted) n = min(max(p.accepted[b], 0), n);
  return n;
}
// Whether a row's lengths are out of range: its boundaries (which may not decrease
// either), its tokens, or how many of them are accepted.
__device__ __forceinline__ bool bad_row(const ChunkParams &p, int b) {
  const int s0 = p.cu[b], s1 = p.cu[b + 1];
  bool bad = s0 < 0 || s1 > p.total || s1 < s0;
  const int n = max(clamp_token(s1, p.total) - clamp_token(s0, p.total), 0);
  bad |= n > p.max_chunk;
  if (p.accepted) bad |= p.accepted[b] < 0 || p.accepted[b] > min(n, p.max_chunk);
  return bad;
}

// One workgroup's 64-token block of one unit.
struct ChunkBlock {
  int b, u, start, n, first;   // row, unit, the row's first token and tokens, the block's first token
  int index;                   // of the block among the head's
};

// Decision (1: opens a slot) and importance of token t of the block's row.
template <int ES>
__device__ __forceinline__ bool opens(const ChunkParams &p, const ChunkBlock &c, int dg, int t, bool empty) {
  const float k0 = load_elem<ES>(p.k, int64_t(c.start + t) * p.ks[0] + dg * p.ks[1]);
  return !(k0 > p.c) || (t == 0 && empty);
}
template <int ES>
__device__ __forceinline__ float importance(const ChunkParams &p, const ChunkBlock &c, int dg, int t) {
  if (p.omega_src == 2) return 1.0f;   // uniform weighting
  const int G = p.hq / p.hkv;
  const int64_t at = int64_t(c.start + t) * p.qs[0] + int64_t(dg) * G * p.qs[1];
  if (p.omega_src == 0) return sigmoid_floor(load_elem<ES>(p.q, at));
  float x[8], sum = 0.0f;   // (up to eight heads: every load in flight)
#pragma unroll
  for (int h = 0; h < 8; ++h) x[h] = load_elem<ES>(p.q, at + min(h, G - 1) * p.qs[1]);
#pragma unroll
  for (int h = 0; h < 8; ++h) sum += h < G ? sigmoid_floor(x[h]) : 0.0f;
  return fmaxf(sum / G, 0x1p-100f);
}

// Page and slot address of slot s (key row; the value row or column follows).
__device__ __forceinline__ char *page_of(const ChunkParams &p, int u, int s) {
  return p.pool + int64_t(p.ptab[int64_t(u) * p.maxpages + (s >> p.log2p)]) * p.page_bytes;
}

// One workgroup = one 64-token block of one unit: wave w takes tokens 8 w .. + 8,
// lanes 0..31 the key's elements, lanes 32..63 the value's.  The wave's rows are
// loaded once into registers; the segment's sums before each wave come from the
// waves before it (LDS), before the block from the block records, before the row
// from the open slot.
//   SUMS    the block's record for longer rows: sums of the segment that is open at its end
//   ATTEND  every state, closed states, counts; and the plan of the attention (one more workgroup)
//   APPEND  closed states and the last one into the pages (pages allocated before)
//   ONE     the same for rows of one block: allocates the pages itself
// Bound by reading k, v and writing the states (6 prompts up to 4096 tokens, 32
// heads, d 128: SUMS 68-100 us, ATTEND 136, APPEND 120), or by the round trips of one
// workgroup on a few tokens (24 rows of 6: 10 us, 1 row of 4: 6).  Sums and z are
// fp32; a state is rounded to the cache's type as a slot of that cache is, which is
// what the token attends to.
enum { SUMS, ATTEND, APPEND, ONE };

__device__ void plan_pieces(const ChunkParams &p);

// n pages from the pool's bump pointer, all or none (by one lane): the first one, or -1.
// At rest the pointer is at most the pool's end.  The unit whose addition takes it past
// the end puts it back; until then nobody else can get pages, as every addition starts
// past the end, so that what it puts back is still what has been handed out.  Units that
// add meanwhile wait for that (their additions are undone with it) and look again, so
// that a refused request never costs another unit its pages.
// (Compare and swap serves one unit a round trip: of 24 rows of 32 heads, half or all of
// which need a page, 0.8 and 1.8 ms for the launch of 6 tokens a row; this way 18 us.)
__device__ __forceinline__ long long take_pages(const ChunkParams &p, int n) {
  unsigned long long *used = &p.ctrl->pages_used;
  const unsigned long long end = static_cast<unsigned long long>(p.num_pages), more = static_cast<unsigned long long>(n);
  for (int polls = 0; polls < (1 << 16);) {   // (a bound; the wait is for the few instructions of a running wave)
    const unsigned long long at = atomicAdd(used, more);
    if (at + more <= end) return static_cast<long long>(at);
    if (at <= end) {
      atomicExch(used, at);
      return -1;
    }
    unsigned long long now = at;
    for (; now > end && polls < (1 << 16); ++polls) {
      __builtin_amdgcn_s_sleep(1);
      now = __hip_atomic_load(used, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (now + more > end) return -1;
  }
  return -1;
}

// Pages for a unit that grows from l to l + grow slots, into the page table (by one
// wave).  False when they do not exist.
__device__ __forceinline__ bool grow_unit(const ChunkParams &p, int u, int l, int grow) {
  const int lane = threadIdx.x & 63;
  if (grow > p.max_slots - l) {
    if (lane == 0) atomicOr(&p.ctrl->flags, FLAG_SLOTS_EXHAUSTED);
    return false;
  }
  const int P = 1 << p.log2p;
  const int have = (l + P - 1) >> p.log2p, need = (l + grow + P - 1) >> p.log2p;
  if (need == have) return true;
  long long at = lane == 0 ? take_pages(p, need - have) : 0;
  at = __shfl(at, 0, 64);
  if (at < 0) {
    if (lane == 0) atomicOr(&p.ctrl->flags, FLAG_POOL_EXHAUSTED);
    return false;
  }
  for (int i = have + lane; i < need; i += 64)
    p.ptab[int64_t(u) * p.maxpages + i] = static_cast<int32_t>(at) + (i - have);
  return true;
}

template <int ES, int D, bool VT, int MODE>
__global__ __launch_bounds__(kStateThreads) void chunk_states_kernel(ChunkParams p) {
  constexpr int E = D / 32, RB = D * ES;
  constexpr bool kAppend = MODE == APPEND || MODE == ONE;
  __shared__ float s_omega[kBlock];
  __shared__ float s_sum[kStateWaves][64 * E];   // a wave's sums of its open segment
  __shared__ float s_sumz[kStateWaves];
  __shared__ unsigned long long s_mask;
  __shared__ int s_next, s_first, s_prior, s_base, s_end;
  if constexpr (MODE == ATTEND) {
    if (blockIdx.x == static_cast<unsigned>(p.blocks64)) {
      if (blockIdx.y == 0) plan_pieces(p);
      return;
    }
  }
  if (MODE != SUMS && blockIdx.x == 0 && blockIdx.y == 0) {   // (every row, also those without tokens)
    bool bad = false;
    for (int b = threadIdx.x; b < p.rows; b += kStateThreads) bad |= bad_row(p, b);
    if (bad) atomicOr(&p.ctrl->flags, FLAG_BAD_LENGTH);
  }
  const int g = blockIdx.y;
  const PackedTile pt = packed_tile(p.cu, p.rows, p.total, blockIdx.x, kBlockShift);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (pt.tile < 0 || pt.tile * kBlock >= pt.n) return;
  ChunkBlock c;
  c.b = pt.seq;
  c.u = c.b * p.hkv + g;
  c.start = pt.start;
  c.n = row_tokens(p, c.b, pt.n);
  c.first = pt.tile * kBlock;
  c.index = blockIdx.x;
  if (kAppend && p.slot_index) {   // tokens that are not appended
    for (int t = c.first + tid; t < min(c.first + kBlock, pt.n); t += kStateThreads)
      if (t >= c.n) p.slot_index[int64_t(c.start + t) * p.hkv + g] = -1;
  }
  if (c.first >= c.n) return;
  const int cnt = min(kBlock, c.n - c.first);
  const int dg = p.decision_src ? 0 : g;   // head whose neurons decide for this unit
  const int l = MODE == APPEND ? p.old_len[c.u] : p.len[c.u];
  const float zold = MODE == APPEND ? p.old_z[c.u] : p.z[c.u];
  if (MODE == APPEND && l < 0) {   // no room: dropped
    if (p.slot_index && tid < cnt) p.slot_index[int64_t(c.start + c.first + tid) * p.hkv + g] = -1;
    return;
  }

  // The wave's rows and the open slot, loaded ahead of the decisions.
  const int hb = lane >> 5, el = (lane & 31) * E;
  const char *rows = hb ? static_cast<const char *>(p.v) + (int64_t(c.start) * p.vs[0] + g * p.vs[1] + el) * ES
                        : static_cast<const char *>(p.k) + (int64_t(c.start) * p.ks[0] + g * p.ks[1] + el) * ES;
  const int64_t rst = (hb ? p.vs[0] : p.ks[0]) * ES;
  const int w0 = wave * kWaveTokens, wcnt = max(0, min(kWaveTokens, cnt - w0));
  Elems<ES, E> x[kWaveTokens];
#pragma unroll
  for (int i = 0; i < kWaveTokens; ++i)
    x[i].load(rows + int64_t(c.first + min(w0 + i, cnt - 1)) * rst);
  Elems<ES, E> open_slot;   // the cached open slot, for the row's first block
  if (pt.tile == 0 && l > 0) {
    const char *page = page_of(p, c.u, l - 1);
    const int P = 1 << p.log2p, r = (l - 1) & (P - 1);
    if (VT && hb) {
#pragma unroll
      for (int e = 0; e < E; ++e) open_slot.f[e] = load_elem<2>(page + int64_t(P) * RB, int64_t(el + e) * P + r);
    } else {
      open_slot.load(page + (int64_t(hb ? P : 0) + r) * RB + el * ES);
    }
  }
  if (wave == 0) {
    const bool here = lane < cnt;
    const int t = c.first + min(lane, cnt - 1);
    const bool o = opens<ES>(p, c, dg, t, l == 0);
    s_omega[lane] = importance<ES>(p, c, dg, t);
    const unsigned long long mask = __ballot(here && o);
    // whether the token after the block opens a slot, and the row's first token did
    const bool next = c.first + kBlock < c.n && opens<ES>(p, c, dg, c.first + kBlock, false);
    const bool first = pt.tile == 0 ? mask & 1 : opens<ES>(p, c, dg, 0, l == 0);
    // segment starts in the row's blocks before this one
    int prior = 0;
    if constexpr (MODE == ATTEND || MODE == APPEND) {
      for (int i = lane; i < pt.tile; i += 64) prior += p.starts[int64_t(g) * p.blocks64 + c.index - pt.tile + i];
#pragma unroll
      for (int o2 = 32; o2 > 0; o2 >>= 1) prior += __shfl_xor(prior, o2, 64);
    }
    prior = min(max(prior, 0), c.first);
    int base = l, end = MODE == APPEND ? p.len[c.u] : 0;   // length after the append
    if constexpr (MODE == ONE) {
      const int grow = __popcll(mask);
      end = l + grow;
      if (!grow_unit(p, c.u, l, grow)) base = -1;
    }
    if (lane == 0) {
      s_mask = mask;
      s_next = next;
      s_first = first;
      s_prior = prior;
      s_base = base;
      s_end = end;
      if constexpr (MODE == SUMS) p.starts[int64_t(g) * p.blocks64 + c.index] = __popcll(mask);
      if constexpr (MODE == ATTEND) {
        if (pt.tile == 0) p.visible[c.u] = l - (l > 0 && !first ? 1 : 0);
      }
    }
  }
  if (hb == 0 && el == 0) {   // k_t[0] <- 0
#pragma unroll
    for (int i = 0; i < kWaveTokens; ++i) x[i].f[0] = 0.0f;
  }
  __syncthreads();   // (also the new pages' table entries, in ONE)
  const unsigned long long mask = s_mask;
  if (MODE == ONE && s_base < 0) {
    if (p.slot_index && tid < cnt) p.slot_index[int64_t(c.start + c.first + tid) * p.hkv + g] = -1;
    return;
  }
  // (every wave has read the old length before the barrier)
  if (MODE == ONE && tid == 0) p.len[c.u] = s_end;
  // Sums of the wave's tokens since its last segment start.
  // (past the row's end: its last token again, used by nobody)
  const uint32_t wmask = static_cast<uint32_t>(mask >> w0) & ((1u << kWaveTokens) - 1);
  float sum[E], zs = 0.0f;
#pragma unroll
  for (int e = 0; e < E; ++e) sum[e] = 0.0f;
#pragma unroll
  for (int i = 0; i < kWaveTokens; ++i) {
    const bool keep = ((wmask >> i) & 1) == 0;
    const float w = s_omega[w0 + i];
    zs = (keep ? zs : 0.0f) + w;
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = fmaf(w, x[i].f[e], keep ? sum[e] : 0.0f);
  }
#pragma unroll
  for (int e = 0; e < E; ++e) s_sum[wave][lane * E + e] = sum[e];
  if (lane == 0) s_sumz[wave] = zs;
  __syncthreads();

  // Sums of the segment that is open before token `t0` of the block (wave w's first
  // token, or its end): waves back to the one with a start, else the blocks before.
  auto open_before = [&](int w, float (&o)[E], float &z) {
    z = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.0f;
    for (int j = w - 1; j >= 0; --j) {
      z += s_sumz[j];
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] += s_sum[j][lane * E + e];
      if ((static_cast<uint32_t>(mask >> (j * kWaveTokens)) & ((1u << kWaveTokens) - 1)) != 0) return;
    }
    if (pt.tile == 0) {   // the cached open slot (an empty unit's first token opens one)
      if (l > 0) {
        z += zold;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = fmaf(zold, open_slot.f[e], o[e]);
      }
      return;
    }
    // records of the blocks before, back to one with a start (its record holds
    // what is open at its end; the first block's includes the cached open slot);
    // one after another, so a row that never opens a slot walks back over all of it
    const int32_t *st = p.starts + int64_t(g) * p.blocks64 + c.index;
    for (int j = 1; j <= pt.tile; ++j) {
      const float *cr = p.carry + (int64_t(g) * p.blocks64 + c.index - j) * carry_stride(D);
      z += cr[2 * D];
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] += cr[hb * D + el + e];
      if (st[-j] > 0) break;
    }
  };

  if constexpr (MODE == SUMS) {
    if (wave != 0) return;
    // what is open at the block's end: without the blocks before (their records
    // are added by the readers), but with the cached open slot in the first block
    float o[E], z = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.0f;
    if (pt.tile == 0) {
      open_before(kStateWaves, o, z);
    } else {
      for (int j = kStateWaves - 1; j >= 0; --j) {
        z += s_sumz[j];
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] += s_sum[j][lane * E + e];
        if ((static_cast<uint32_t>(mask >> (j * kWaveTokens)) & ((1u << kWaveTokens) - 1)) != 0) break;
      }
    }
    float *cr = p.carry + (int64_t(g) * p.blocks64 + c.index) * carry_stride(D);
#pragma unroll
    for (int e = 0; e < E; ++e) cr[hb * D + el + e] = o[e];
    if (lane == 0) cr[2 * D] = z;
    return;
  }
  if (wcnt == 0) return;
  // Pages of the wave's slots (its tokens' lie side by side), one to a lane.
  const int slot0 = l - 1 + s_prior + __popcll(mask & ((1ull << w0) - 1)), page0 = max(slot0, 0) >> p.log2p;
  int pages = 0;
  if (kAppend && lane < 4) pages = p.ptab[int64_t(c.u) * p.maxpages + min(page0 + lane, p.maxpages - 1)];
  open_before(wave, sum, zs);
  const int P = 1 << p.log2p;
  const int64_t out_row = (int64_t(g) * p.total + c.start + c.first) * D + el;
  const int blk32 = (c.start >> 5) + c.b;   // the row's first block of closed states
#pragma unroll
  for (int i = 0; i < kWaveTokens; ++i) {
    const int t = w0 + i;
    const bool keep = ((wmask >> i) & 1) == 0;
    const float w = s_omega[t];
    zs = (keep ? zs : 0.0f) + w;
    Elems<ES, E> s;
    // (bf16: the reciprocal's last bit is far below the state's rounding)
    const float inv = ES == 2 ? __builtin_amdgcn_rcpf(zs) : 1.0f / zs;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      sum[e] = fmaf(w, x[i].f[e], keep ? sum[e] : 0.0f);
      s.f[e] = sum[e] * inv;
    }
    if (i >= wcnt) continue;
    // segments opened up to this token, and whether it is the last of its own
    const int seg = s_prior + __popcll(mask & (~0ull >> (63 - t)));
    const bool last = c.first + t + 1 == c.n;
    const bool closed = !last && (t == kBlock - 1 ? s_next != 0 : ((mask >> (t + 1)) & 1) != 0);
    if constexpr (MODE == ATTEND) {
      const int ord = seg - s_first;   // closed states of the row before this token
      s.store((hb ? p.state_v : p.state_k) + (out_row + int64_t(t) * D) * ES);
      if (lane == 0) p.before[int64_t(g) * p.total + c.start + c.first + t] = ord;
      if (closed) {
        const int64_t block = int64_t(g) * p.blocks32 + blk32 + (ord >> 5);
        if (VT && hb) {
#pragma unroll
          for (int e = 0; e < E; ++e)
            store_e<2, 1>(p.closed_v + ((block * D + el + e) * 32 + (ord & 31)) * 2, &s.f[e]);
        } else {
          s.store((hb ? p.closed_v : p.closed_k) + ((block * 32 + (ord & 31)) * D + el) * ES);
        }
      }
    } else {
      const int slot = l - 1 + seg;
      if (lane == 0 && p.slot_index) p.slot_index[int64_t(c.start + c.first + t) * p.hkv + g] = slot;
      if ((closed || last) && slot >= 0 && slot < s_end) {   // (always, for boundaries that do not decrease)
        char *page = p.pool + int64_t(__shfl(pages, (slot >> p.log2p) - page0, 64)) * p.page_bytes;
        const int r = slot & (P - 1);
        if (VT && hb) {
#pragma unroll
          for (int e = 0; e < E; ++e)
            store_e<2, 1>(page + int64_t(P) * RB + (int64_t(el + e) * P + r) * 2, &s.f[e]);
        } else {
          s.store(page + (int64_t(hb ? P : 0) + r) * RB + el * ES);
        }
        if (last && lane == 0) p.z[c.u] = zs;
      }
    }
  }
}

// Append of longer rows, one wave per unit: the new length from the blocks'
// segment starts, pages; old length and z are kept for the state pass.
__global__ __launch_bounds__(kThreads) void chunk_grow_kernel(ChunkParams p) {
  const int lane = threadIdx.x & 63;
  const int u = __builtin_amdgcn_readfirstlane(blockIdx.x * kWaves + (threadIdx.x >> 6));
  if (u >= p.units) return;
  const int b = u / p.hkv, g = u - b * p.hkv;
  const int s0 = clamp_token(p.cu[b], p.total), s1 = clamp_token(p.cu[b + 1], p.total);
  const int n = row_tokens(p, b, max(s1 - s0, 0));
  if (n == 0) return;
  const int blocks = (n + kBlock - 1) >> kBlockShift;
  const int64_t at = int64_t(g) * p.blocks64 + (s0 >> kBlockShift) + b;
  int grow = 0;
  for (int i = lane; i < blocks; i += 64) grow += p.starts[at + i];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) grow += __shfl_xor(grow, o, 64);
  grow = min(max(grow, 0), n);   // (as clamped in the state pass, for boundaries that decrease)
  const int l = p.len[u];
  const bool ok = grow_unit(p, u, l, grow);
  if (lane == 0) {
    p.old_len[u] = ok ? l : -1;
    p.old_z[u] = p.z[u];
    if (ok) p.len[u] = l + grow;
  }
}

// ---------------------------------------------------------------------------
// Attention.  A tile is 32 (narrow) or 128 (wide) query columns of one unit,
// token-major (column c is token c / G, head c % G).  What it attends to is a
// list of 32-row blocks: the unit's visible cached slots, then the closed states
// before its last token; plus each column's own state.  A unit's tiles are cut
// into pieces of that list where units are few or long, which meet in a combine
// pass; one workgroup per piece.  The lengths are on the device, so the plan is
// made there: a piece is about total / budget blocks, so that there are never
// more than tiles + budget pieces.  Few units of one narrow tile each get a fixed
// number of places instead (fixed_parts), which takes no plan and fewer loads that
// wait for each other.
// ---------------------------------------------------------------------------
struct UnitPlan {
  int start, n;        // the row's first token and tokens
  int tiles, blocks;   // column tiles; 32-row blocks of the whole list
};
__device__ __forceinline__ UnitPlan unit_plan(const ChunkParams &p, int u) {
  const int b = u / p.hkv;
  const int s0 = clamp_token(p.cu[b], p.total), s1 = clamp_token(p.cu[b + 1], p.total);
  const int n = min(max(s1 - s0, 0), p.max_chunk);
  UnitPlan x;
  x.start = s0;
  x.n = n;
  x.tiles = (n + (1 << p.tile_shift) - 1) >> p.tile_shift;
  // (the chunk's share at most every token a slot; half of it on average over the tiles)
  x.blocks = ((p.len[u] + 31) >> 5) + ((n + 63) >> 6);
  return x;
}

// Units are dealt to the XCDs (each with its own L2, so that a unit's tiles share
// its slots there) in descending order of their blocks, back and forth: rows and
// heads differ by orders of magnitude (a ragged batch of prompts, heads of other
// compression).  The order comes from a counting sort by cost, eight buckets to a
// factor of two.
constexpr int kCostBuckets = 64 * 8;
__device__ __forceinline__ int cost_bucket(float cost) {   // (most expensive first)
  const int e = static_cast<int>(__float_as_uint(cost + 1.0f) >> 20) - (127 << 3);
  return kCostBuckets - 1 - min(e, kCostBuckets - 1);
}

__device__ void plan_pieces(const ChunkParams &p) {
  __shared__ long long s_total[kStateWaves];
  __shared__ int s_split[kStateWaves], s_bucket[kCostBuckets], s_sum[kStateWaves], s_pieces[8 * 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (p.units + kStateThreads - 1) / kStateThreads;
  const int i0 = min(tid * per, p.units), i1 = min(i0 + per, p.units);
  UnitPlan own{};   // the thread's first unit (its only one, of up to 512)
  if (i0 < i1) own = unit_plan(p, i0);
  auto plan_of = [&](int u) { return u == i0 ? own : unit_plan(p, u); };
  for (int i = tid; i < kCostBuckets; i += kStateThreads) s_bucket[i] = 0;
  __syncthreads();
  long long total = 0;
  for (int u = i0; u < i1; ++u) {
    const UnitPlan x = plan_of(u);
    total += static_cast<long long>(x.tiles) * x.blocks;
    atomicAdd(&s_bucket[cost_bucket(static_cast<float>(x.tiles) * x.blocks)], 1);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o, 64);
  if (lane == 0) s_total[wave] = total;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int w = 0; w < kStateWaves; ++w) total += s_total[w];
  int size = 1 << 30;
  if (p.piece_budget > 0) {
    const long long want = (total + p.piece_budget - 1) / p.piece_budget;
    size = static_cast<int>(want > p.piece_min ? min(want, 1ll << 30) : p.piece_min);
  }
  // Bucket sizes -> first positions.
  static_assert(kCostBuckets == kStateThreads, "a bucket to a thread");
  const int here = s_bucket[tid];
  int ends = here;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(ends, o, 64);
    if (lane >= o) ends += t;
  }
  if (lane == 63) s_sum[wave] = ends;
  // Pieces per tile.  Units of several have floor(blocks / size) >= 2 of them per
  // tile, so that their pieces, which have a record each, are at most the budget.
  int split = 0;
  for (int u = i0; u < i1; ++u) {
    const UnitPlan x = plan_of(u);
    const int np = max(1, x.blocks / size);
    p.pieces[u] = np;   // (for the combine pass)
    split += np > 1 ? x.tiles * np : 0;
  }
  int incs = split;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int ts = __shfl_up(incs, o, 64);
    if (lane >= o) incs += ts;
  }
  if (lane == 63) s_split[wave] = incs;
  __syncthreads();
  int first = ends - here, rec = incs - split;
  for (int w = 0; w < wave; ++w) {
    first += s_sum[w];
    rec += s_split[w];
  }
  s_bucket[tid] = first;
  __syncthreads();
  const int row = (p.units + 7) >> 3;   // units of an XCD
  for (int u = i0; u < i1; ++u) {
    const UnitPlan x = plan_of(u);
    const int at = atomicAdd(&s_bucket[cost_bucket(static_cast<float>(x.tiles) * x.blocks)], 1);
    const int k = at >> 3, xcd = k & 1 ? 7 - (at & 7) : at & 7, np = max(1, x.blocks / size);
    int32_t *info = p.unit_order + (int64_t(xcd) * row + k) * 8;
    *reinterpret_cast<int4 *>(info) = make_int4(u, np, rec, x.start);
    info[4] = x.n;
    if (row < 64) s_pieces[xcd * 64 + k] = x.tiles * np;
    else p.piece_base[xcd * (row + 1) + k + 1] = x.tiles * np;
    p.record_base[u] = rec;
    rec += np > 1 ? x.tiles * np : 0;
  }
  if (tid < 8 * row - p.units) {   // places without a unit, in the last line
    const int at = p.units + tid, k = at >> 3, xcd = k & 1 ? 7 - (at & 7) : at & 7;
    int32_t *info = p.unit_order + (int64_t(xcd) * row + k) * 8;   // (no pieces: never looked up)
    *reinterpret_cast<int4 *>(info) = make_int4(0, 1, 0, 0);
    info[4] = 0;
    if (row < 64) s_pieces[xcd * 64 + k] = 0;
    else p.piece_base[xcd * (row + 1) + k + 1] = 0;
  }
  __syncthreads();   // (counts of all units written, by this workgroup)
  for (int xcd = wave; xcd < 8; xcd += kStateWaves) {   // counts -> pieces before
    int32_t *base = p.piece_base + xcd * (row + 1);
    int run = 0;
    for (int i = 0; i < row; i += 64) {
      int incl = i + lane >= row ? 0 : row < 64 ? s_pieces[xcd * 64 + lane] : base[i + lane + 1];
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int t = __shfl_up(incl, o, 64);
        if (lane >= o) incl += t;
      }
      if (i + lane < row) base[i + lane + 1] = run + incl;
      run += __shfl(incl, 63, 64);
    }
    if (lane == 0) base[0] = 0;
  }
}

// A workgroup's piece of a tile.
struct Piece {
  int u, b, g, start, n;   // unit, row, kv head, the row's first token and tokens
  int tile, part, parts;   // column tile, piece of it
  int record;              // its partial record, if the tile has several pieces
};
__device__ __forceinline__ bool find_piece(const ChunkParams &p, Piece &x) {
  const int lane = threadIdx.x & 63;
  if (p.fixed_parts > 0) {
    x.u = blockIdx.x / p.fixed_parts;
    x.part = blockIdx.x - x.u * p.fixed_parts;
    x.parts = p.fixed_parts;
    x.record = blockIdx.x;
    x.b = x.u / p.hkv;
    x.g = x.u - x.b * p.hkv;
    x.tile = 0;
    x.start = __builtin_amdgcn_readfirstlane(clamp_token(p.cu[x.b], p.total));
    const int end = __builtin_amdgcn_readfirstlane(clamp_token(p.cu[x.b + 1], p.total));
    x.n = min(max(end - x.start, 0), p.max_chunk);
    return x.n > 0;
  }
  const int row = (p.units + 7) >> 3, slots = gridDim.x >> 3;
  int xcd = blockIdx.x & 7, idx = blockIdx.x >> 3;   // (workgroup i runs on XCD i mod 8)
  const int mine = p.piece_base[(lane & 7) * (row + 1) + row];   // pieces of XCD `lane`
  const int step0 = (row + 63) >> 6, at0 = min(lane * step0, row);
  int before = p.piece_base[xcd * (row + 1) + at0];   // (ahead of what decides whether it is needed)
  const int count = __builtin_amdgcn_readlane(mine, xcd);
  if (idx >= count) {   // a place left over: a piece of an XCD that has more than its places
    int spare = idx - count;
    for (int i = 0; i < xcd; ++i) spare += max(slots - __builtin_amdgcn_readlane(mine, i), 0);
    for (xcd = 0; xcd < 8; ++xcd) {
      const int over = max(__builtin_amdgcn_readlane(mine, xcd) - slots, 0);
      if (spare < over) break;
      spare -= over;
    }
    if (xcd == 8) return false;
    idx = slots + spare;
    before = p.piece_base[xcd * (row + 1) + at0];
  }
  const int32_t *base = p.piece_base + xcd * (row + 1);
  int lo = 0, n = row, step = step0;   // the last of its units with pieces before <= idx
  while (true) {
    const bool le = lane == 0 || (lane * step < n && before <= idx);
    const int k = 63 - __clzll(static_cast<long long>(__ballot(le)));
    const int end = lo + n;
    lo += k * step;
    n = min(step, end - lo);
    before = __builtin_amdgcn_readlane(before, k);
    if (n <= 1) break;
    step = (n + 63) >> 6;
    before = base[lo + min(lane * step, n - 1)];
  }
  // (visibly uniform: every branch on them would otherwise be made per lane)
  const int rel = __builtin_amdgcn_readfirstlane(idx - before);
  const int32_t *info = p.unit_order + __builtin_amdgcn_readfirstlane(xcd * row + lo) * int64_t(8);
  const int4 i4 = *reinterpret_cast<const int4 *>(info);
  x.n = __builtin_amdgcn_readfirstlane(info[4]);
  x.u = __builtin_amdgcn_readfirstlane(i4.x);
  x.b = x.u / p.hkv;
  x.g = x.u - x.b * p.hkv;
  x.parts = __builtin_amdgcn_readfirstlane(i4.y);
  x.record = __builtin_amdgcn_readfirstlane(i4.z) + rel;
  x.start = __builtin_amdgcn_readfirstlane(i4.w);
  const int tiles = (x.n + (1 << p.tile_shift) - 1) >> p.tile_shift;
  const int t = rel / x.parts;
  x.part = rel - t * x.parts;
  x.tile = tiles - 1 - t;   // latest tokens (most states) first
  return x.tile >= 0;
}

// Closed states of the row before its token t, and cached slots that the unit's
// chunk attends to, as the state pass left them.  (Clamped: with boundaries that
// decrease, rows overlap or have no pass of their own; what they read then is
// undefined, but stays inside the workspace and the unit's pages.)
__device__ __forceinline__ int closed_before(const ChunkParams &p, const Piece &x, int t) {
  return min(max(p.before[int64_t(x.g) * p.total + x.start + t], 0), t);
}
__device__ __forceinline__ int visible_slots(const ChunkParams &p, int u) {
  return __builtin_amdgcn_readfirstlane(min(max(p.visible[u], 0), p.len[u]));
}

// Pieces of a unit's one tile where every unit has fixed_parts places: as many as
// give each piece_min of its nb blocks, or one.
__device__ __forceinline__ int fixed_parts_of(const ChunkParams &p, int nb) {
  return max(1, min(p.fixed_parts, nb / p.piece_min));
}

// A page-table entry by a scalar load (uniform address; written by earlier launches).
__device__ __forceinline__ int page_entry(const int32_t *ptab, int64_t i) {
  return *reinterpret_cast<const __attribute__((address_space(4))) int32_t *>(reinterpret_cast<uintptr_t>(ptab + i));
}

// ---------------------------------------------------------------------------
// bf16, on v_mfma_f32_32x32x16_bf16 (lane l: column l % 32, half l / 32):
//   S^T[slot][col] = K . Q^T,   O^T[dim][col] += V^T P^T
// with score row m holding slot pi(m), so that a lane's score registers are its
// operand of the second product.  Every column starts from its own state in one
// of its tile's pieces (weight 1, its score the running maximum).
//
// WIDE (many query rows): four waves of 32 columns share the blocks, which come
// into LDS by direct transfers (a ring of four, three ahead); bound by the
// matrix cores and the softmax (512 tokens of 4 rows, 64/8 heads, on 6000 slots: 502
// us, matrix pipes busy for 40 % of the SIMD cycles, vector issue 31 %, LDS 20 %).
// Narrow (few rows): one tile of 32 columns whose waves take every fourth block, the
// keys straight into registers and the values into a ring of two blocks of the wave's
// own, one block ahead; bound by memory (two workgroups and 128 KB of requests per
// compute unit; 24 rows of 6 tokens, 32 heads, up to 4096 slots: 90 us, 5.2 TB/s).
// (Medians of a trace.)  The kernels for pages smaller than a block spill 3 to 7
// registers at d = 128.
//
// BIG: pages of >= 32 slots (a block lies in one page); VT: value pages, and
// the blocks of closed values, stored transposed.
// ---------------------------------------------------------------------------
template <int D, int G, bool VT, bool BIG, bool WIDE>
__global__ __launch_bounds__(kThreads, 2) void chunk_attend_kernel(ChunkParams p) {
  static_assert(!VT || BIG, "transposed value pages hold 32 slots");
  constexpr int T = 32 / G;                 // tokens of 32 columns
  constexpr int KS = D / 16, NTL = D / 32, RB = D * 2, CPR = D / 8, BLK = 32 * RB;
  constexpr int kSt = WIDE ? 4 : 2;
  constexpr int DPW = BLK / 16 / kThreads;  // WIDE: transfers per thread, block and half
  constexpr int DPB = BLK / 1024;           // narrow: transfers per wave and block of values
  constexpr int COLS = WIDE ? kWaves * 32 : 32;
  // WIDE: a block's keys, then its values; narrow: each wave's values.
  constexpr int SLOT = WIDE ? 2 * BLK : kWaves * BLK;
  __shared__ __align__(16) unsigned char ring0[SLOT], ring1[SLOT];
  __shared__ __align__(16) unsigned char ring2[WIDE ? SLOT : 16], ring3[WIDE ? SLOT : 16];
  __shared__ float s_m[WIDE ? 1 : kWaves * 32], s_l[WIDE ? 1 : kWaves * 32];
  auto slot = [&](auto st_c) -> unsigned char * {
    constexpr int S = decltype(st_c)::value;
    if constexpr (S == 0) return ring0;
    else if constexpr (S == 1) return ring1;
    else if constexpr (S == 2) return ring2;
    else return ring3;
  };
  Piece x;
  if (!find_piece(p, x)) return;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, hb = lane >> 5;
  const int t0 = x.tile << p.tile_shift;                       // the tile's first token
  const int a = WIDE ? t0 + wave * T : t0;                     // this wave's
  const int cnt = max(0, min(T, x.n - a));
  const int tok = col / G, head = col - tok * G;
  const bool colv = tok < cnt;
  const int64_t token = x.start + (colv ? a + tok : 0);
  const int last = min(t0 + (WIDE ? kWaves * T : T), x.n) - 1;   // the tile's last token
  const int lim = colv ? closed_before(p, x, a + tok) : 0;     // closed states that the column sees
  const int top = __builtin_amdgcn_readfirstlane(closed_before(p, x, last));   // that the tile sees
  const int lim_hi = cnt > 0 ? __builtin_amdgcn_readfirstlane(closed_before(p, x, a + cnt - 1)) : 0;   // the wave
  const int lim_lo = cnt == T ? __builtin_amdgcn_readfirstlane(closed_before(p, x, a)) : 0;   // every column
  const int vis = visible_slots(p, x.u);
  const int nbc = (vis + 31) >> 5, nb = nbc + ((top + 31) >> 5);
  if (p.fixed_parts > 0) {
    x.parts = fixed_parts_of(p, nb);
    if (x.part >= x.parts) return;
  }
  const int b0 = static_cast<int>(int64_t(nb) * x.part / x.parts);
  const int b1 = static_cast<int>(int64_t(nb) * (x.part + 1) / x.parts);   // this piece's blocks
  const uint4 zero4 = make_uint4(0, 0, 0, 0);
  const float sl2 = p.scale_log2;

  uint4 qop[KS];
  // (the lowest finite value: a wave that has seen nothing must not outweigh any score)
  float m = lowest(), ls = 0.0f;
  f32x16_t acc[NTL];
#pragma unroll
  for (int i = 0; i < NTL; ++i) acc[i] = f32x16_t{};
  // Queries and own states of the columns, once the first blocks are on their way.
  auto load_columns = [&]() {
    // Q^T operand (q[0] is not part of the score).
    const char *qr = static_cast<const char *>(p.q) + (token * p.qs[0] + (x.g * G + head) * p.qs[1]) * 2;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qop[ks] = colv ? ld16(qr + ks * 32 + hb * 16) : zero4;
    if (hb == 0) qop[0].x &= 0xffff0000u;
    // The column's own state, in the tile's last piece (by the narrow wave with the fewest blocks).
    if (x.part != x.parts - 1 || !(WIDE || wave == ((b1 - b0) & (kWaves - 1)))) return;
    const int64_t row = (int64_t(x.g) * p.total + token) * RB;
    float d = 0.0f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const uint4 kv = ld16(p.state_k + row + ks * 32 + hb * 16);
      QSlice<2> q;
      q.w = qop[ks];
      d += q.dot(kv);
    }
    d += __shfl_xor(d, 32, 64);
    if (colv) {
      m = d * sl2;
      // weight 1, relative to itself; 0 for a score of -infinity (NaN for the row if it sees nothing else), and
      // a score of +infinity or NaN makes the row NaN, whatever else it sees
      const float w = m == neg_inf() ? 0.0f : m < -neg_inf() ? 1.0f : __builtin_nanf("");
      if (m == neg_inf()) m = lowest();
      ls = hb == 0 ? w : 0.0f;   // (counted once per column)
#pragma unroll
      for (int i = 0; i < NTL; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint2 v = *reinterpret_cast<const uint2 *>(p.state_v + row + (32 * i + 8 * j + 4 * hb) * 2);
          acc[i][4 * j + 0] = w * bf16_lo(v.x);
          acc[i][4 * j + 1] = w * bf16_hi(v.x);
          acc[i][4 * j + 2] = w * bf16_lo(v.y);
          acc[i][4 * j + 3] = w * bf16_hi(v.y);
        }
    }
  };

  // Where a block lies.  Cached: BIG pages hold it whole; of smaller pages, a run
  // of rows (8 or more, so that a transfer of 1 KB lies in one) each.
  const int P = 1 << p.log2p;
  const int64_t table = int64_t(x.u) * p.maxpages;
  const int64_t closed = int64_t(x.g) * p.blocks32 + (x.start >> 5) + x.b;   // the row's first block of closed states
  auto page_index = [&](int s) { return page_entry(p.ptab, table + (min(s, max(vis - 1, 0)) >> p.log2p)); };
  const char *kclosed = p.closed_k + closed * BLK, *vclosed = p.closed_v + closed * BLK;

  // The scores of one block's slots against the columns -> probabilities, in
  // the operand layout; `first`: the block's first slot, cached or closed state.
  bool left_out = false;
  auto weights = [&](const f32x16_t &sc, int kb, float (&sv)[16], bool &masked) {
    const bool cached = kb < nbc;
    const int first = (cached ? kb : kb - nbc) * 32;
    masked = first + 32 > (cached ? vis : lim_lo);
#pragma unroll
    for (int rr = 0; rr < 16; ++rr) sv[rr] = sc[rr];
    if (masked) {
      const int rel = one_register((cached ? vis : lim) - first - 8 * hb);
#pragma unroll
      for (int rr = 0; rr < 16; ++rr)
        if (score_row(rr) >= rel) sv[rr] = neg_inf();
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
  };
  // P rounded to bf16, the type of the value product's operands (off by at most 2^-8 of
  // each, at random; the output is rounded by as much); its sum is over the rounded
  // values, so that the weights add up to 1.
  auto operands = [&](const float (&ev)[16], uint4 (&pb)[2]) {
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      uint32_t w[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        w[q] = cvt_pk_bf16(ev[8 * kk + 2 * q], ev[8 * kk + 2 * q + 1]);
        ls = add_pair(w[q], ls);
      }
      pb[kk] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  };
  // A masked block's values: rows past the slots hold anything and are cleared;
  // closed states that only some columns see keep their finite elements.
  auto clean_values = [&](uint4 (&va)[NTL][2], int kb) {
    const bool cached = kb < nbc;
    const int end = (cached ? vis : top) - (cached ? kb : kb - nbc) * 32;
    if (end < 32) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        const int keep = end - (16 * kk + 8 * hb);
        uint32_t msk[4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
          msk[q] = (2 * q < keep ? 0x0000ffffu : 0u) | (2 * q + 1 < keep ? 0xffff0000u : 0u);
#pragma unroll
        for (int i = 0; i < NTL; ++i) {
          va[i][kk].x &= msk[0];
          va[i][kk].y &= msk[1];
          va[i][kk].z &= msk[2];
          va[i][kk].w &= msk[3];
        }
      }
    }
    if (!cached) {
#pragma unroll
      for (int i = 0; i < NTL; ++i) left_out |= leave_out_nonfinite(va[i]);
    }
  };
  uint32_t traddr[NTL][2], vtaddr[2];
  if constexpr (VT) {
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) vtaddr[kk] = col * 64 + (((2 * kk + hb) ^ vt_swizzle(col)) * 16);
  } else {
    tr_offsets<D, 1>(lane, traddr);
  }
  auto value_operand = [&](const char *vd, int i, int kk) {
    if constexpr (VT) return *reinterpret_cast<const uint4 *>(vd + 2048 * i + vtaddr[kk]);
    else return tr_operand<RB>(vd, traddr[i], kk);
  };
  const int krow = score_slot(col);

  if constexpr (WIDE) {
    // This thread's chunks of a block and their offsets (rows XOR-swizzled).
    uint32_t koff[DPW], voff[DPW];
    int krow_of[DPW];
#pragma unroll
    for (int i = 0; i < DPW; ++i) {
      const int c = (i * kWaves + wave) * 64 + lane;
      const int row = c / CPR, pc = c - row * CPR;
      krow_of[i] = row;
      koff[i] = row * RB + (pc ^ k_swizzle<CPR>(row)) * 16;
      if constexpr (VT) {
        const int dim = c >> 2;
        voff[i] = dim * 64 + ((c & 3) ^ vt_swizzle(dim)) * 16;
      } else {
        voff[i] = row * RB + (pc ^ v_swizzle<CPR>(row)) * 16;
      }
    }
    // Pages of the block that is issued next, looked up one issue ahead.
    int pg[BIG ? 1 : DPW];
    auto look_up = [&](int kb) {
#pragma unroll
      for (int i = 0; i < (BIG ? 1 : DPW); ++i)
        pg[i] = kb < min(nbc, b1) ? page_index(kb * 32 + (BIG ? 0 : (i * kWaves + wave) * (1024 / RB))) : 0;
    };
    // Every call issues 2 DPW transfers per wave; those past the piece are off.
    auto issue = [&](int kb, auto st_c) {
      unsigned char *dst = slot(st_c);
      const bool on = kb < b1, cached = kb < nbc;
      const int first = (cached ? kb : kb - nbc) * 32;
#pragma unroll
      for (int i = 0; i < DPW; ++i) {
        unsigned char *kdst = dst + (i * kWaves + wave) * 1024;
        if (BIG || !cached) {
          const char *kp, *vp;
          if (cached) {
            const char *page = p.pool + int64_t(pg[0]) * p.page_bytes;
            kp = page + int64_t(first & (P - 1)) * RB;
            vp = VT ? page + int64_t(P) * RB : kp + int64_t(P) * RB;
          } else {
            kp = kclosed + int64_t(first) * RB;
            vp = vclosed + int64_t(first) * RB;
          }
          dma16_s(kdst, uniform_ptr(kp), koff[i], on);
          dma16_s(kdst + BLK, uniform_ptr(vp), voff[i], on);
        } else {
          const int r0 = (i * kWaves + wave) * (1024 / RB), s = first + r0;   // first row of the transfer
          const bool live = on && s < vis;
          const char *base = uniform_ptr(p.pool + int64_t(pg[BIG ? 0 : i]) * p.page_bytes +
                                         int64_t(live ? s & (P - 1) : 0) * RB);
          const bool lane_on = first + krow_of[i] < vis;
          const uint32_t rel = uint32_t(r0 * RB);
          dma16_s(kdst, base, lane_on ? koff[i] - rel : kOutOfRange, live);
          dma16_s(kdst + BLK, base, lane_on ? uint32_t(P * RB) + voff[i] - rel : kOutOfRange, live);
        }
      }
      look_up(kb + 1);
    };
    uint32_t kaddr[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kaddr[ks] = row_offset<D, 0>(krow, ks, hb);
    // Whether the wave's columns see anything of a block.
    auto seen = [&](int kb) { return cnt > 0 && kb < b1 && (kb < nbc || (kb - nbc) * 32 < lim_hi); };
    look_up(b0);
    issue(b0, std::integral_constant<int, 0>{});
    issue(b0 + 1, std::integral_constant<int, 1>{});
    issue(b0 + 2, std::integral_constant<int, 2>{});
    load_columns();
    f32x16_t scn = f32x16_t{};
    wait_vmcnt<(kSt - 2) * 2 * DPW>();   // block b0 has landed
    ring_barrier();
    if (seen(b0)) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        scn = mfma_32x32x16(*reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(ring0) + kaddr[ks]),
                            qop[ks], scn);
    }
    // Step kb runs block kb's exponentials between the score products of block
    // kb + 1 (order pinned), then block kb's value product.
    auto step = [&](auto stage_c, int kb) {
      constexpr int ST = decltype(stage_c)::value, SN = (ST + 1) % kSt;
      wait_vmcnt<(kSt - 3) * 2 * DPW>();   // block kb + 1 has landed
      ring_barrier();   // every wave is past step kb - 1: its ring slot is free
      issue(kb + kSt - 1, std::integral_constant<int, (ST + kSt - 1) % kSt>{});
      if (!seen(kb)) return;
      const char *vd = reinterpret_cast<const char *>(slot(stage_c)) + BLK;
      const char *kn = reinterpret_cast<const char *>(slot(std::integral_constant<int, SN>{}));   // block kb + 1's keys
      // (past the piece the next scores are not used)
      uint4 kr[4], va[NTL][2];
#pragma unroll
      for (int i = 0; i < 3; ++i) kr[i] = *reinterpret_cast<const uint4 *>(kn + kaddr[i]);
      float sv[16];
      bool masked;
      weights(scn, kb, sv, masked);
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
        va[ks >> 1][ks & 1] = value_operand(vd, ks >> 1, ks & 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      scn = sc;
      uint4 pb[2];
      operands(ev, pb);
      if (masked) clean_values(va, kb);
#pragma unroll
      for (int i = 0; i < NTL; ++i)
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) acc[i] = mfma_32x32x16(va[i][kk], pb[kk], acc[i]);
    };
    for (int kb = b0; kb < b1; kb += kSt) {
      step(std::integral_constant<int, 0>{}, kb);
      step(std::integral_constant<int, 1>{}, kb + 1);
      step(std::integral_constant<int, 2>{}, kb + 2);
      step(std::integral_constant<int, 3>{}, kb + 3);
    }
  } else {
    // A block's keys: row pi(col), 16-byte slices 2 ks + hb; of pages smaller than
    // a block each lane its row's page.  Slots past the visible ones read the last.
    int page = 0;   // of the block that is issued next (BIG), looked up one block ahead
    auto look_up = [&](int kb) {
      if (BIG) page = kb < min(nbc, b1) ? page_index(kb * 32) : 0;
    };
    auto load_keys = [&](int kb, uint4 (&k)[KS]) {
      const bool cached = kb < nbc;
      const int first = (cached ? kb : kb - nbc) * 32;
      const char *row;
      if (!cached) {
        row = kclosed + int64_t(first + krow) * RB;
      } else if constexpr (BIG) {
        row = p.pool + int64_t(page) * p.page_bytes + int64_t((first & (P - 1)) + krow) * RB;
      } else {
        const int s = min(first + krow, vis - 1);
        row = p.pool + int64_t(p.ptab[table + (s >> p.log2p)]) * p.page_bytes + int64_t(s & (P - 1)) * RB;
      }
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) k[ks] = ld16(row + ks * 32 + hb * 16);
    };
    uint32_t voff[DPB];
#pragma unroll
    for (int i = 0; i < DPB; ++i) {
      const int c = i * 64 + lane;
      if constexpr (VT) {
        const int dim = c >> 2;
        voff[i] = dim * 64 + ((c & 3) ^ vt_swizzle(dim)) * 16;
      } else {
        const int row = c / CPR, pc = c - row * CPR;
        voff[i] = row * RB + (pc ^ v_swizzle<CPR>(row)) * 16;
      }
    }
    auto issue_values = [&](int kb, auto st_c) {
      unsigned char *dst = slot(st_c) + wave * BLK;
      const bool cached = kb < nbc;
      const int first = (cached ? kb : kb - nbc) * 32;
      if (BIG || !cached) {
        const char *vp = vclosed + int64_t(first) * RB;
        if (cached) {
          vp = p.pool + int64_t(page) * p.page_bytes + int64_t(P) * RB + (VT ? 0 : int64_t(first & (P - 1)) * RB);
        }
        vp = uniform_ptr(vp);
#pragma unroll
        for (int i = 0; i < DPB; ++i) dma16_s(dst + i * 1024, vp, voff[i]);
      } else {
        constexpr int RT = 1024 / RB;   // rows of a transfer
#pragma unroll
        for (int i = 0; i < DPB; ++i) {
          const int s = min(first + i * RT, (vis - 1) & ~(RT - 1));   // (past the visible slots: rows of the last page)
          const char *base = uniform_ptr(p.pool + int64_t(page_index(s)) * p.page_bytes + int64_t(P + (s & (P - 1))) * RB);
          dma16_s(dst + i * 1024, base, voff[i] - uint32_t(i * 1024));
        }
      }
    };
    uint4 kv[2][KS];
    int kb = b0 + wave;
    auto step = [&](auto stage_c, bool more) {   // more: another block follows
      constexpr int ST = decltype(stage_c)::value;
      wave_ring_sync();   // this wave is past its reads of the ring slot refilled now
      const int next = kb + kWaves;
      if (more) {
        issue_values(next, std::integral_constant<int, ST ^ 1>{});
        load_keys(next, kv[ST ^ 1]);
        look_up(next + kWaves);
      }
      f32x16_t sc = f32x16_t{};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) sc = mfma_32x32x16(kv[ST][ks], qop[ks], sc);
      float sv[16], ev[16];
      bool masked;
      weights(sc, kb, sv, masked);
#pragma unroll
      for (int i = 0; i < 16; ++i) ev[i] = fast_exp2(fmaf(sv[i], sl2, -m));
      uint4 pb[2];
      operands(ev, pb);
      const char *vd = reinterpret_cast<const char *>(slot(stage_c)) + wave * BLK;
      uint4 va[NTL][2];
#pragma unroll
      for (int i = 0; i < NTL; ++i)
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) va[i][kk] = value_operand(vd, i, kk);
      if (masked) clean_values(va, kb);
#pragma unroll
      for (int i = 0; i < NTL; ++i)
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) acc[i] = mfma_32x32x16(va[i][kk], pb[kk], acc[i]);
      kb = next;
    };
    if (kb < b1) {
      look_up(kb);
      issue_values(kb, std::integral_constant<int, 0>{});
      load_keys(kb, kv[0]);
      look_up(kb + kWaves);
    }
    load_columns();
    if (kb < b1) {
      while (true) {
        step(std::integral_constant<int, 0>{}, kb + kWaves < b1);
        if (kb >= b1) break;
        step(std::integral_constant<int, 1>{}, kb + kWaves < b1);
        if (kb >= b1) break;
      }
    }
  }
  if (__any(left_out)) {   // non-finite elements of closed states, for the columns that see them
    for (int kb = max(b0, nbc); kb < b1; ++kb) {
      const int first = (kb - nbc) * 32;
      if (first + 32 <= lim_lo || (!WIDE && ((kb - b0) & (kWaves - 1)) != wave)) continue;
      add_nonfinite<D, false>(
          acc,
          [&](int i, int e) {
            if constexpr (VT) {
              const uint16_t *v = reinterpret_cast<const uint16_t *>(vclosed + int64_t(first) * RB) + e * 32 + i;
              return make_uint2(v[0] | (uint32_t(v[32]) << 16), v[64] | (uint32_t(v[96]) << 16));
            } else {
              return row4(vclosed + int64_t(first + i) * RB, e);
            }
          },
          [&](int i) { return colv && first + i < lim; }, hb);
    }
  }

  float lt = ls + __shfl_xor(ls, 32, 64);
  if constexpr (!WIDE) {   // the waves' states meet: wave 0 holds the sum
    if (hb == 0) {
      s_m[wave * 32 + col] = m;
      s_l[wave * 32 + col] = lt;
    }
    __syncthreads();   // (and every wave is past its ring)
    float M = s_m[col];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, s_m[w * 32 + col]);
    const float f = fast_exp2(m - M);
    lt = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) lt += s_l[w * 32 + col] * fast_exp2(s_m[w * 32 + col] - M);
    m = M;
#pragma unroll
    for (int i = 0; i < NTL; ++i) acc[i] *= f;
    float *area = reinterpret_cast<float *>(ring0);   // [2][16 NTL][64]
    static_assert(2 * 16 * NTL * 64 * 4 <= SLOT, "merge area");
#pragma unroll
    for (int half = 2; half >= 1; half >>= 1) {
      if (wave >= half && wave < 2 * half) {
#pragma unroll
        for (int i = 0; i < NTL; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) area[((wave - half) * NTL * 16 + i * 16 + r) * 64 + lane] = acc[i][r];
      }
      __syncthreads();
      if (wave < half) {
#pragma unroll
        for (int i = 0; i < NTL; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[i][r] += area[(wave * NTL * 16 + i * 16 + r) * 64 + lane];
      }
      __syncthreads();
    }
    if (wave != 0) return;
  }
  if (!colv) return;
  if (x.parts == 1) {   // lane holds dims 32 i + 8 j + 4 hb .. + 4 of its column
    const float inv = 1.0f / lt;
    char *orow = static_cast<char *>(p.out) + (token * p.os[0] + (x.g * G + head) * p.os[1]) * 2;
#pragma unroll
    for (int i = 0; i < NTL; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t lo = cvt_pk_bf16(acc[i][4 * j] * inv, acc[i][4 * j + 1] * inv);
        const uint32_t hi = cvt_pk_bf16(acc[i][4 * j + 2] * inv, acc[i][4 * j + 3] * inv);
        *reinterpret_cast<uint2 *>(orow + (32 * i + 8 * j + 4 * hb) * 2) = make_uint2(lo, hi);
      }
  } else {
    float *rec = p.partials + (int64_t(x.record) * COLS + (WIDE ? wave * 32 : 0) + col) * (D + 4);
    if (hb == 0) {
      rec[0] = m;
      rec[1] = lt;
    }
#pragma unroll
    for (int i = 0; i < NTL; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<float4 *>(rec + 4 + 32 * i + 8 * j + 4 * hb) =
            make_float4(acc[i][4 * j], acc[i][4 * j + 1], acc[i][4 * j + 2], acc[i][4 * j + 3]);
  }
}

// ---------------------------------------------------------------------------
// fp32, on v_mfma_f32_32x32x2_f32 (operand forms: F32): one tile of 32 columns,
// whose four waves take every fourth block of its piece straight from the pages
// and the closed states; their online-softmax states meet in LDS.  Bound by the
// fp32 matrix rate, and by the chain of blocks of a wave (5 rows of 77 tokens, 12/6
// heads, d 64, on up to 1500 tokens' slots: 22 us).
// ---------------------------------------------------------------------------
template <int D, int G>
__global__ __launch_bounds__(kThreads) void chunk_attend_f32_kernel(ChunkParams p) {
  using F = F32<D>;
  constexpr int T = 32 / G, NT = F::NT, RB = D * 4;
  __shared__ __align__(16) float s_acc[F::kArea];
  __shared__ float s_m[kWaves * 32], s_l[kWaves * 32];
  Piece x;
  if (!find_piece(p, x)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 31, hb = lane >> 5;
  const int a = x.tile << p.tile_shift, cnt = min(T, x.n - a);
  const int tok = col / G;
  const bool colv = tok < cnt;
  const int64_t token = x.start + (colv ? a + tok : 0);
  const int lim = colv ? closed_before(p, x, a + tok) : 0;
  const int top = __builtin_amdgcn_readfirstlane(closed_before(p, x, a + cnt - 1));
  const int lim_lo = cnt == T ? __builtin_amdgcn_readfirstlane(closed_before(p, x, a)) : 0;
  const int vis = visible_slots(p, x.u);
  const int nbc = (vis + 31) >> 5, nb = nbc + ((top + 31) >> 5);
  if (p.fixed_parts > 0) {
    x.parts = fixed_parts_of(p, nb);
    if (x.part >= x.parts) return;
  }
  const int b0 = static_cast<int>(int64_t(nb) * x.part / x.parts);
  const int b1 = static_cast<int>(int64_t(nb) * (x.part + 1) / x.parts);

  auto column = [&](const void *base, const int64_t (&st)[2], int c) {
    return static_cast<const float *>(base) + int64_t(x.start + a + c / G) * st[0] + (x.g * G + c % G) * st[1];
  };
  F::stage(s_acc, [&](int c) -> const float * { return c / G < cnt ? column(p.q, p.qs, c) : nullptr; }, true);
  __syncthreads();
  const float *qs = F::staged(s_acc, lane);
  float m = lowest(), ls = 0.0f;
  f32x16_t acc[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) acc[i] = f32x16_t{};
  if (x.part == x.parts - 1 && wave == ((b1 - b0) & (kWaves - 1))) {   // own states
    const float *ks = reinterpret_cast<const float *>(p.state_k) + (int64_t(x.g) * p.total + token) * D;
    const float *vs = reinterpret_cast<const float *>(p.state_v) + (int64_t(x.g) * p.total + token) * D;
    float d = 0.0f;
#pragma unroll
    for (int j = 0; j < F::NJ; ++j) {
      const typename F::f4_t k4 = *reinterpret_cast<const typename F::f4_t *>(ks + 8 * j + 4 * hb);
      const typename F::f4_t q4 = *reinterpret_cast<const typename F::f4_t *>(qs + 8 * j);
      float part = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) part = fmaf(q4[i], k4[i], part);
      d += part;
    }
    d += __shfl_xor(d, 32, 64);
    if (colv) {
      m = d * p.scale_log2;
      const float w = m == neg_inf() ? 0.0f : 1.0f;   // (-infinity: as in the bf16 kernel)
      if (m == neg_inf()) m = lowest();
      ls = hb == 0 ? w : 0.0f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const typename F::col_t e = *reinterpret_cast<const typename F::col_t *>(vs + NT * F::row(r, hb));
#pragma unroll
        for (int i = 0; i < NT; ++i) acc[i][r] = w * e[i];
      }
    }
  }

  // Lane `col` looks its slot's page up one block ahead; a group of eight slots
  // lies in one page, whose number its first lane holds.
  const int P = 1 << p.log2p;
  const int32_t *pt = p.ptab + int64_t(x.u) * p.maxpages;
  const int64_t closed = (int64_t(x.g) * p.blocks32 + (x.start >> 5) + x.b) * 32;
  const float *kclosed = reinterpret_cast<const float *>(p.closed_k) + closed * D;
  const float *vclosed = reinterpret_cast<const float *>(p.closed_v) + closed * D;
  auto lookup = [&](int kb) { return kb < nbc ? pt[min(kb * 32 + col, vis - 1) >> p.log2p] : 0; };
  typename F::f4_t kr[F::NJ];
  auto load_keys = [&](int kb, int pg) {
    if (kb >= b1) return;
    if (kb < nbc) {
      const int s = min(kb * 32 + col, vis - 1);
      F::load_row(kr, reinterpret_cast<const float *>(p.pool + int64_t(pg) * p.page_bytes + int64_t(s & (P - 1)) * RB), hb);
    } else {
      F::load_row(kr, kclosed + int64_t(min((kb - nbc) * 32 + col, top - 1)) * D, hb);
    }
  };
  auto value_row = [&](int kb, int pg, int i) {
    if (kb >= nbc) return vclosed + int64_t(min((kb - nbc) * 32 + i, top - 1)) * D;
    const int q8 = i & ~7, pq = __builtin_amdgcn_readlane(pg, q8);
    // (slots past the visible ones: rows of the page of the last)
    return reinterpret_cast<const float *>(p.pool + int64_t(pq) * p.page_bytes +
                                           int64_t(P + ((kb * 32 + q8) & (P - 1)) + (i & 7)) * RB);
  };
  int page = lookup(b0 + wave);
  load_keys(b0 + wave, page);
  bool left_out = false;
  auto block = [&](int kb, auto masked_c) {
    constexpr bool MASKED = decltype(masked_c)::value;
    const int next = lookup(kb + kWaves);
    typename F::Cols vc;
    auto vrow = [&](int i) { return value_row(kb, page, i); };
    vc.load(vrow, 0, lane);
    const f32x16_t sc = F::dots(kr, qs);
    load_keys(kb + kWaves, next);
    const int rel = kb < nbc ? vis - kb * 32 : lim - (kb - nbc) * 32;   // rows that the column sees
    float w[16], mx = neg_inf();
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      w[r] = sc[r] * p.scale_log2;
      if (MASKED && F::row(r, hb) >= rel) w[r] = neg_inf();
      mx = fmaxf(mx, w[r]);
    }
    const float mn = fmaxf(m, max_halves(mx));
    const float f = fast_exp2(m - mn);
    m = mn;
    ls *= f;
#pragma unroll
    for (int i = 0; i < NT; ++i) acc[i] *= f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      w[r] = fast_exp2(w[r] - mn);
      ls += w[r];
    }
    left_out |= F::template add_rows<MASKED>(acc, vc, vrow, w, lane);
    page = next;
  };
  auto whole = [&](int kb) { return kb < nbc ? kb * 32 + 32 <= vis : (kb - nbc) * 32 + 32 <= lim_lo; };
#pragma unroll 1
  for (int kb = b0 + wave; kb < b1; kb += kWaves) {
    if (whole(kb)) block(kb, std::false_type{});
    else block(kb, std::true_type{});
  }
  if (__any(left_out)) {
    for (int kb = b0 + wave; kb < b1; kb += kWaves) {
      if (whole(kb)) continue;
      const int pg = lookup(kb), rel = kb < nbc ? vis - kb * 32 : lim - (kb - nbc) * 32;
      F::add_nonfinite(acc, [&](int i) { return value_row(kb, pg, i); }, [&](int i) { return colv && i < rel; }, lane);
    }
  }

  ls += __shfl_xor(ls, 32, 64);
  if (hb == 0) {
    s_m[wave * 32 + col] = m;
    s_l[wave * 32 + col] = ls;
  }
  __syncthreads();
  float M = s_m[col], L = 0.0f;
#pragma unroll
  for (int w = 1; w < kWaves; ++w) M = fmaxf(M, s_m[w * 32 + col]);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) L += s_l[w * 32 + col] * fast_exp2(s_m[w * 32 + col] - M);
  const bool one = x.parts == 1;
  const float f = fast_exp2(m - M) / (one ? L : 1.0f);
#pragma unroll
  for (int i = 0; i < NT; ++i) acc[i] *= f;
  F::put(s_acc, wave, lane, acc);   // (every wave is past its last use of the staged rows)
  float *recs = p.partials + int64_t(x.record) * 32 * (D + 4);
  if (!one && tid < 32 && colv) {
    recs[col * (D + 4)] = M;
    recs[col * (D + 4) + 1] = L;
  }
  __syncthreads();
  for (int i = tid; i < 32 * D / 4; i += kThreads) {
    const int c = i / (D / 4), e = i % (D / 4);
    if (c / G >= cnt) continue;
    float *o = one ? const_cast<float *>(column(p.out, p.os, c)) + 4 * e : recs + c * (D + 4) + 4 + 4 * e;
    *reinterpret_cast<typename F::f4_t *>(o) = F::sum(s_acc, c, e);
  }
}

// Tile `idx` where every row has row_tiles places.
__device__ __forceinline__ PackedTile row_tile(const ChunkParams &p, int idx) {
  PackedTile t;
  t.seq = idx / p.row_tiles;
  t.tile = idx - t.seq * p.row_tiles;
  t.start = clamp_token(p.cu[t.seq], p.total);
  t.n = max(clamp_token(p.cu[t.seq + 1], p.total) - t.start, 0);
  return t;
}

// The pieces of a tile put together: o = sum_i 2^(m_i - M) acc_i / sum_i
// 2^(m_i - M) l_i.  One wave per column, lanes own D / 64 elements; bound by latency:
// records are read sixteen at a time, or four where there are no more (256 wide tiles
// of two pieces: 21 us, 40 with sixteen loads for the two; 24 rows of 32 heads and 6
// tokens: 4.8).  Tiles of one piece have been written already.
template <int ES, int D, int G, int COLS>
__global__ __launch_bounds__(kThreads) void chunk_combine_kernel(ChunkParams p) {
  constexpr int E = D / 64, REC = D + 4;
  const int g = blockIdx.y, lane = threadIdx.x & 63;
  const int c = blockIdx.z * kWaves + (threadIdx.x >> 6);
  const PackedTile pt = p.row_tiles > 0 ? row_tile(p, blockIdx.x)
                                        : packed_tile(p.cu, p.rows, p.total, blockIdx.x, p.tile_shift);
  const int n = min(pt.n, p.max_chunk);
  const int t = (pt.tile << p.tile_shift) + c / G;
  if (pt.tile < 0 || t >= n) return;
  const int u = pt.seq * p.hkv + g;
  int parts, first;
  if (p.fixed_parts > 0) {
    const Piece x{u, pt.seq, g, pt.start, n, 0, 0, 0, 0};
    const int nb = ((visible_slots(p, u) + 31) >> 5) + ((closed_before(p, x, n - 1) + 31) >> 5);
    parts = fixed_parts_of(p, nb);
    first = u * p.fixed_parts;
  } else {
    const int tiles = (n + (1 << p.tile_shift) - 1) >> p.tile_shift;
    parts = p.pieces[u];
    first = p.record_base[u] + (tiles - 1 - pt.tile) * parts;
  }
  parts = __builtin_amdgcn_readfirstlane(parts);
  first = __builtin_amdgcn_readfirstlane(first);
  if (parts == 1) return;
  const float *rec = p.partials + (int64_t(first) * COLS + c) * REC;
  float M = lowest(), L = 0.0f, A[E];
#pragma unroll
  for (int e = 0; e < E; ++e) A[e] = 0.0f;
  auto of_lane = [](float y, int j) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, y), j));
  };
  auto batch = [&](int i0, auto r_c) {
    constexpr int R = decltype(r_c)::value;
    // lane i < R reads record i's maximum and sum; every load of a batch in one round trip
    const float *mine = rec + int64_t(min(i0 + (lane & (R - 1)), parts - 1)) * COLS * REC;
    float mi = mine[0], li = mine[1], a[R][E];
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const float *r = rec + int64_t(min(i0 + j, parts - 1)) * COLS * REC + 4 + lane * E;
#pragma unroll
      for (int e = 0; e < E; ++e) a[j][e] = r[e];
    }
    if (i0 + (lane & (R - 1)) >= parts) {   // (the last record again: without weight)
      mi = lowest();
      li = 0.0f;
    }
    float mn = M;
#pragma unroll
    for (int j = 0; j < R; ++j) mn = fmaxf(mn, of_lane(mi, j));
    const float f = fast_exp2(M - mn), w = i0 + (lane & (R - 1)) < parts ? fast_exp2(mi - mn) : 0.0f;
    M = mn;
    L *= f;
#pragma unroll
    for (int e = 0; e < E; ++e) A[e] *= f;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const float wj = of_lane(w, j);
      if (i0 + j < parts) {
        L = fmaf(wj, of_lane(li, j), L);
#pragma unroll
        for (int e = 0; e < E; ++e) A[e] = fmaf(wj, a[j][e], A[e]);
      }
    }
  };
  if (parts <= 4) batch(0, std::integral_constant<int, 4>{});
  else
    for (int i0 = 0; i0 < parts; i0 += 16) batch(i0, std::integral_constant<int, 16>{});
  const float inv = 1.0f / L;
#pragma unroll
  for (int e = 0; e < E; ++e) A[e] *= inv;
  store_e<ES, E>(static_cast<char *>(p.out) +
                     (int64_t(pt.start + t) * p.os[0] + (g * G + c % G) * p.os[1] + lane * E) * ES, A);
}

template <int ES, int D, bool VT>
hipError_t chunk_states(const ChunkParams &p, hipStream_t s) {
  if (p.max_chunk > kBlock)
    hipLaunchKernelGGL((chunk_states_kernel<ES, D, VT, SUMS>), dim3(p.blocks64, p.hkv), dim3(kStateThreads), 0, s, p);
  const int plan = p.fixed_parts > 0 ? 0 : 1;   // the workgroup that plans
  hipLaunchKernelGGL((chunk_states_kernel<ES, D, VT, ATTEND>), dim3(p.blocks64 + plan, p.hkv), dim3(kStateThreads), 0, s, p);
  return hipGetLastError();
}

template <int D, int G, bool VT, bool BIG>
void attend_bf16(const ChunkParams &p, bool wide, unsigned pieces, hipStream_t s) {
  if (wide)
    hipLaunchKernelGGL((chunk_attend_kernel<D, G, VT, BIG, true>), dim3(pieces), dim3(kThreads), 0, s, p);
  else
    hipLaunchKernelGGL((chunk_attend_kernel<D, G, VT, BIG, false>), dim3(pieces), dim3(kThreads), 0, s, p);
}

template <int ES, int D, int G>
hipError_t chunk_attend(ChunkParams p, bool vt, bool wide, hipStream_t s) {
  hipError_t e = vt ? chunk_states<ES, D, (ES == 2 && G >= 4)>(p, s) : chunk_states<ES, D, false>(p, s);
  if (e != hipSuccess) return e;
  // Tiles by the tensors' length, or by the longest rows where that makes less than half of them: a buffer may be
  // far longer than the rows' tokens.  us by length -> by rows: 1 row of 4 tokens, 16/4 heads, 900 slots, in 1M rows
  // 944 -> 56; 16 rows of 4, 64/8 heads, 8000 slots, in 64K rows 457 -> 68; but 4 rows of 512 in 2048, where the
  // packed count leaves an XCD more spare places, 476 -> 481.
  const int64_t row_tiles = (int64_t(std::min(p.max_chunk, p.total)) + (1 << p.tile_shift) - 1) >> p.tile_shift;
  const int64_t packed = int64_t(p.total >> p.tile_shift) + p.rows;
  p.row_tiles = 2 * row_tiles * p.rows <= packed ? static_cast<int32_t>(row_tiles) : 0;
  const unsigned tiles = static_cast<unsigned>(p.row_tiles > 0 ? row_tiles * p.rows : packed);
  const unsigned pieces = p.fixed_parts > 0 ? unsigned(p.units) * p.fixed_parts
                                            : (tiles * p.hkv + p.piece_budget + 7) / 8 * 8;
  if constexpr (ES == 2) {
    if (vt) {
      if constexpr (G >= 4) attend_bf16<D, G, true, true>(p, wide, pieces, s);
    } else if (p.log2p >= 5) {
      attend_bf16<D, G, false, true>(p, wide, pieces, s);
    } else {
      attend_bf16<D, G, false, false>(p, wide, pieces, s);
    }
  } else {
    hipLaunchKernelGGL((chunk_attend_f32_kernel<D, G>), dim3(pieces), dim3(kThreads), 0, s, p);
  }
  e = hipGetLastError();
  if (e != hipSuccess || (p.fixed_parts <= 1 && p.piece_budget == 0)) return e;   // every tile is whole
  if (wide)
    hipLaunchKernelGGL((chunk_combine_kernel<ES, D, G, 128>), dim3(tiles, p.hkv, 128 / kWaves), dim3(kThreads), 0, s, p);
  else
    hipLaunchKernelGGL((chunk_combine_kernel<ES, D, G, 32>), dim3(tiles, p.hkv, 32 / kWaves), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

template <int ES, int D>
hipError_t attend_by_group(int group, const ChunkParams &p, bool vt, bool wide, hipStream_t s) {
  switch (group) {
    case 1: return chunk_attend<ES, D, 1>(p, vt, wide, s);
    case 2: return chunk_attend<ES, D, 2>(p, vt, wide, s);
    case 4: return chunk_attend<ES, D, 4>(p, vt, wide, s);
    case 8: return chunk_attend<ES, D, 8>(p, vt, wide, s);
    default: return hipErrorInvalidValue;
  }
}

template <int ES, int D, bool VT>
hipError_t chunk_append(const ChunkParams &p, hipStream_t s) {
  const dim3 grid(p.blocks64, p.hkv), threads(kStateThreads);
  if (p.max_chunk <= kBlock) {
    hipLaunchKernelGGL((chunk_states_kernel<ES, D, VT, ONE>), grid, threads, 0, s, p);
  } else {
    hipLaunchKernelGGL((chunk_states_kernel<ES, D, VT, SUMS>), grid, threads, 0, s, p);
    hipLaunchKernelGGL(chunk_grow_kernel, dim3((p.units + kWaves - 1) / kWaves), dim3(kThreads), 0, s, p);
    hipLaunchKernelGGL((chunk_states_kernel<ES, D, VT, APPEND>), grid, threads, 0, s, p);
  }
  return hipGetLastError();
}

}  // namespace

// Wide tiles read a cache once for four times as many columns, narrow ones leave
// more workgroups for a small one.  us of the attention and its combine pass (32/8
// heads, d 128), narrow / wide, by the layer's cached slots and max_chunk * G:
//              16K       32K       64K     8 x 8K     512K
//    40       18/20       -         -         -       69/62
//    64       18/21     20/22     27/24     28/24     77/65
//   128       20/25     28/28     39/32     39/31    107/85
//   256       29/28       -         -         -      197/143
// (Lengths are on the device: by what the caches can hold.  A cache that is nearly
// empty loses the few us of its own column.)
bool chunk_wide(int elem_bytes, int group, int max_chunk, int64_t slots) {
  return elem_bytes == 2 && max_chunk * int64_t(group) > (slots >= (1 << 16) ? 32 : 128);
}

int chunk_tile_shift(int group, bool wide) {
  int shift = wide ? 7 : 5;
  for (; group > 1; group >>= 1) --shift;
  return shift;
}

hipError_t launch_chunk_attend(int elem_bytes, int head_dim, int group, bool vt, bool wide, const ChunkParams &p,
                               hipStream_t s) {
  if (elem_bytes == 2)
    return head_dim == 128 ? attend_by_group<2, 128>(group, p, vt, wide, s) : attend_by_group<2, 64>(group, p, vt, wide, s);
  return head_dim == 128 ? attend_by_group<4, 128>(group, p, vt, wide, s) : attend_by_group<4, 64>(group, p, vt, wide, s);
}

hipError_t launch_chunk_append(int elem_bytes, int head_dim, bool vt, const ChunkParams &p, hipStream_t s) {
  if (elem_bytes == 4) return head_dim == 128 ? chunk_append<4, 128, false>(p, s) : chunk_append<4, 64, false>(p, s);
  if (vt) return head_dim == 128 ? chunk_append<2, 128, true>(p, s) : chunk_append<2, 64, true>(p, s);
  return head_dim == 128 ? chunk_append<2, 128, false>(p, s) : chunk_append<2, 64, false>(p, s);
}

}  // namespace dmc
