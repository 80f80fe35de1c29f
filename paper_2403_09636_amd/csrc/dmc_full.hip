// gfx950 kernels of layers that keep their full cache: the position rotation of
// packed queries and keys (and its gradients), the append of rotated keys and
// values to a paged cache, and the attention of new tokens over it (Sec. 2.1 of
// the DMC paper: softmax of q.k/sqrt(d), every element, no compression).
//
// Row b of the cache holds n = lengths[b] tokens and gets m new ones (one, or
// the tokens cu[b] .. cu[b + 1] - 1) at the positions n .. n + m - 1; token p lies
// in slot p mod P of page table[b][p / P] of the pools [page][kv head][P][d].
#include <algorithm>
#include <type_traits>

#include "dmc_full.h"
#include "dmc_mfma.h"

namespace dmc {
namespace {

constexpr float kLn2 = 0.6931471805599453f;

enum : int32_t { kRowFull = FLAG_SLOTS_EXHAUSTED, kBadRows = FLAG_BAD_LENGTH, kBadPage = FLAG_BAD_PAGE };

__device__ __forceinline__ void raise(int32_t *flags, int32_t bits) {
  if (flags) atomicOr(flags, bits);
}

// What a call does with row b: its tokens start at `start`, the first `m` of them
// (of `given`) have a place behind the n cached ones.
struct FullRow {
  int start, given, n, m;
};
__device__ __forceinline__ FullRow full_row(const int32_t *cu, const int32_t *len, int total, int capacity, int b) {
  FullRow r;
  r.start = cu ? clamp_token(cu[b], total) : b;
  r.given = cu ? max(clamp_token(cu[b + 1], total) - r.start, 0) : 1;
  const int n = len[b];
  r.n = min(n, capacity);
  r.m = n < 0 ? 0 : min(r.given, capacity - r.n);
  return r;
}
// The flags of row b's boundaries and length.
__device__ __forceinline__ int32_t row_flags(const int32_t *cu, const int32_t *len, int total, int capacity, int b,
                                             int max_chunk) {
  const int lo = cu ? cu[b] : b, hi = cu ? cu[b + 1] : b + 1;
  int32_t f = 0;
  if (lo < 0 || hi > total || hi < lo || len[b] > capacity || (hi > lo && hi - lo > max_chunk)) f |= kBadRows;
  const FullRow r = full_row(cu, len, total, capacity, b);
  if (r.n >= 0 && r.m < r.given) f |= kRowFull;
  return f;
}

// The row that holds token t: the last one that starts at or before it (64
// candidates a step, by the whole wave).
__device__ __forceinline__ int row_of_token(const int32_t *cu, int rows, int total, int t) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = rows;   // the answer lies in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 63) >> 6, i = lo + lane * step;
    const bool le = lane == 0 || (i < lo + n && clamp_token(cu[i], total) <= t);
    const int k = 63 - __clzll(static_cast<long long>(__ballot(le)));
    const int end = lo + n;
    lo += k * step;
    n = min(step, end - lo);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// ---------------------------------------------------------------------------
// Rotation and append.  A workgroup takes one token: its first wave forms the cosines
// and sines of the pairs (in 64 bits up to the fraction of a turn), which every head
// uses from LDS; then each thread moves units of two 16-byte vectors of a head, the
// two halves of 16 / ES pairs (or 16 / ES adjacent pairs), in grid.y shares of the
// token's units.  Bound by HBM, each element read and written once: 6 sequences of up to
// 4096 tokens, 32 + 32 heads of 128 in bf16, take 88 us (5.9 TB/s of reads and writes), in
// append 148.  Four tokens to a workgroup: 102 and 157 us; four units of a thread in flight
// at once, with fewer waves (not taken): 2048 tokens 28.6 us against 24.7.  The rotation's stores
// stream (without: 91 us; the causal attention that reads them next takes the same time
// after either), the append's do not (with: 157 us).
// ---------------------------------------------------------------------------
// A store that cannot be to LDS (from pointers of several origins the compiler makes
// flat stores, which count as LDS accesses too).
template <bool STREAM>
__device__ __forceinline__ void store_global(char *p, const uint4 &v) {
  typedef __attribute__((address_space(1))) u32x4 gv;
  gv *at = reinterpret_cast<gv *>(reinterpret_cast<uintptr_t>(p));
  if constexpr (STREAM) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), at);
  else *at = __builtin_bit_cast(u32x4, v);
}

template <int ES, int D, bool PAGED>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotateParams p) {
  constexpr int N = 16 / ES, UPR = D * ES / 32;   // elements of a vector, units of a row
  __shared__ __align__(16) float cosv[64], sinv[64];
  __shared__ int64_t place;   // element offset of the token's slot of kv head 0 (-1: none)
  __shared__ int state;       // 0: no token of a row, 1: here, 2: dropped
  const int tid = threadIdx.x, lane = tid & 63;
  if constexpr (PAGED) {
    if (blockIdx.x == gridDim.x - 1) {   // the rows' boundaries and lengths
      if (blockIdx.y == 0 && p.flags) {
        int32_t f = 0;
        for (int b = tid; b < p.rows; b += kThreads) f |= row_flags(p.cu, p.len, p.total, p.capacity, b, 0x7fffffff);
        if (f) raise(p.flags, f);
      }
      return;
    }
  }
  const int64_t t = blockIdx.x;
  if (tid < 64) {
    int pos, st = 1;
    int64_t at = -1;
    if constexpr (PAGED) {
      const int b = p.cu ? row_of_token(p.cu, p.rows, p.total, blockIdx.x) : blockIdx.x;
      const FullRow r = full_row(p.cu, p.len, p.total, p.capacity, b);
      const int i = static_cast<int>(blockIdx.x) - r.start;
      pos = r.n + i;
      st = i < 0 || i >= r.given ? 0 : i < r.m ? 1 : 2;
      if (st == 1) {
        const int page = p.table[int64_t(b) * p.max_pages + (pos >> p.log2p)];
        if (static_cast<uint32_t>(page) < static_cast<uint32_t>(p.num_pages))
          at = (((int64_t(page) * p.hkv) << p.log2p) + (pos & ((1 << p.log2p) - 1))) * D;
        else if (lane == 0 && blockIdx.y == 0)
          raise(p.flags, kBadPage);
      }
    } else {
      pos = p.positions[t];
    }
    if (lane == 0) {
      place = at;
      state = st;
    }
    if (lane < p.r / 2) {
      // turns: the product and its fraction in 64 bits; cosine and sine at the fraction in 32
      // bits, then turned by what those leave out (at most 2^-26 turns)
      const double turns = pos * (double(p.inv_freq[lane]) * 0.15915494309189533577);
      const double part = turns - rint(turns);
      const float near = static_cast<float>(part);
      const float rest = static_cast<float>(part - near) * 6.2831853071795864769f;
      float s, c;
      sincospif(2.0f * near, &s, &c);
      cosv[lane] = fmaf(-s, rest, c);
      sinv[lane] = p.inverse ? -fmaf(c, rest, s) : fmaf(c, rest, s);
    }
  }
  __syncthreads();

  const int st = PAGED ? state : 1;
  if (st == 0) return;
  const int units = (p.hq + (PAGED ? 2 : 1) * p.hkv) * UPR;
  const int rv2 = p.r * ES / 32;   // rotated units of a row
  for (int idx = blockIdx.y * kThreads + tid; idx < units; idx += kThreads * gridDim.y) {
    const int u = idx % UPR, row = idx / UPR;
    const bool is_q = row < p.hq, is_v = PAGED && row >= p.hq + p.hkv;
    const bool turned = u < rv2 && !is_v && st == 1;
    int v0 = 2 * u, gap = 16;   // first vector; bytes to the second one
    if (u < rv2 && !is_v && p.halves) {
      v0 = u;
      gap = rv2 * 16;
    }
    const char *src;
    char *dst;
    if (is_q) {
      src = static_cast<const char *>(p.q) + (t * p.qs[0] + row * p.qs[1]) * ES;
      dst = static_cast<char *>(p.qo) + (t * p.qos[0] + row * p.qos[1]) * ES + v0 * 16;
    } else {
      const int h = row - p.hq - (is_v ? p.hkv : 0);
      src = is_v ? static_cast<const char *>(p.v) + (t * p.vs[0] + h * p.vs[1]) * ES
                 : static_cast<const char *>(p.k) + (t * p.ks[0] + h * p.ks[1]) * ES;
      if constexpr (PAGED) {
        if (place < 0) continue;
        dst = (is_v ? p.vp : p.kp) + (place + ((int64_t(h) * D) << p.log2p)) * ES + v0 * 16;
      } else {
        dst = static_cast<char *>(p.ko) + (t * p.kos[0] + h * p.kos[1]) * ES + v0 * 16;
      }
    }
    uint4 x = make_uint4(0, 0, 0, 0), y = x;   // (a dropped token's queries: zeros)
    if (st == 1) {
      x = ld16(src + v0 * 16);
      y = ld16(src + v0 * 16 + gap);
    }
    if (turned) {
      float a[N], b[N], c[N], s[N];
      V16<ES>::unpack(x, a);
      V16<ES>::unpack(y, b);
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        *reinterpret_cast<f32x4_t *>(c + i) = *reinterpret_cast<const f32x4_t *>(cosv + u * N + i);
        *reinterpret_cast<f32x4_t *>(s + i) = *reinterpret_cast<const f32x4_t *>(sinv + u * N + i);
      }
      if (p.halves) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float xa = a[i], xb = b[i];
          a[i] = xa * c[i] - xb * s[i];
          b[i] = xa * s[i] + xb * c[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
          const float xa = a[2 * i], xb = a[2 * i + 1], ya = b[2 * i], yb = b[2 * i + 1];
          a[2 * i] = xa * c[i] - xb * s[i];
          a[2 * i + 1] = xa * s[i] + xb * c[i];
          b[2 * i] = ya * c[N / 2 + i] - yb * s[N / 2 + i];
          b[2 * i + 1] = ya * s[N / 2 + i] + yb * c[N / 2 + i];
        }
      }
      x = V16<ES>::pack(a);
      y = V16<ES>::pack(b);
    }
    store_global<!PAGED>(dst, x);
    store_global<!PAGED>(dst + gap, y);
  }
}

// ---------------------------------------------------------------------------
// Attention: how the work is shared out.  A unit is one column tile (query
// columns: the pairs of a new token and a head of one kv head's group) of one row
// and kv head; it takes as many keys as its row holds (or its last token sees).
// Units are cut into pieces of keys, in ranges, one to a workgroup:
//   - few units and keys (latency counts): every unit in equal pieces (one, where there
//     are about as many units as workgroups), one piece to a workgroup;
//   - else the units of all rows lie one after another in a space of keys, row by
//     row, which is cut into equal ranges; a block of keys belongs to the range that
//     its first key lies in.  A range may hold several pieces.
// A unit in one piece goes straight to the output.  Else every piece leaves a
// record (running maximum, sum and accumulator), to be joined in the order of the
// keys: o = sum_i 2^(m_i - M) acc_i / sum_i 2^(m_i - M) l_i.  That is done by the
// workgroup that finishes a unit's last piece (a counter tells) where the caches'
// capacity is small (full_one_launch), else by a second launch, since the counting and
// the writes through to memory cost more than a launch there.
// ---------------------------------------------------------------------------

// A wave-uniform value, made visibly so (SGPRs).
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
  const uint32_t lo = uniform(static_cast<int>(x)), hi = uniform(static_cast<int>(x >> 32));
  return static_cast<int64_t>((uint64_t(hi) << 32) | lo);
}

// Sums over the wave's lanes up to each (row_shr 1, 2, 4, 8, row_bcast 15, 31: no LDS).
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}

// Workgroup i runs on XCD i mod 8: each XCD takes one run of ranges, so that the
// tiles of a kv head read its keys through one L2.
__device__ __forceinline__ int range_of_block(int blocks) {
  return (blocks & 7) ? static_cast<int>(blockIdx.x) : (blockIdx.x & 7) * (blocks >> 3) + (blockIdx.x >> 3);
}

// Rows of out and lse of tokens that are dropped (their row is not in use, or full): `dropped`
// tokens from `first` on, a token and head at a time, shared out among `parts` workgroups of
// which this is number `part`; LANES threads of each take part, this one being `lane`.
// 8192 tokens of 64 heads: 24.7 us, by one workgroup 5225; 4 rows of 512 tokens on 4000, one of
// them not in use: 255.5 us (as with one token in that row), by one workgroup 578.
template <int ES, int D, int LANES>
__device__ __forceinline__ void clear_dropped(const FullParams &p, int first, int dropped, uint32_t part, uint32_t parts,
                                              uint32_t lane) {
  constexpr int VPR = D * ES / 16, STEP = LANES / VPR;   // vectors of a row; rows of a workgroup at a time
  const uint32_t items = uint32_t(dropped) * p.hq;       // (up to 2^30)
  for (uint32_t x = part * STEP + lane / VPR; x < items; x += parts * STEP) {
    const uint32_t i = x / uint32_t(p.hq), h = x - i * p.hq, v = lane % VPR;
    const int64_t t = int64_t(first) + i;
    st16(static_cast<char *>(p.out) + (t * p.os[0] + h * p.os[1]) * ES + v * 16, make_uint4(0, 0, 0, 0));
    if (p.lse && v == 0) p.lse[t * p.hq + h] = neg_inf();
  }
}
// The part that this workgroup takes of row b's dropped tokens, where all of them share these.
__device__ __forceinline__ uint32_t part_of_row(int b) { return (blockIdx.x + gridDim.x - b % gridDim.x) % gridDim.x; }
// Dropped items (tokens times heads) of a row up to which one workgroup alone writes them.
// In batches of up to 64 rows every workgroup knows the rows, and takes a few cycles for each
// one that is shared (32 of 64 rows not in use, 64 heads: steps 41.1 us, shared 44.1; 4 tokens
// a row 43.3, shared 46.6; 8 tokens 47.5 and 50.2).  In larger ones it has to look for those
// with more (200 rows, one with 200, 600 and 2000 dropped tokens of 8 heads: alone 27.8, 61.6
// and 184 us, shared 28.3, 28.3 and 28.4; 4096 rows: 218 us without such a row, 231 with one).
constexpr int kAloneFew = 512, kAloneMany = 2048;

// A page id of the table, page 0 where the table names none.
__device__ __forceinline__ int checked_page(const FullParams &p, int page) {
  if (static_cast<uint32_t>(page) < static_cast<uint32_t>(p.num_pages)) return page;
  raise(p.flags, kBadPage);
  return 0;
}
// An entry of the page table at a wave-uniform index, by a scalar load (nothing
// writes the table while a kernel runs): it does not queue behind vector loads.
__device__ __forceinline__ int table_entry(const int32_t *table, int i) {
  typedef const __attribute__((address_space(4))) int32_t const_i32_t;
  return reinterpret_cast<const_i32_t *>(reinterpret_cast<uintptr_t>(table))[__builtin_amdgcn_readfirstlane(i)];
}

// Fewest keys of a piece: shorter ones cost more in records than they gain.  Narrow
// tiles (each wave takes a fourth of the keys; 16/4 heads of 128 in bf16, one row of 900
// keys): 64 14.0 us, 128 11.3, 256 11.6; 5 rows of up to 1500, fp32: 17.2, 15.0, 19.6.
// fp32 chunks, whose waves take every key (64 tokens on 500, 4 rows of 8/4 heads of
// 128): 32 26.4 us, 64 27.8, 128 35.5; 256 in an empty cache: 28.7, 27.0, 34.5.  Wide
// tiles (64 tokens on 16000, 32/8 heads): 256 46.2 us, 512 46.5, 1024 68.4; 4 rows of
// 512 tokens on 12000, 64/8 heads: 862, 855, 858.
// kEqualKeys: the keys per workgroup up to which units are cut equally where there are
// at least 4 workgroups to a unit, half of it where there are fewer (then the ranges
// fill the chip better).  64 tokens on 16000: 46.5 us, with 256 58.8; 8 rows of 8 tokens
// on 4000, 32 heads: 90 us, with 4096 144.  Units that are not cut (60 rows of up to 500
// keys, 8 kv heads): 20.2 us, in ranges 27.6; the rule's edge, 40 rows of up to 1000:
// 33.7 us against 30.4.
constexpr int kNarrowRange = 128, kChunkRange = 64, kWideRange = 512, kEqualKeys = 1024;

// a / G for a < 2^31, by a multiplication (G = 1: group_shift < 0).
__device__ __forceinline__ int div_group(const FullParams &p, int a) {
  return p.group_shift < 0 ? a : static_cast<int>(__umulhi(static_cast<uint32_t>(a), p.group_magic) >> p.group_shift);
}
// a / b for a < 2^22, b > 0 (a tenth of a microsecond less than the general division).
__device__ __forceinline__ int small_div(int a, int b) {
  int q = static_cast<int>(static_cast<float>(a) * __builtin_amdgcn_rcpf(static_cast<float>(b)));
  const int r = a - q * b;
  q += r >= b ? 1 : r < 0 ? -1 : 0;
  return uniform(q);
}

// How the columns of a row and kv head are cut into tiles.  A row of m new tokens
// at n ..:
//   whole rows (TRI false): tiles of `cols` columns, each over all n + m keys;
//   TRI: tiles of `per` = cols / G whole tokens, tile t over the keys that its last
//     token sees, n + min(m, (t + 1) per); the keys of the tiles before tile t are
//     t n + per t (t + 1) / 2.
template <bool TRI>
struct Tiles {
  int n, m, count, step;   // step: tokens of a tile (TRI) or its columns
  __device__ __forceinline__ Tiles(int n_, int m_, int G, int cols, int tokens) : n(n_), m(m_) {
    step = TRI ? tokens : cols;
    const int all = TRI ? m : m * G;
    count = all <= step ? 1 : (all + step - 1) / step;
  }
  __device__ __forceinline__ int keys(int t) const { return TRI ? n + min(m, (t + 1) * step) : n + m; }
  __device__ __forceinline__ int64_t before(int t) const {
    return TRI ? int64_t(t) * n + int64_t(step) * t * (t + 1) / 2 : int64_t(t) * (n + m);
  }
  __device__ __forceinline__ int64_t all() const { return m > 0 ? before(count - 1) + keys(count - 1) : 0; }
  // The tile that holds key `off` of the row's and head's space.
  __device__ __forceinline__ int at(int64_t off) const {
    int lo = 0, hi = count;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (before(mid) <= off) lo = mid;
      else hi = mid;
    }
    return lo;
  }
  __device__ __forceinline__ int first_col(int t, int G) const { return TRI ? t * step * G : t * step; }
};

typedef FullPiece Piece;

// The rows and their shares of the work.  Up to 64 rows: every wave loads them all,
// one to a lane, and keeps its own copy in LDS (no barrier, and no second load of a
// row when a piece of it is taken); else sums before every row in LDS
// (prefix[rows + 1]).
struct RowPlace {
  int64_t before;   // keys (or ranges) of the rows before it
  int32_t start, n, m, pieces;
};
struct SpaceLds {
  RowPlace rows[kWaves][64];
  int64_t sums[kWaves];
  int32_t many[kWaves];
};
template <int ES, int D, bool TRI, int LEAST>   // LEAST: fewest keys of a piece
struct Space {
  const FullParams &p;
  int64_t *prefix;
  RowPlace *places;
  int64_t all, per, pos, hi;   // pos, hi: what is left of this workgroup's range
  int G, range;
  bool few, equal;             // equal: equal pieces of every unit

  __device__ __forceinline__ Tiles<TRI> tiles(int n, int m) const { return Tiles<TRI>(n, m, G, p.tile_cols, p.tile_tokens); }
  __device__ __forceinline__ FullRow load(int i) const { return full_row(p.cu, p.len, p.total, p.capacity, i); }

  // Sums up the rows; writes the rows of dropped tokens, and in the first workgroup
  // the flags of what it finds wrong.
  __device__ __forceinline__ Space(const FullParams &p_, int64_t *prefix_, SpaceLds &lds)
      : p(p_), prefix(prefix_), G(p_.hq / p_.hkv), range(range_of_block(gridDim.x)), few(p_.rows <= 64), equal(false) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int grid = gridDim.x;
    places = lds.rows[wave];
    if (few) {
      FullRow row{0, 0, 0, 0};
      if (lane < p.rows) row = load(lane);
      const int m = min(row.m, p.max_chunk), keys = row.n + m;
      const Tiles<TRI> t = tiles(row.n, m);
      // (capped, so that 64 of them stay below 2^31: more is more than kEqualKeys)
      const int units = m > 0 ? static_cast<int>(min(int64_t(p.hkv) * t.count, int64_t(1) << 24)) : 0;
      const int count = __builtin_amdgcn_readlane(wave_scan(units), 63);
      const int sum = __builtin_amdgcn_readlane(wave_scan(static_cast<int>(min(int64_t(units) * keys, int64_t(1) << 24))), 63);
      equal = count <= grid && sum <= (4 * count <= grid ? kEqualKeys : kEqualKeys / 2) * grid;
      int64_t share, x;
      int pieces = 0;
      if (equal) {
        const int each = max(small_div(sum, max(grid - count, 1)) + 1, LEAST);
        pieces = (keys + each - 1) / each;
        share = units * pieces;
        x = wave_scan(units * pieces);
      } else {
        share = m > 0 ? p.hkv * t.all() : int64_t(0);
        x = share;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const int64_t y = __shfl_up(x, o, 64);
          if (lane >= o) x += y;
        }
      }
      all = uniform(__shfl(x, 63, 64));
      places[lane] = RowPlace{x - share, row.start, row.n, m, pieces};
      wave_lds_sync();
      if (__any(row.m < row.given)) {   // (never in lanes past the rows)
        const int items = (row.given - row.m) * p.hq;
        static_assert(kFullPlaces >= 64, "a workgroup for every row");
        const unsigned long long alone = __ballot(items > 0 && items <= kAloneFew);
        unsigned long long dropped = __ballot(items > kAloneFew);
        if (blockIdx.x < 64 && (alone >> blockIdx.x & 1)) {
          const FullRow r = load(blockIdx.x);
          clear_dropped<ES, D, kThreads>(p, r.start + r.m, r.given - r.m, 0, 1, tid);
        }
        while (dropped) {
          const int i = __ffsll(dropped) - 1;
          dropped &= dropped - 1;
          clear_dropped<ES, D, kThreads>(p, __builtin_amdgcn_readlane(row.start + row.m, i),
                                         __builtin_amdgcn_readlane(row.given - row.m, i), part_of_row(i), grid, tid);
        }
      }
      if (blockIdx.x == 0 && wave == 0 && lane < p.rows && p.flags) {
        const int32_t f = row_flags(p.cu, p.len, p.total, p.capacity, lane, p.max_chunk);
        if (f) raise(p.flags, f);
      }
    } else {
      const int each = (p.rows + kThreads - 1) / kThreads, b0 = min(tid * each, p.rows), b1 = min(b0 + each, p.rows);
      int64_t own = 0;
      bool many = false;   // a row with many dropped tokens
      for (int i = b0; i < b1; ++i) {
        prefix[i] = own;
        const FullRow r = load(i);
        const int m = min(r.m, p.max_chunk);
        many |= (r.given - r.m) * p.hq > kAloneMany;
        if (m > 0) own += p.hkv * tiles(r.n, m).all();
        if (blockIdx.x == 0 && p.flags) {
          const int32_t f = row_flags(p.cu, p.len, p.total, p.capacity, i, p.max_chunk);
          if (f) raise(p.flags, f);
        }
      }
      int64_t x = own;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int64_t y = __shfl_up(x, o, 64);
        if (lane >= o) x += y;
      }
      many = __any(many);
      if (lane == 63) {
        lds.sums[wave] = x;
        lds.many[wave] = many;
      }
      __syncthreads();
      int64_t first = x - own;
      all = 0;
      many = false;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        if (i < wave) first += lds.sums[i];
        all += lds.sums[i];
        many |= lds.many[i] != 0;
      }
      for (int i = b0; i < b1; ++i) prefix[i] += first;
      if (tid == 0) prefix[p.rows] = all;
      __syncthreads();
      for (int i = blockIdx.x; i < p.rows; i += grid) {
        const FullRow r = load(i);
        if (r.m < r.given && (r.given - r.m) * p.hq <= kAloneMany)
          clear_dropped<ES, D, kThreads>(p, r.start + r.m, r.given - r.m, 0, 1, tid);
      }
      for (int base = wave * 64; many && base < p.rows; base += kThreads) {   // each wave for itself
        FullRow r{0, 0, 0, 0};
        if (base + lane < p.rows) r = load(base + lane);
        unsigned long long dropped = __ballot((r.given - r.m) * p.hq > kAloneMany);
        while (dropped) {
          const int i = __ffsll(dropped) - 1;
          dropped &= dropped - 1;
          clear_dropped<ES, D, 64>(p, __builtin_amdgcn_readlane(r.start + r.m, i), __builtin_amdgcn_readlane(r.given - r.m, i),
                                   part_of_row(base + i), grid, lane);
        }
      }
    }
    all = uniform(all);
    per = equal ? 1 : max((all + grid - 1) / grid, int64_t(LEAST));
    pos = boundary(range);
    hi = boundary(range + 1);
  }

  // A range's end that lies within kSnap keys of a unit's end moves there: a cut unit
  // costs two records and their join, as much as some hundred keys (32 rows of 200 keys,
  // 32 heads: 20.7 us, without 34.4; 4 prompts of up to 2048 tokens, 32/8 heads, wide:
  // 138 us, without 152; fp32 chunks with 512 in place of 128, 2 rows of 1000 tokens:
  // 149 us against 86).
  static constexpr int kSnap = TRI && ES == 2 ? 512 : 128;
  __device__ __forceinline__ int64_t boundary(int i) {
    const int64_t v = min(i * per, all);
    if (equal || v == 0 || v == all) return v;
    const Unit u = unit_at(v);
    return v - u.begin <= kSnap ? u.begin : u.begin + u.keys - v <= kSnap ? u.begin + u.keys : v;
  }

  // The unit that holds key (or range) v of the space: tile t of a row and head.
  struct Unit {
    int b, n, start, m, pieces, h, t, keys, index;   // index: piece (equal pieces)
    int64_t begin;                                   // its first key (not of equal pieces)
  };
  __device__ __forceinline__ Unit unit_at(int64_t v) {
    Unit u;
    int64_t off;
    u.pieces = 0;
    if (few) {
      const RowPlace mine = places[threadIdx.x & 63];
      u.b = 63 - __clzll(static_cast<long long>(__ballot(mine.m > 0 && mine.before <= v)));
      const RowPlace r = places[u.b];
      u.n = uniform(r.n);
      u.start = uniform(r.start);
      u.m = uniform(r.m);
      u.pieces = uniform(r.pieces);
      off = v - uniform(r.before);
    } else {
      int lo = 0, end = p.rows;   // prefix[lo] <= v < prefix[end]
      while (end - lo > 1) {
        const int mid = (lo + end) >> 1;
        if (prefix[mid] <= v) lo = mid;
        else end = mid;
      }
      u.b = uniform(lo);
      const FullRow r = load(u.b);
      u.n = uniform(r.n);
      u.start = uniform(r.start);
      u.m = min(uniform(r.m), p.max_chunk);
      off = v - uniform(prefix[u.b]);
    }
    const Tiles<TRI> ts = tiles(u.n, u.m);
    if (equal) {
      const int o = static_cast<int>(off), unit = small_div(o, u.pieces);
      u.index = o - unit * u.pieces;
      u.h = small_div(unit, ts.count);
      u.t = unit - u.h * ts.count;
    } else {
      const int64_t per_head = ts.all();
      u.h = uniform(static_cast<int>(off / per_head));
      const int64_t in_head = off - u.h * per_head;
      u.t = uniform(ts.at(in_head));
      u.begin = v - in_head + ts.before(u.t);
    }
    u.keys = ts.keys(u.t);
    return u;
  }

  // The next piece of the range; pos moves behind it.
  __device__ __forceinline__ Piece next() {
    const Unit u = unit_at(pos);
    Piece x;
    x.b = u.b;
    x.n = u.n;
    x.start = u.start;
    x.h = u.h;
    x.keys = u.keys;
    if (equal) {
      x.pieces = u.pieces;
      x.index = u.index;
      x.first = range - x.index;
      const int size = (small_div(x.keys + x.pieces - 1, x.pieces) + 31) & ~31;
      x.k0 = min(x.index * size, x.keys);
      x.k1 = min(x.k0 + size, x.keys);
      pos = hi;
    } else {
      x.k0 = static_cast<int>(pos - u.begin);
      x.k1 = static_cast<int>(min(int64_t(x.keys), x.k0 + (hi - pos)));
      // ranges that end within the unit: at i per in (begin + kSnap, begin + keys - kSnap)
      x.first = static_cast<int>((u.begin + min(kSnap, x.keys - 1)) / per);
      x.pieces = max(static_cast<int>((u.begin + x.keys - kSnap - 1) / per) - x.first, 0) + 1;
      x.index = range - x.first;
      pos += x.k1 - x.k0;
    }
    const Tiles<TRI> ts = tiles(u.n, u.m);
    x.col0 = ts.first_col(u.t, G);
    x.cols = min(TRI ? ts.step * G : ts.step, u.m * G - x.col0);
    return x;
  }
};

// A record: [D / 2][tile columns] pairs of the accumulator's elements, then [tile
// columns] (running maximum, sum): a wave, whose lanes hold different columns, writes
// and reads whole lines.
// The record of a piece: that of a unit that started in an earlier range in its
// range's first place, that of one that goes on in the next range in the second.
__device__ __forceinline__ int record_index(int first, int index) { return 2 * (first + index) + (index == 0 ? 1 : 0); }
__device__ __forceinline__ float *record_of(const FullParams &p, int first, int index) {
  return p.partials + record_index(first, index) * p.record_floats;
}

// E floats to E elements in memory, rounded to nearest even.
template <int ES, int E>
__device__ __forceinline__ void store_out(char *dst, const float *f) {
  if constexpr (ES == 4) {
#pragma unroll
    for (int i = 0; i < E; i += 4) *reinterpret_cast<f32x4_t *>(dst + 4 * i) = *reinterpret_cast<const f32x4_t *>(f + i);
  } else if constexpr (E == 8) {
    st16(dst, make_uint4(cvt_pk_bf16(f[0], f[1]), cvt_pk_bf16(f[2], f[3]), cvt_pk_bf16(f[4], f[5]),
                         cvt_pk_bf16(f[6], f[7])));
  } else {
    *reinterpret_cast<uint2 *>(dst) = make_uint2(cvt_pk_bf16(f[0], f[1]), cvt_pk_bf16(f[2], f[3]));
  }
}

// In one launch records go between workgroups of different XCDs, whose L2 caches are
// not kept coherent: they are written through, 8 bytes at a time (relaxed atomics of
// the agent's scope), and read with plain loads after an acquire fence, which only
// the workgroup that joins makes.
__device__ __forceinline__ void put2(const FullParams &q, float *p, float a, float b) {
  if (q.one_launch) {
    const uint64_t x = (uint64_t(__float_as_uint(b)) << 32) | __float_as_uint(a);
    __hip_atomic_store(reinterpret_cast<uint64_t *>(p), x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  } else {
    *reinterpret_cast<float2 *>(p) = make_float2(a, b);
  }
}

// Joins records from, from + step .. (`count` >= 2 of them) of a unit: into the first
// of them, or the output.  The statistics of all columns and records first (to LDS,
// as weights), then the accumulators, two columns' pairs (16 bytes) AT_ONCE times to a
// thread, all of a step's reads in flight together.  Columns begin (even) .. end - 1.
constexpr int kJoinPairs = 1024;
static_assert(kJoinPairs >= 2 * kFullPlaces, "a step takes two columns of every record");
template <int ES, int D, int AT_ONCE>
__device__ __forceinline__ void join_records(const FullParams &p, const Piece &x, int begin, int end, int from, int step,
                                             int count, bool last, float2 *w) {
  const int tid = threadIdx.x, G = p.hq / p.hkv, most = (kJoinPairs / count) & ~1, tc = p.tile_cols;
  float *into = record_of(p, x.first, from);
  for (int c0 = begin; c0 < end; c0 += most) {
    const int cols = min(most, end - c0), halves = (cols + 1) >> 1;   // (a record's columns are an even number)
    const int64_t stats = int64_t(tc) * D + 2 * c0;
    __syncthreads();
    for (int i = tid; i < cols * count; i += kThreads) {
      const int col = i / count;
      w[i] = *reinterpret_cast<const float2 *>(record_of(p, x.first, from + (i - col * count) * step) + stats + 2 * col);
    }
    __syncthreads();
    if (tid < cols) {
      float2 *c = w + tid * count;
      float top = c[0].x, sum = 0.0f;
      for (int i = 1; i < count; ++i) top = fmaxf(top, c[i].x);
      for (int i = 0; i < count; ++i) {
        c[i].x = fast_exp2(c[i].x - top);
        sum = fmaf(c[i].y, c[i].x, sum);
      }
      c[0].y = sum;
      const int i = div_group(p, x.col0 + c0 + tid), head = x.h * G + (x.col0 + c0 + tid) - i * G;
      if (!last) put2(p, into + stats + 2 * tid, top, sum);
      else if (p.lse) p.lse[int64_t(x.start + i) * p.hq + head] = (top + __log2f(sum)) * kLn2;
    }
    __syncthreads();
    // item: two columns' pair number e2
    for (int base = tid; base < halves * (D / 2); base += AT_ONCE * kThreads) {
      f32x4_t o[AT_ONCE] = {};
      int e2[AT_ONCE], ca[AT_ONCE], cb[AT_ONCE];
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) {
        const int item = min(base + k * kThreads, halves * (D / 2) - 1);
        e2[k] = (halves & (halves - 1)) == 0 ? item >> (31 - __clz(halves)) : item / halves;
        ca[k] = 2 * (item - e2[k] * halves);
        cb[k] = min(ca[k] + 1, cols - 1);
      }
#pragma unroll 4
      for (int i = 0; i < count; ++i) {
        const float *r = record_of(p, x.first, from + i * step) + 2 * c0;
        f32x4_t a[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) a[k] = *reinterpret_cast<const f32x4_t *>(r + 2 * (e2[k] * tc + ca[k]));
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
          const float fa = w[ca[k] * count + i].x, fb = w[cb[k] * count + i].x;
          o[k][0] = fmaf(a[k][0], fa, o[k][0]);
          o[k][1] = fmaf(a[k][1], fa, o[k][1]);
          o[k][2] = fmaf(a[k][2], fb, o[k][2]);
          o[k][3] = fmaf(a[k][3], fb, o[k][3]);
        }
      }
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) {
        if (base + k * kThreads >= halves * (D / 2)) break;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int cc = ca[k] + u;
          if (cc >= cols) break;
          if (last) {
            const int col = x.col0 + c0 + cc, i = div_group(p, col), head = x.h * G + col - i * G;
            const float inv = 1.0f / w[cc * count].y, a = o[k][2 * u] * inv, b = o[k][2 * u + 1] * inv;
            char *dst = static_cast<char *>(p.out) + (int64_t(x.start + i) * p.os[0] + head * p.os[1] + 2 * e2[k]) * ES;
            if constexpr (ES == 2) *reinterpret_cast<uint32_t *>(dst) = cvt_pk_bf16(a, b);
            else *reinterpret_cast<float2 *>(dst) = make_float2(a, b);
          } else {
            put2(p, into + 2 * (e2[k] * tc + c0 + cc), o[k][2 * u], o[k][2 * u + 1]);
          }
        }
      }
    }
  }
}

// The cut units of a workgroup's range, at most two (one that started in an earlier
// range, one that goes on in the next).
struct Cuts {
  Piece piece[2];
  int last[2], n;
};

// Joins what is complete once the workgroup's records are written: each wave's
// stores have arrived before the barrier lets it through (vmcnt 0), and the last
// workgroup to count reads only after it has counted; it leaves the counter at 0.
// Counting at the end of the range, not after each piece, keeps the wait out of the
// stream of keys.  Only tiles of 16 and 32 columns are joined so (JOIN); wider ones always
// take two launches.  More than kJoin pieces are joined in groups of kJoin first, so
// that no workgroup reads more than a few dozen records (a row of 100000 keys, 8/1 heads:
// groups of 8 36.2 us, 16 30.5, 32 31.6; 30000, 64/8 heads: 33.7, 34.6, 38.2).  Counters: one per record for
// the groups that start with it, one per range for the unit that starts in it.
constexpr int kJoin = 16;
__device__ __forceinline__ int count_up(int32_t *counter, int count) {
  const int before = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  if (before == count - 1) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return before == count - 1;
}
template <int ES, int D, bool JOIN>
__device__ __forceinline__ void join_cuts(const FullParams &p, Cuts &cuts, void *lds) {
  if (!JOIN || !p.one_launch) {
    if (threadIdx.x == 0) {
      Piece *unit = p.cut_units + range_of_block(gridDim.x);   // the one that starts here and goes on
      if (cuts.n > 0 && cuts.piece[cuts.n - 1].index == 0) *unit = cuts.piece[cuts.n - 1];
      else unit->pieces = 0;
    }
    return;
  }
  if constexpr (JOIN) {
    float2 *w = static_cast<float2 *>(lds);
    wait_vmcnt<0>();
    __syncthreads();
    const int n = uniform(cuts.n);
    if (n == 0) return;
    auto unit_counter = [&](const Piece &x) { return p.counters + 2 * p.places + x.first; };
    if (threadIdx.x < n) {
      const Piece &x = cuts.piece[threadIdx.x];
      const int from = x.index / kJoin * kJoin;
      cuts.last[threadIdx.x] = x.pieces > kJoin ? count_up(p.counters + record_index(x.first, from), min(kJoin, x.pieces - from))
                                                : count_up(unit_counter(x), x.pieces);
    }
    __syncthreads();
    for (int i = 0; i < n; ++i) {
      if (!uniform(cuts.last[i])) continue;
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
      const Piece x = cuts.piece[i];
      if (x.pieces <= kJoin) {
        join_records<ES, D, 4>(p, x, 0, x.cols, 0, 1, x.pieces, true, w);
        continue;
      }
      const int from = x.index / kJoin * kJoin, groups = (x.pieces + kJoin - 1) / kJoin;
      const int members = min(kJoin, x.pieces - from);
      if (members > 1) join_records<ES, D, 4>(p, x, 0, x.cols, from, 1, members, false, w);
      wait_vmcnt<0>();
      __syncthreads();
      if (threadIdx.x == 0) cuts.last[i] = count_up(unit_counter(x), groups);
      __syncthreads();
      if (!uniform(cuts.last[i])) continue;
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
      join_records<ES, D, 4>(p, x, 0, x.cols, 0, kJoin, groups, true, w);
    }
  }
}

// The second launch: a workgroup per range (one unit at most starts in it and goes
// on) and `step` columns; 5 to 6 us beside 144 of the first (16 rows of up to 24000).
// Steps of 32 columns in place of 8: drafts of 4 tokens 72.1 us against 68.7.
template <int ES, int D>
__global__ __launch_bounds__(kThreads) void full_join_kernel(FullParams p, int step) {
  __shared__ float2 w[kJoinPairs];
  const Piece x = p.cut_units[blockIdx.x];
  const int begin = blockIdx.y * step;
  if (x.pieces < 2 || begin >= x.cols) return;
  join_records<ES, D, 1>(p, x, begin, min(begin + step, x.cols), 0, 1, x.pieces, true, w);
}

// ---------------------------------------------------------------------------
// Tiles of 16 and 32 columns in registers: decode steps, drafts, all of fp32.
// Bound by HBM: keys and values go from memory straight into the operands of the
// 16x16 matrix instructions, without LDS (each is used by one wave only).  48 rows of
// 4095 keys, 32 heads of 128: 483 us, 6.7 TB/s; 16 rows of up to 24000, 64/8 heads: 144
// us, 6.2 TB/s.  Short rows are bound by latency: one row of 900, 16/4 heads: 10.8 us.
// Blocks of 16 U keys; with lane l = 16 g +
// c (g < 4, c < 16):
//   S[key][col] = K Q^T: lane rows are keys 16 u + c, and its slices of the head dim
//     any 16 bytes, as long as Q's are the same; the result's registers hold keys
//     16 u + 4 g + r (r < 4) of column c;
//   O[dim][col] += V^T P^T: those 4 U probabilities are the operand as they are if the
//     contraction's index 4 U g + 4 u + r means key 16 u + 4 g + r: lane l loads E =
//     d / 16 elements, dims E c .. + E, of those keys, and one permutation per two
//     elements makes of them the E operands whose row c is dim E c + j (fp32: loaded
//     values are the operands).
// In bf16, P enters as the sum of two bf16 terms (what is left of 32 bits costs no
// time here), and l is the sum of its 32-bit values.
// SPLIT_KEYS: a tile is 16 NT columns and each wave takes every fourth block;
// otherwise (fp32 chunks, bound by the matrix cores) it is four times as many, each
// wave taking 16 NT of them over every block, which the four read through one L1.
// No variant spills registers (fp32 at d = 128 takes blocks of 16 keys and 16
// columns for that).
// ---------------------------------------------------------------------------
// Loads through pointers of the global address space: from generic ones the compiler
// makes flat loads, which count as LDS accesses too, so that every wait for one of
// those (or for a scalar load) waits for all keys and values in flight.
typedef const __attribute__((address_space(1))) char gchar;
template <typename V, bool STREAM>
__device__ __forceinline__ V load_global(gchar *p) {
  typedef const __attribute__((address_space(1))) V gv;
  if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<gv *>(p));
  else return *reinterpret_cast<gv *>(p);
}
// A wave-uniform address (SGPRs).
__device__ __forceinline__ gchar *uniform_global(const char *p) {
  return reinterpret_cast<gchar *>(reinterpret_cast<uintptr_t>(uniform_ptr(p)));
}

template <int ES, int D>
struct Narrow;

template <int D>
struct Narrow<2, D> {
  static constexpr int E = D / 16, KC = D / 32;   // elements of a value slice; 16-byte slices of a key row
  typedef unsigned int vrow_t __attribute__((ext_vector_type(E / 2)));
  static constexpr int U = 2;
  struct Keys { uint4 x[U][KC]; };
  struct Values { vrow_t x[4 * U]; };
  struct Query { uint4 x[KC]; };
  static constexpr int kKeyStep = 64;             // bytes between a lane's slices of a row
  __device__ static __forceinline__ int key_offset(int g) { return g * 16; }
  template <bool STREAM>
  __device__ static __forceinline__ void load_row(uint4 (&x)[KC], gchar *row) {
#pragma unroll
    for (int c = 0; c < KC; ++c) x[c] = __builtin_bit_cast(uint4, load_global<u32x4, STREAM>(row + c * kKeyStep));
  }
  template <bool STREAM>
  __device__ static __forceinline__ vrow_t load_value(gchar *p) {
    return load_global<vrow_t, STREAM>(p);
  }
  __device__ static __forceinline__ f32x4_t scores(const uint4 (&k)[KC], const Query &q) {
    f32x4_t s = f32x4_t{};
#pragma unroll
    for (int c = 0; c < KC; ++c) s = mfma_16x16x32(k[c], q.x[c], s);
    return s;
  }
  // Operand j of the value product: dim E c + j of the lane's eight keys.
  __device__ static __forceinline__ uint4 operand(const Values &v, int j) {
    const uint32_t sel = (j & 1) ? 0x07060302u : 0x05040100u;
    return make_uint4(__builtin_amdgcn_perm(v.x[1][j / 2], v.x[0][j / 2], sel),
                      __builtin_amdgcn_perm(v.x[3][j / 2], v.x[2][j / 2], sel),
                      __builtin_amdgcn_perm(v.x[5][j / 2], v.x[4][j / 2], sel),
                      __builtin_amdgcn_perm(v.x[7][j / 2], v.x[6][j / 2], sel));
  }
  // Values that are not finite are left out of every block's products (0 times
  // them, and their product with the second term of P, would be NaN) and reported.
  __device__ static __forceinline__ bool leave_out(Values &v, bool) {
    float acc = 0.0f;
    const bf16x2_t zero = __builtin_bit_cast(bf16x2_t, 0u);
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < E / 2; ++j) {
        const uint32_t w = v.x[i][j];   // (a bit cast of the vector's element itself takes element 0)
        acc = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w), zero, acc, false);
      }
    if (!__any(acc != 0.0f)) return false;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < E / 2; ++j) v.x[i][j] &= finite_halves(v.x[i][j]);
    return true;
  }
  template <int NT>
  __device__ static __forceinline__ void add(f32x4_t (&acc)[NT][E], const float (&p)[NT][8], const Values &v) {
    uint4 hi[NT], lo[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      uint32_t h[4], l[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        h[i] = cvt_pk_bf16(p[t][2 * i], p[t][2 * i + 1]);
        l[i] = cvt_pk_bf16(p[t][2 * i] - bf16_lo(h[i]), p[t][2 * i + 1] - bf16_hi(h[i]));
      }
      hi[t] = make_uint4(h[0], h[1], h[2], h[3]);
      lo[t] = make_uint4(l[0], l[1], l[2], l[3]);
    }
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const uint4 a = operand(v, j);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        acc[t][j] = mfma_16x16x32(a, hi[t], acc[t][j]);
        acc[t][j] = mfma_16x16x32(a, lo[t], acc[t][j]);
      }
    }
  }
};

template <int D>
struct Narrow<4, D> {
  static constexpr int E = D / 16, KC = D / 16;
  typedef float vrow_t __attribute__((ext_vector_type(E)));
  static constexpr int U = D == 128 ? 1 : 2;
  struct Keys { f32x4_t x[U][KC]; };
  struct Values { vrow_t x[4 * U]; };
  struct Query { f32x4_t x[KC]; };
  static constexpr int kKeyStep = 64;
  __device__ static __forceinline__ int key_offset(int g) { return g * 16; }
  template <bool STREAM>
  __device__ static __forceinline__ void load_row(f32x4_t (&x)[KC], gchar *row) {
#pragma unroll
    for (int c = 0; c < KC; ++c) x[c] = load_global<f32x4_t, STREAM>(row + c * kKeyStep);
  }
  template <bool STREAM>
  __device__ static __forceinline__ vrow_t load_value(gchar *p) {
    vrow_t v;
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
      const f32x4_t x = load_global<f32x4_t, STREAM>(p + 16 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * i + e] = x[e];
    }
    return v;
  }
  __device__ static __forceinline__ f32x4_t mfma(float a, float b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
  }
  // (in chains of 16 elements added up: one long chain rounds more)
  __device__ static __forceinline__ f32x4_t scores(const f32x4_t (&k)[KC], const Query &q) {
    f32x4_t s = f32x4_t{};
#pragma unroll
    for (int c = 0; c < KC; c += 2) {
      f32x4_t x = f32x4_t{}, y = f32x4_t{};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x = mfma(k[c][e], q.x[c][e], x);
        y = mfma(k[c + 1][e], q.x[c + 1][e], y);
      }
      s += x + y;
    }
    return s;
  }
  // Needed only where some column does not see a key of the block.
  __device__ static __forceinline__ bool leave_out(Values &v, bool masked) {
    if (!masked) return false;
    bool some = false;
#pragma unroll
    for (int i = 0; i < 4 * U; ++i)
#pragma unroll
      for (int j = 0; j < E; ++j) some |= !is_finite(v.x[i][j]);
    if (!__any(some)) return false;
#pragma unroll
    for (int i = 0; i < 4 * U; ++i)
#pragma unroll
      for (int j = 0; j < E; ++j) v.x[i][j] = is_finite(v.x[i][j]) ? v.x[i][j] : 0.0f;
    return true;
  }
  template <int NT>
  __device__ static __forceinline__ void add(f32x4_t (&acc)[NT][E], const float (&p)[NT][4 * U], const Values &v) {
#pragma unroll
    for (int i = 0; i < 4 * U; ++i)
#pragma unroll
      for (int j = 0; j < E; ++j)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[t][j] = mfma(v.x[i][j], p[t][i], acc[t][j]);
  }
};

// SMALL: pages of fewer tokens than a block.
template <int ES, int D, int NT, bool SMALL, bool SPLIT_KEYS>
__global__ __launch_bounds__(kThreads, 2) void full_narrow_kernel(FullParams p) {
  using X = Narrow<ES, D>;
  constexpr int E = X::E, U = X::U, KEYS = 16 * U, RB = D * ES, JS = D + 4, STEP = SPLIT_KEYS ? kWaves : 1;
  constexpr int COLS = 16 * NT * (SPLIT_KEYS ? 1 : kWaves);
  constexpr bool TRI = !SPLIT_KEYS;
  // Keys are read in 64-byte parts of a line: with 32 columns plain loads are faster
  // (drafts of 4 tokens on 8192, 64/8 heads: 68.7 us, streamed 71.9), with 16 slower (16
  // rows of up to 24000, 64/8 heads: 154.5 us, streamed 147.5).
  constexpr bool STREAM_KEYS = SPLIT_KEYS && NT == 1;
  extern __shared__ int64_t prefix[];
  __shared__ SpaceLds space_lds;
  __shared__ Cuts cuts;
  __shared__ __align__(16) float area[SPLIT_KEYS ? kWaves : 1][SPLIT_KEYS ? 16 : 1][JS];   // (all of SPLIT_KEYS)
  __shared__ float stat[kWaves][16][2];
  const int tid = threadIdx.x, lane = tid & 63, c16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = p.hq / p.hkv;

  Space<ES, D, TRI, SPLIT_KEYS ? kNarrowRange : kChunkRange> space(p, prefix, space_lds);
  if (tid == 0) cuts.n = 0;
  while (space.pos < space.hi) {
    const Piece x = space.next();
    const int col0 = x.col0 + (SPLIT_KEYS ? 0 : wave * 16 * NT), cols = min(16 * NT, x.col0 + x.cols - col0);   // this wave's
    // Keys that this wave's columns see, and the last key that they all do.
    const int keys = SPLIT_KEYS ? x.keys : cols > 0 ? x.n + div_group(p, col0 + cols - 1) + 1 : 0;
    const int full_end = x.n + div_group(p, col0);

    typename X::Query q[NT];
    int lim[NT];   // the last key that this lane's column sees
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int c = t * 16 + c16;
      const int i = div_group(p, col0 + c), head = x.h * G + (col0 + c) - i * G;
      lim[t] = x.n + i;
      if (c < cols) {
        const char *src = static_cast<const char *>(p.q) + (int64_t(x.start + i) * p.qs[0] + head * p.qs[1]) * ES +
                          X::key_offset(g4);
#pragma unroll
        for (int k = 0; k < X::KC; ++k)
          q[t].x[k] = *reinterpret_cast<const std::remove_reference_t<decltype(q[t].x[k])> *>(src + k * X::kKeyStep);
      } else {
#pragma unroll
        for (int k = 0; k < X::KC; ++k) q[t].x[k] = {};
      }
    }

    const int32_t *table = p.table + int64_t(x.b) * p.max_pages;
    const int kb1 = (min(x.k1, keys) + KEYS - 1) / KEYS;
    // Pages of a block: the block's, or those of this lane's keys and values.
    struct Pages { int x[SMALL ? 2 * U : 1]; };
    auto pages_of = [&](int kb) {
      Pages pg;
      if constexpr (SMALL) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          pg.x[u] = table[min(kb * KEYS + u * 16 + c16, keys - 1) >> p.log2p];
          pg.x[U + u] = table[min(kb * KEYS + u * 16 + g4 * 4, keys - 1) >> p.log2p];
        }
      } else {
        pg.x[0] = table_entry(table, min(kb * KEYS, keys - 1) >> p.log2p);
      }
      return pg;
    };
    const int mask = (1 << p.log2p) - 1;
    // First byte of kv head h's rows in a page.
    auto page_at = [&](const char *pool, int page) {
      return reinterpret_cast<gchar *>(reinterpret_cast<uintptr_t>(pool)) +
             ((int64_t(checked_page(p, page)) * p.hkv + x.h) << p.log2p) * RB;
    };
    auto block_at = [&](const char *pool, int page, int kb) {   // of a block that lies in one page
      return uniform_global(pool + ((int64_t(checked_page(p, page)) * p.hkv + x.h) << p.log2p) * RB +
                            int64_t((kb * KEYS) & mask) * RB);
    };
    typename X::Keys kx;
    typename X::Values vx;
    auto load_keys = [&](int kb, const Pages &pg) {
      if constexpr (SMALL) {
#pragma unroll
        for (int u = 0; u < U; ++u)
          X::template load_row<STREAM_KEYS>(kx.x[u], page_at(p.kp, pg.x[u]) +
              (min(kb * KEYS + u * 16 + c16, keys - 1) & mask) * RB + X::key_offset(g4));
      } else {
        gchar *at = block_at(p.kp, pg.x[0], kb);
        const uint32_t last = keys - 1 - kb * KEYS;
#pragma unroll
        for (int u = 0; u < U; ++u)
          X::template load_row<STREAM_KEYS>(kx.x[u], at + (min(uint32_t(u * 16 + c16), last) * RB + X::key_offset(g4)));
      }
    };
    auto load_values = [&](int kb, const Pages &pg) {
      if constexpr (SMALL) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          gchar *at = page_at(p.vp, pg.x[U + u]) + c16 * (E * ES);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            vx.x[u * 4 + i] = X::template load_value<SPLIT_KEYS>(
                at + (min(kb * KEYS + u * 16 + g4 * 4 + i, keys - 1) & mask) * RB);
        }
      } else {
        gchar *at = block_at(p.vp, pg.x[0], kb);
        const uint32_t last = keys - 1 - kb * KEYS;
#pragma unroll
        for (int i = 0; i < 4 * U; ++i)
          vx.x[i] = X::template load_value<SPLIT_KEYS>(
              at + (min(uint32_t((i >> 2) * 16 + g4 * 4 + (i & 3)), last) * RB + c16 * (E * ES)));
      }
    };

    // (the lowest finite value: no score may lie below the running maximum's start)
    float mx[NT], ls[NT];
    f32x4_t acc[NT][E];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      mx[t] = lowest();
      ls[t] = 0.0f;
#pragma unroll
      for (int j = 0; j < E; ++j) acc[t][j] = f32x4_t{};
    }
    int kb = (x.k0 + KEYS - 1) / KEYS + (SPLIT_KEYS ? wave : 0);
    if (kb < kb1) {
      Pages next = pages_of(kb);
      load_keys(kb, next);
      load_values(kb, next);
      next = pages_of(min(kb + STEP, kb1 - 1));
      for (; kb < kb1; kb += STEP) {
        float pr[NT][4 * U];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const f32x4_t s = X::scores(kx.x[u], q[t]);
#pragma unroll
            for (int r = 0; r < 4; ++r) pr[t][4 * u + r] = s[r];
          }
        const bool more = kb + STEP < kb1;
        const Pages cur = next;
        if (more) {
          next = pages_of(min(kb + 2 * STEP, kb1 - 1));
          load_keys(kb + STEP, cur);
        }
        const bool masked = kb * KEYS + KEYS - 1 > full_end;
        if (masked) {
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4 * U; ++i)
              if (kb * KEYS + (i >> 2) * 16 + g4 * 4 + (i & 3) > lim[t]) pr[t][i] = neg_inf();
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          float top = fmaxf(fmaxf(pr[t][0], pr[t][1]), fmaxf(pr[t][2], pr[t][3]));
          if constexpr (U == 2) top = fmaxf(top, fmaxf(fmaxf(pr[t][4], pr[t][5]), fmaxf(pr[t][6], pr[t][7])));
          top = max_halves(max_rows16(top)) * p.scale_log2;
          // (only the columns that need it: no column's bits depend on another's)
          const bool grown = top > mx[t] + kLazyRescale;
          if (__any(grown)) {
            const float mn = grown ? top : mx[t], f = fast_exp2(mx[t] - mn);
            mx[t] = mn;
            ls[t] *= f;
#pragma unroll
            for (int j = 0; j < E; ++j) acc[t][j] *= f;
          }
#pragma unroll
          for (int i = 0; i < 4 * U; ++i) {
            pr[t][i] = fast_exp2(fmaf(pr[t][i], p.scale_log2, -mx[t]));
            ls[t] += pr[t][i];
          }
        }
        const bool left_out = X::leave_out(vx, masked);
        X::template add<NT>(acc, pr, vx);
        if (left_out) {   // to the columns that see them, with any positive weight
#pragma unroll 1
          for (int i = 0; i < KEYS; ++i) {
            const int key = kb * KEYS + i;
            if (key >= keys) break;
            const char *row = p.vp + (((int64_t(checked_page(p, table_entry(table, key >> p.log2p))) * p.hkv + x.h) << p.log2p) +
                                      (key & mask)) * RB;
#pragma unroll
            for (int rj = 0; rj < 4 * E; ++rj) {
              const float f = load_elem<ES>(row, g4 * 4 * E + rj);
#pragma unroll
              for (int t = 0; t < NT; ++t)
                if (key <= lim[t] && !is_finite(f)) acc[t][rj % E][rj / E] += f;
            }
          }
        }
        if (more) load_values(kb + STEP, cur);
      }
    }

    const bool whole = x.pieces == 1;
    float *rec = record_of(p, x.first, x.index);
    // E elements e0 .. of a column of the tile to the output.
    auto put = [&](int col, int e0, float top, float sum, float (&o)[E]) {
      const int i = div_group(p, x.col0 + col), head = x.h * G + (x.col0 + col) - i * G;
      const int64_t token = x.start + i;
      const float inv = 1.0f / sum;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] *= inv;
      store_out<ES, E>(static_cast<char *>(p.out) + (token * p.os[0] + head * p.os[1] + e0) * ES, o);
      if (p.lse && e0 == 0) p.lse[token * p.hq + head] = (top + __log2f(sum)) * kLn2;
    };
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float l = ls[t] + __shfl_xor(ls[t], 16, 64);
      l += __shfl_xor(l, 32, 64);
      if constexpr (SPLIT_KEYS) {   // the four waves' parts: E elements of a column to a thread
        __syncthreads();
        if (g4 == 0) {
          stat[wave][c16][0] = mx[t];
          stat[wave][c16][1] = l;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int j = 0; j < E; j += 4)
            *reinterpret_cast<f32x4_t *>(&area[wave][c16][(g4 * 4 + r) * E + j]) =
                f32x4_t{acc[t][j][r], acc[t][j + 1][r], acc[t][j + 2][r], acc[t][j + 3][r]};
        __syncthreads();
        // to the output 16 threads take a column, to a record 16 columns' pairs
        const int c = whole ? tid >> 4 : tid & 15, part = whole ? tid & 15 : tid >> 4, col = t * 16 + c;
        if (col < x.cols) {
          float top = stat[0][c][0];
#pragma unroll
          for (int w = 1; w < kWaves; ++w) top = fmaxf(top, stat[w][c][0]);
          float sum = 0.0f, f[kWaves];
#pragma unroll
          for (int w = 0; w < kWaves; ++w) {
            f[w] = fast_exp2(stat[w][c][0] - top);
            sum = fmaf(stat[w][c][1], f[w], sum);
          }
          if (whole) {
            float o[E] = {};
#pragma unroll
            for (int w = 0; w < kWaves; ++w)
#pragma unroll
              for (int e = 0; e < E; ++e) o[e] = fmaf(area[w][c][part * E + e], f[w], o[e]);
            put(col, part * E, top, sum, o);
          } else {
#pragma unroll
            for (int k = 0; k < E / 2; ++k) {
              const int e2 = k * 16 + part;
              float a = 0.0f, bb = 0.0f;
#pragma unroll
              for (int w = 0; w < kWaves; ++w) {
                a = fmaf(area[w][c][2 * e2], f[w], a);
                bb = fmaf(area[w][c][2 * e2 + 1], f[w], bb);
              }
              put2(p, rec + 2 * (e2 * COLS + col), a, bb);
            }
            if (part == 0) put2(p, rec + COLS * D + 2 * col, top, sum);
          }
        }
      } else if (t * 16 + c16 < cols) {
        const int col = wave * 16 * NT + t * 16 + c16;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int e0 = (g4 * 4 + r) * E;
          float o[E];
#pragma unroll
          for (int j = 0; j < E; ++j) o[j] = acc[t][j][r];
          if (whole) {
            put(col, e0, mx[t], l, o);
          } else {
#pragma unroll
            for (int j = 0; j < E; j += 2)
              *reinterpret_cast<float2 *>(rec + 2 * ((e0 + j) / 2 * COLS + col)) = make_float2(o[j], o[j + 1]);
            if (e0 == 0) *reinterpret_cast<float2 *>(rec + COLS * D + 2 * col) = make_float2(mx[t], l);
          }
        }
      }
    }
    if (!whole && tid == 0) cuts.piece[cuts.n++] = x;
  }
  static_assert(!SPLIT_KEYS || sizeof(area) >= kJoinPairs * sizeof(float2), "join area");
  join_cuts<ES, D, SPLIT_KEYS>(p, cuts, area);
}

// ---------------------------------------------------------------------------
// Wide tiles (128 columns, bf16): pieces of prompts, turns, long drafts.  Bound by
// the matrix cores and the vector work of the softmax beside them (busy 48 % and 43 % of
// the cycles, which share the issue slots): 4 rows of 512 tokens on 12000, 64/8 heads,
// take 855 to 925 us (cards differ), 890 to 960 TFLOP/s, 77 to 84 % of a large product's.  One workgroup =
// 4 waves, a wave owning 32 columns (lane l: column l % 32, half l / 32), so that
// all heads of a kv head's group share its keys.  Keys and values stream through LDS
// in blocks of 32 (direct global -> LDS transfers, a ring of four blocks, three
// ahead), from whichever pages hold them: the rows of one transfer instruction (4
// or 8) lie in one page, whose id comes by a scalar load one block earlier.
//   S^T[key][col] = K . Q^T;   O^T[dim][col] += V^T P^T
// Score row m is key pi(m) (bits 2 and 3 of m swapped), which makes a lane's score
// registers the operand of the second product.  Block kb's exponentials run between
// the score products of block kb + 1.
// ---------------------------------------------------------------------------
constexpr int kWideCols = 128;

template <int D>
__global__ __launch_bounds__(kThreads, 2) void full_wide_kernel(FullParams p) {
  constexpr int kSt = 4;               // ring slots
  constexpr int KS = D / 16, NTL = D / 32, RB = D * 2, CPR = D / 8, BLK = 32 * RB;
  constexpr int DPW = BLK / 16 / kThreads, RPI = 64 / CPR;   // transfers of a wave per block; rows of one
  static_assert(DPW >= 1 && BLK % (16 * kThreads) == 0 && RPI <= 8, "block split");
  static_assert(KS == 2 * NTL && KS > 3, "one transposed operand per score product");
  __shared__ __align__(16) unsigned char ring0[2 * BLK], ring1[2 * BLK], ring2[2 * BLK], ring3[2 * BLK];
  auto slot = [&](auto st_c) -> unsigned char * {
    constexpr int S = decltype(st_c)::value;
    if constexpr (S == 0) return ring0;
    else if constexpr (S == 1) return ring1;
    else if constexpr (S == 2) return ring2;
    else return ring3;
  };
  extern __shared__ int64_t prefix[];
  __shared__ SpaceLds space_lds;
  __shared__ Cuts cuts;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, hb = lane >> 5;
  const int G = p.hq / p.hkv;
  Space<2, D, true, kWideRange> space(p, prefix, space_lds);
  const float sl2 = p.scale_log2;
  const int mask = (1 << p.log2p) - 1;

  // This lane's part of a transfer: row within the instruction's rows, and the
  // chunk that its LDS place holds.
  uint32_t kchunk[DPW], vchunk[DPW];
  const int lrow = lane / CPR;
#pragma unroll
  for (int i = 0; i < DPW; ++i) {
    const int row = (i * kWaves + wave) * RPI + lrow, pc = lane - lrow * CPR;
    kchunk[i] = (pc ^ block_swizzle<CPR, 0>(row)) * 16;
    vchunk[i] = (pc ^ block_swizzle<CPR, 1>(row)) * 16;
  }
  const int krow_s = score_slot(col);
  uint32_t kaddr[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) kaddr[ks] = row_offset<D, 0>(krow_s, ks, hb);
  uint32_t traddr[NTL][2];
  tr_offsets<D, 1>(lane, traddr);

  if (tid == 0) cuts.n = 0;
  while (space.pos < space.hi) {
    const Piece x = space.next();
    const int c = wave * 32 + col, ti = div_group(p, x.col0 + c), head = x.h * G + (x.col0 + c) - ti * G;
    const bool colv = c < x.cols;
    const int64_t token = x.start + ti;
    const int lim = x.n + ti;   // the last key that this column sees
    const int blk0 = (x.k0 + 31) >> 5, nblk = (x.k1 + 31) >> 5;
    // Keys < wave_hi feed this wave, those up to full_end all of its columns.
    const int wcols = min(32, x.cols - wave * 32);
    const int wave_hi = wcols > 0 ? min(x.n + div_group(p, x.col0 + wave * 32 + wcols - 1) + 1, nblk * 32) : 0;
    const int full_end = x.n + div_group(p, x.col0 + wave * 32);

    uint4 qop[KS];
    {
      const char *qr = static_cast<const char *>(p.q) + ((colv ? token : x.start) * p.qs[0] + (colv ? head : 0) * p.qs[1]) * 2;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) qop[ks] = colv ? ld16(qr + ks * 32 + hb * 16) : make_uint4(0, 0, 0, 0);
    }
    // (the lowest finite value: no score may lie below the running maximum's start)
    float m = lowest(), ls = 0.0f;
    f32x16_t acc[NTL];
#pragma unroll
    for (int i = 0; i < NTL; ++i) acc[i] = f32x16_t{};
    bool left_out = false;

    const int32_t *table = p.table + int64_t(x.b) * p.max_pages;
    struct Pages { int x[DPW]; };
    auto pages_of = [&](int kb) {
      Pages pg;
#pragma unroll
      for (int i = 0; i < DPW; ++i)
        pg.x[i] = table_entry(table, min(min(kb, nblk - 1) * 32 + (i * kWaves + wave) * RPI, x.keys - 1) >> p.log2p);
      return pg;
    };
    // Every call issues 2 DPW transfers per wave; those of blocks past the last
    // one are switched off.  Rows past the last key are the last one again.
    auto issue = [&](int kb, const Pages &pg, auto st_c) {
      const bool on = kb < nblk;
#pragma unroll
      for (int i = 0; i < DPW; ++i) {
        const int first = min(kb * 32 + (i * kWaves + wave) * RPI, x.keys - 1);
        const int64_t at = (((int64_t(checked_page(p, pg.x[i])) * p.hkv + x.h) << p.log2p) + (first & mask)) * RB;
        const uint32_t row = min(lrow, x.keys - 1 - first);
        unsigned char *dst = slot(st_c) + (i * kWaves + wave) * 1024;
        dma16_s(dst, uniform_ptr(p.kp + at), row * RB + kchunk[i], on);
        dma16_s(dst + BLK, uniform_ptr(p.vp + at), row * RB + vchunk[i], on);
      }
    };

    if (blk0 < nblk) {
      issue(blk0, pages_of(blk0), std::integral_constant<int, 0>{});
      issue(blk0 + 1, pages_of(blk0 + 1), std::integral_constant<int, 1>{});
      issue(blk0 + 2, pages_of(blk0 + 2), std::integral_constant<int, 2>{});
      Pages next = pages_of(blk0 + 3);
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
        issue(kb + kSt - 1, next, std::integral_constant<int, (ST + kSt - 1) % kSt>{});
        next = pages_of(kb + kSt);
        if (kb * 32 >= wave_hi) return;
        const bool masked = kb * 32 + 31 > full_end;
        const char *vd = reinterpret_cast<const char *>(slot(stage_c)) + BLK;
        const char *kn = reinterpret_cast<const char *>(slot(std::integral_constant<int, SN>{}));   // block kb + 1's keys
        // (past the last block the next scores are not used)
        uint4 kr[4], va[NTL][2];
#pragma unroll
        for (int i = 0; i < 3; ++i) kr[i] = *reinterpret_cast<const uint4 *>(kn + kaddr[i]);
        float sv[16];
#pragma unroll
        for (int rr = 0; rr < 16; ++rr) sv[rr] = scn[rr];
        if (masked) {
          const int tr = one_register(lim - kb * 32 - 8 * hb);
#pragma unroll
          for (int rr = 0; rr < 16; ++rr)
            if (score_row(rr) > tr) sv[rr] = neg_inf();
        }
        float mx = fmaxf(fmaxf(sv[0], sv[1]), sv[2]);
#pragma unroll
        for (int rr = 3; rr < 15; rr += 2) mx = fmaxf(fmaxf(mx, sv[rr]), sv[rr + 1]);
        mx = fmaxf(mx, sv[15]);
        mx = max_halves(mx) * sl2;
        // (only the columns that need it: no column's bits depend on another's)
        const bool grown = mx > m + kLazyRescale;
        if (__any(grown)) {
          const float mn = grown ? mx : m;
          const float f = fast_exp2(m - mn);
          m = mn;
          ls *= f;
#pragma unroll
          for (int i = 0; i < NTL; ++i) acc[i] *= f;
        }
        // This wave's matrix work goes before the other wave's vector work (4 rows, 64/8
        // heads, 512 tokens on 12000: 929 -> 877 us).
        __builtin_amdgcn_s_setprio(1);
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
        __builtin_amdgcn_s_setprio(2);
        // P enters the value product rounded to bf16 (off by at most 2^-8 of a
        // probability, at random); its sum is taken in fp32 before that.
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
        if (masked) {
#pragma unroll
          for (int i = 0; i < NTL; ++i) left_out |= leave_out_nonfinite(va[i]);
        }
#pragma unroll
        for (int i = 0; i < NTL; ++i)
#pragma unroll
          for (int kk = 0; kk < 2; ++kk) acc[i] = mfma_32x32x16(va[i][kk], pb[kk], acc[i]);
        __builtin_amdgcn_s_setprio(0);
      };
      // Whole rounds of four steps (a step past the last block only keeps the
      // barriers and transfer counts in step).
      for (int kb = blk0; kb < nblk; kb += kSt) {
        step(std::integral_constant<int, 0>{}, kb);
        step(std::integral_constant<int, 1>{}, kb + 1);
        step(std::integral_constant<int, 2>{}, kb + 2);
        step(std::integral_constant<int, 3>{}, kb + 3);
      }
      // The ring is free for the next piece: no transfer is in flight, no wave reads.
      wait_vmcnt<0>();
      ring_barrier();
    }

    if (__any(left_out)) {
      for (int kb = max(blk0, (full_end + 1) >> 5); kb * 32 < wave_hi; ++kb) {
        auto load4 = [&](int i, int e) {
          const int key = kb * 32 + i;
          const char *row = p.vp + (((int64_t(checked_page(p, table[key >> p.log2p])) * p.hkv + x.h) << p.log2p) +
                                    (key & mask)) * RB;
          return row4(row, e);
        };
        add_nonfinite<D, false>(acc, load4, [&](int i) { return colv && kb * 32 + i <= lim; }, hb);
      }
    }

    ls += __shfl_xor(ls, 32, 64);
    const bool whole = x.pieces == 1;
    if (colv) {
      if (whole) {
        const float inv = 1.0f / ls;
        char *dst = static_cast<char *>(p.out) + (token * p.os[0] + head * p.os[1]) * 2;
#pragma unroll
        for (int i = 0; i < NTL; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float f[4] = {acc[i][4 * j] * inv, acc[i][4 * j + 1] * inv, acc[i][4 * j + 2] * inv, acc[i][4 * j + 3] * inv};
            store_out<2, 4>(dst + (32 * i + 8 * j + 4 * hb) * 2, f);
          }
        if (p.lse && hb == 0) p.lse[token * p.hq + head] = (m + __log2f(ls)) * kLn2;
      } else {
        float *rec = record_of(p, x.first, x.index);
        const uint32_t at = (2 * hb * kWideCols + c) * 8;   // bytes; the rest is the same for all lanes
#pragma unroll
        for (int i = 0; i < NTL; ++i)
#pragma unroll
          for (int j = 0; j < 16; j += 2) {
            typedef __attribute__((address_space(1))) uint64_t gpair;
            const char *row = uniform_ptr(reinterpret_cast<const char *>(rec) + (16 * i + 4 * (j >> 2) + (j & 3) / 2) * kWideCols * 8);
            *reinterpret_cast<gpair *>(reinterpret_cast<uintptr_t>(row) + at) =
                (uint64_t(__float_as_uint(acc[i][j + 1])) << 32) | __float_as_uint(acc[i][j]);
          }
        if (hb == 0) *reinterpret_cast<float2 *>(rec + kWideCols * D + 2 * c) = make_float2(m, ls);
      }
    }
    if (!whole && tid == 0) cuts.piece[cuts.n++] = x;
  }
  join_cuts<2, D, false>(p, cuts, nullptr);
}

template <int ES, int D, int NT, bool SPLIT_KEYS>
void launch_narrow(const FullParams &p, size_t lds, hipStream_t s) {
  constexpr int kLog2Keys = Narrow<ES, D>::U == 2 ? 5 : 4;
  const dim3 grid(p.places), threads(kThreads);
  if (p.log2p < kLog2Keys) hipLaunchKernelGGL((full_narrow_kernel<ES, D, NT, true, SPLIT_KEYS>), grid, threads, lds, s, p);
  else hipLaunchKernelGGL((full_narrow_kernel<ES, D, NT, false, SPLIT_KEYS>), grid, threads, lds, s, p);
}

template <int ES, int D>
hipError_t launch_rotation(const RotateParams &p, bool paged, hipStream_t s) {
  // Few tokens: the heads of each shared out to workgroups of 256 units, so that the chip is
  // filled (32 + 32 heads of 128 in bf16: 32 tokens 2.9 us, in one workgroup each 3.6; 512 4.0
  // and 4.5; 1024 5.1 and 5.2). Many: one workgroup forms a token's angles once (2048: 10.6 us,
  // shared 10.8; what sharing gains beyond, 3 % at 8192 and 1 % at 14000, is not taken: it
  // would multiply the workgroups of the largest launches).
  const int units = (p.hq + (paged ? 2 : 1) * p.hkv) * (D * ES / 32);
  const int shares = int64_t(units) * p.total < int64_t(2048) * kThreads ? (units + kThreads - 1) / kThreads : 1;
  const dim3 grid(p.total + (paged ? 1 : 0), shares);
  if (paged) hipLaunchKernelGGL((rotate_kernel<ES, D, true>), grid, dim3(kThreads), 0, s, p);
  else hipLaunchKernelGGL((rotate_kernel<ES, D, false>), grid, dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

template <int ES, int D>
hipError_t attend(const FullParams &p, hipStream_t s) {
  if (p.one_launch && p.tile_cols > (ES == 2 ? 32 : 16)) return hipErrorInvalidValue;   // (only narrow tiles join)
  const size_t lds = p.rows <= 64 ? 0 : (size_t(p.rows) + 1) * sizeof(int64_t);   // the sums before every row
  if constexpr (ES == 2) {
    if (p.tile_cols == kWideCols) hipLaunchKernelGGL((full_wide_kernel<D>), dim3(p.places), dim3(kThreads), lds, s, p);
    else if (p.tile_cols == 32) launch_narrow<ES, D, 2, true>(p, lds, s);
    else launch_narrow<ES, D, 1, true>(p, lds, s);
  } else {
    if (p.tile_cols == 64) launch_narrow<ES, D, 1, false>(p, lds, s);
    else launch_narrow<ES, D, 1, true>(p, lds, s);
  }
  if (!p.one_launch) {
    const int cols = static_cast<int>(std::min<int64_t>(p.tile_cols, int64_t(p.max_chunk) * (p.hq / p.hkv)));
    const int step = cols > 16 ? 8 : 2;
    hipLaunchKernelGGL((full_join_kernel<ES, D>), dim3(p.places, (cols + step - 1) / step), dim3(kThreads), 0, s, p, step);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(int elem_bytes, int head_dim, bool paged, const RotateParams &p, hipStream_t s) {
  if (elem_bytes == 2) return head_dim == 128 ? launch_rotation<2, 128>(p, paged, s) : launch_rotation<2, 64>(p, paged, s);
  return head_dim == 128 ? launch_rotation<4, 128>(p, paged, s) : launch_rotation<4, 64>(p, paged, s);
}

hipError_t launch_full_attend(int elem_bytes, int head_dim, const FullParams &p, hipStream_t s) {
  if (elem_bytes == 2) return head_dim == 128 ? attend<2, 128>(p, s) : attend<2, 64>(p, s);
  return head_dim == 128 ? attend<4, 128>(p, s) : attend<4, 64>(p, s);
}

}  // namespace dmc
