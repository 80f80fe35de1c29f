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
// Rotation and append.  A workgroup takes 1 << shift tokens (1 or 4): one wave
// per token forms the cosines and sines of its pairs (in 64 bits up to the
// fraction of a turn), which every head of the token uses from LDS; then each
// thread moves units of two 16-byte vectors of a head, the two halves of 16 / ES
// pairs (or 16 / ES adjacent pairs), in grid.y shares of the group's units.
// Bound by HBM, each element read and written once.
// ---------------------------------------------------------------------------
constexpr int kRotTokens = 4;

template <int ES, int D, bool PAGED>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotateParams p, int shift) {
  constexpr int N = 16 / ES, UPR = D * ES / 32;   // elements of a vector, units of a row
  constexpr int kBatch = 4;                       // units of a thread whose loads are in flight at once
  __shared__ __align__(16) float cosv[kRotTokens][64], sinv[kRotTokens][64];
  __shared__ int64_t place[kRotTokens];   // element offset of the token's slot of kv head 0 (-1: none)
  __shared__ int state[kRotTokens];       // 0: no token of a row, 1: here, 2: dropped
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
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
  const int t0 = blockIdx.x << shift, ntok = min(1 << shift, p.total - t0);
  if (wave < ntok) {
    const int t = t0 + wave;
    int pos, st = 1;
    int64_t at = -1;
    if constexpr (PAGED) {
      const int b = p.cu ? row_of_token(p.cu, p.rows, p.total, t) : t;
      const FullRow r = full_row(p.cu, p.len, p.total, p.capacity, b);
      const int i = t - r.start;
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
      place[wave] = at;
      state[wave] = st;
    }
    if (lane < p.r / 2) {
      // turns: the product and its fraction in 64 bits
      const double turns = pos * (double(p.inv_freq[lane]) * 0.15915494309189533577);
      float s, c;
      sincospif(2.0f * static_cast<float>(turns - rint(turns)), &s, &c);
      cosv[wave][lane] = c;
      sinv[wave][lane] = p.inverse ? -s : s;
    }
  }
  __syncthreads();

  const int nrows = p.hq + (PAGED ? 2 : 1) * p.hkv, units = ntok * nrows * UPR;
  const int rv2 = p.r * ES / 32, stride = kThreads * gridDim.y;   // rotated units of a row
  for (int base = blockIdx.y * kThreads + tid; base < units; base += stride * kBatch) {
    uint4 x[kBatch][2];
    char *dst[kBatch];       // of the first vector (nullptr: nothing to write)
    int gap[kBatch], cs[kBatch];   // bytes to the second one; first pair (token * 64 + pair), -1: not rotated
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int idx = base + j * stride;
      dst[j] = nullptr;
      gap[j] = 16;
      cs[j] = -1;
      x[j][0] = x[j][1] = make_uint4(0, 0, 0, 0);
      if (idx >= units) continue;
      const int u = idx % UPR, rr = idx / UPR, tok = rr / nrows, row = rr - tok * nrows;
      const int st = PAGED ? state[tok] : 1;
      if (PAGED && st == 0) continue;
      const int64_t t = t0 + tok;
      const bool is_q = row < p.hq, is_v = PAGED && row >= p.hq + p.hkv;
      int v0 = 2 * u;
      if (u < rv2 && !is_v) {
        cs[j] = tok * 64 + u * N;
        if (p.halves) {
          v0 = u;
          gap[j] = rv2 * 16;
        }
      }
      const char *src;
      if (is_q) {
        src = static_cast<const char *>(p.q) + (t * p.qs[0] + row * p.qs[1]) * ES;
        dst[j] = static_cast<char *>(p.qo) + (t * p.qos[0] + row * p.qos[1]) * ES + v0 * 16;
      } else {
        const int h = row - p.hq - (is_v ? p.hkv : 0);
        src = is_v ? static_cast<const char *>(p.v) + (t * p.vs[0] + h * p.vs[1]) * ES
                   : static_cast<const char *>(p.k) + (t * p.ks[0] + h * p.ks[1]) * ES;
        if constexpr (PAGED) {
          if (place[tok] < 0) continue;
          dst[j] = (is_v ? p.vp : p.kp) + (place[tok] + ((int64_t(h) * D) << p.log2p)) * ES + v0 * 16;
        } else {
          dst[j] = static_cast<char *>(p.ko) + (t * p.kos[0] + h * p.kos[1]) * ES + v0 * 16;
        }
      }
      if (st == 2) {   // a dropped token's queries: zeros
        cs[j] = -1;
        continue;
      }
      x[j][0] = ld16(src + v0 * 16);
      x[j][1] = ld16(src + v0 * 16 + gap[j]);
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      if (!dst[j]) continue;
      if (cs[j] >= 0) {
        float a[N], b[N], c[N], s[N];
        V16<ES>::unpack(x[j][0], a);
        V16<ES>::unpack(x[j][1], b);
#pragma unroll
        for (int i = 0; i < N; i += 4) {
          *reinterpret_cast<f32x4_t *>(c + i) = *reinterpret_cast<const f32x4_t *>(&cosv[0][0] + cs[j] + i);
          *reinterpret_cast<f32x4_t *>(s + i) = *reinterpret_cast<const f32x4_t *>(&sinv[0][0] + cs[j] + i);
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
        x[j][0] = V16<ES>::pack(a);
        x[j][1] = V16<ES>::pack(b);
      }
      st16(dst[j], x[j][0]);
      st16(dst[j] + gap[j], x[j][1]);
    }
  }
}

// ---------------------------------------------------------------------------
// Attention: how the work is shared out.  A unit is one column tile (query
// columns: the pairs of a new token and a head of one kv head's group) of one row
// and kv head; it takes as many keys as its row holds.  The units of all rows lie
// one after another in a space of keys, row by row, which is cut into equal
// ranges, one to a workgroup; a block of 32 keys belongs to the range that its
// first key lies in.  A workgroup whose range holds a unit whole writes its output,
// else a partial record (running maximum, sum and accumulator): the record of a
// unit that started in an earlier range in the workgroup's first place, that of
// one that goes on in the next range in its second.  The workgroup where a unit
// starts describes it for the combine pass.
// ---------------------------------------------------------------------------
// Sums of the rows' keys before every row, in LDS (prefix[rows + 1]); the total.
template <typename Weight>
__device__ __forceinline__ int64_t scan_rows(int64_t *prefix, int64_t *sums, int rows, Weight &&weight) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (rows + kThreads - 1) / kThreads, b0 = min(tid * per, rows), b1 = min(b0 + per, rows);
  int64_t own = 0;
  for (int b = b0; b < b1; ++b) {
    prefix[b] = own;
    own += weight(b);
  }
  int64_t x = own;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  if (lane == 63) sums[wave] = x;
  __syncthreads();
  int64_t before = x - own, all = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    if (i < wave) before += sums[i];
    all += sums[i];
  }
  for (int b = b0; b < b1; ++b) prefix[b] += before;
  if (tid == 0) prefix[rows] = all;
  __syncthreads();
  return all;
}
// The row whose keys hold position pos of the space (pos < prefix[rows]).
__device__ __forceinline__ int row_at_key(const int64_t *prefix, int rows, int64_t pos) {
  int lo = 0, hi = rows;   // prefix[lo] <= pos < prefix[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (prefix[mid] <= pos) lo = mid;
    else hi = mid;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Workgroup i runs on XCD i mod 8: each XCD takes one run of ranges, so that the
// tiles of a kv head read its keys through one L2.
__device__ __forceinline__ int range_of_block(int blocks) {
  return (blocks & 7) ? static_cast<int>(blockIdx.x) : (blockIdx.x & 7) * (blocks >> 3) + (blockIdx.x >> 3);
}

// Rows of out and lse of tokens that are dropped (a row not in use, or full).
template <int ES, int D>
__device__ __forceinline__ void clear_dropped(const FullParams &p) {
  for (int b = blockIdx.x; b < p.rows; b += gridDim.x) {
    const FullRow r = full_row(p.cu, p.len, p.total, p.capacity, b);
    const int first = min(r.m, r.given), items = (r.given - first) * p.hq;
    constexpr int VPR = D * ES / 16;
    for (int64_t i = threadIdx.x; i < int64_t(items) * VPR; i += kThreads) {
      const int64_t x = i / VPR, t = r.start + first + x / p.hq, h = x % p.hq;
      st16(static_cast<char *>(p.out) + (t * p.os[0] + h * p.os[1]) * ES + (i % VPR) * 16, make_uint4(0, 0, 0, 0));
      if (p.lse && i % VPR == 0) p.lse[t * p.hq + h] = neg_inf();
    }
  }
}

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

// How the columns of a row and kv head are cut into tiles.  A row of m new tokens
// at n ..:
//   whole rows (TRI false): tiles of `cols` columns, each over all n + m keys;
//   TRI: tiles of `per` = cols / G whole tokens, tile t over the keys that its last
//     token sees, n + min(m, (t + 1) per); the keys of the tiles before tile t are
//     t n + per t (t + 1) / 2.
template <bool TRI>
struct Tiles {
  int n, m, count, step;   // step: tokens of a tile (TRI) or its columns
  __device__ __forceinline__ Tiles(int n_, int m_, int G, int cols) : n(n_), m(m_) {
    if constexpr (TRI) {
      step = cols / G;
      count = (m + step - 1) / step;
    } else {
      step = cols;
      count = (m * G + cols - 1) / cols;
    }
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

// A piece of a unit: keys k0 .. k1 - 1 of the `keys` that tile columns col0 .. col0 +
// cols - 1 of row b and kv head h take.
struct Piece {
  int b, n, start, h, col0, cols, keys, k0, k1;
};
// The next piece of a range of the space that starts at pos (in row b or later).
template <bool TRI>
__device__ __forceinline__ Piece next_piece(const FullParams &p, const int64_t *prefix, int b, int64_t pos, int64_t hi,
                                            int G) {
  while (prefix[b + 1] <= pos) ++b;
  Piece x;
  x.b = __builtin_amdgcn_readfirstlane(b);
  const FullRow r = full_row(p.cu, p.len, p.total, p.capacity, x.b);
  x.n = __builtin_amdgcn_readfirstlane(r.n);
  x.start = __builtin_amdgcn_readfirstlane(r.start);
  const int m = __builtin_amdgcn_readfirstlane(min(r.m, p.max_chunk));
  const Tiles<TRI> tiles(x.n, m, G, p.tile_cols);
  const int64_t per_head = tiles.all(), off = pos - prefix[x.b];
  x.h = __builtin_amdgcn_readfirstlane(static_cast<int>(off / per_head));
  const int64_t in_head = off - x.h * per_head;
  const int t = __builtin_amdgcn_readfirstlane(tiles.at(in_head));
  x.keys = tiles.keys(t);
  x.k0 = __builtin_amdgcn_readfirstlane(static_cast<int>(in_head - tiles.before(t)));
  x.k1 = __builtin_amdgcn_readfirstlane(static_cast<int>(min(int64_t(x.keys), x.k0 + (hi - pos))));
  x.col0 = tiles.first_col(t, G);
  x.cols = min(TRI ? tiles.step * G : tiles.step, m * G - x.col0);
  return x;
}
// The keys of all units of row b.
template <bool TRI>
__device__ __forceinline__ int64_t row_keys(const FullParams &p, int b, int G) {
  const FullRow r = full_row(p.cu, p.len, p.total, p.capacity, b);
  const int m = min(r.m, p.max_chunk);
  return m > 0 ? p.hkv * Tiles<TRI>(r.n, m, G, p.tile_cols).all() : int64_t(0);
}
// Describes the unit that starts in this range and goes on in the next one.
__device__ __forceinline__ void describe_unit(FullUnit *u, const Piece &x, int64_t pos, int64_t per, int range, int G) {
  u->pieces = static_cast<int>((pos + x.keys - 1) / per) - range + 1;
  u->row_start = x.start;
  u->head = x.h * G;
  u->first_col = x.col0;
  u->cols = x.cols;
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

// ---------------------------------------------------------------------------
// Tiles of 16 and 32 columns in registers: decode steps, drafts, all of fp32.
// Bound by HBM: keys and values go from memory straight into the operands of the
// 16x16 matrix instructions, without LDS.  Blocks of 16 U keys; with lane l = 16 g +
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
  __device__ static __forceinline__ void load_row(uint4 (&x)[KC], const char *row) {
#pragma unroll
    for (int c = 0; c < KC; ++c) x[c] = STREAM ? ld16_stream(row + c * kKeyStep) : ld16(row + c * kKeyStep);
  }
  template <bool STREAM>
  __device__ static __forceinline__ vrow_t load_value(const char *p) {
    return STREAM ? __builtin_nontemporal_load(reinterpret_cast<const vrow_t *>(p)) : *reinterpret_cast<const vrow_t *>(p);
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
  __device__ static __forceinline__ f32x4_t load4f(const char *p) {
    return STREAM ? __builtin_nontemporal_load(reinterpret_cast<const f32x4_t *>(p)) : *reinterpret_cast<const f32x4_t *>(p);
  }
  template <bool STREAM>
  __device__ static __forceinline__ void load_row(f32x4_t (&x)[KC], const char *row) {
#pragma unroll
    for (int c = 0; c < KC; ++c) x[c] = load4f<STREAM>(row + c * kKeyStep);
  }
  template <bool STREAM>
  __device__ static __forceinline__ vrow_t load_value(const char *p) {
    vrow_t v;
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
      const f32x4_t x = load4f<STREAM>(p + 16 * i);
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

// Fewest keys of a workgroup's range.
constexpr int kNarrowRange = 256;

// SMALL: pages of fewer tokens than a block.
template <int ES, int D, int NT, bool SMALL, bool SPLIT_KEYS>
__global__ __launch_bounds__(kThreads, 2) void full_narrow_kernel(FullParams p) {
  using X = Narrow<ES, D>;
  constexpr int E = X::E, U = X::U, KEYS = 16 * U, RB = D * ES, JS = D + 4, STEP = SPLIT_KEYS ? kWaves : 1;
  constexpr int COLS = 16 * NT * (SPLIT_KEYS ? 1 : kWaves);
  constexpr bool TRI = !SPLIT_KEYS;
  extern __shared__ int64_t prefix[];
  __shared__ int64_t sums[kWaves];
  __shared__ __align__(16) float area[SPLIT_KEYS ? kWaves : 1][16][JS];
  __shared__ float stat[kWaves][16][2];
  const int tid = threadIdx.x, lane = tid & 63, c16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = p.hq / p.hkv;

  if (blockIdx.x == 0 && p.flags) {
    int32_t f = 0;
    for (int b = tid; b < p.rows; b += kThreads) f |= row_flags(p.cu, p.len, p.total, p.capacity, b, p.max_chunk);
    if (f) raise(p.flags, f);
  }
  const int64_t all = scan_rows(prefix, sums, p.rows, [&](int b) { return row_keys<TRI>(p, b, G); });
  clear_dropped<ES, D>(p);
  const int range = range_of_block(gridDim.x);
  const int64_t per = max((all + gridDim.x - 1) / gridDim.x, int64_t(kNarrowRange));
  const int64_t lo = range * per, hi = min(lo + per, all);
  bool cut = false;
  int b = lo < hi ? row_at_key(prefix, p.rows, lo) : 0;

  for (int64_t pos = lo; pos < hi;) {
    const Piece x = next_piece<TRI>(p, prefix, b, pos, hi, G);
    b = x.b;
    const int col0 = x.col0 + (SPLIT_KEYS ? 0 : wave * 16 * NT), cols = min(16 * NT, x.col0 + x.cols - col0);   // this wave's
    // Keys that this wave's columns see, and the last key that they all do.
    const int keys = SPLIT_KEYS ? x.keys : cols > 0 ? x.n + (col0 + cols - 1) / G + 1 : 0;
    const int full_end = x.n + col0 / G;

    typename X::Query q[NT];
    int lim[NT];   // the last key that this lane's column sees
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int c = t * 16 + c16;
      const int i = (col0 + c) / G, head = x.h * G + (col0 + c) - i * G;
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

    const int32_t *table = p.table + int64_t(b) * p.max_pages;
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
      return pool + ((int64_t(checked_page(p, page)) * p.hkv + x.h) << p.log2p) * RB;
    };
    typename X::Keys kx;
    typename X::Values vx;
    auto load_keys = [&](int kb, const Pages &pg) {
      if constexpr (SMALL) {
#pragma unroll
        for (int u = 0; u < U; ++u)
          X::template load_row<SPLIT_KEYS>(kx.x[u], page_at(p.kp, pg.x[u]) +
              (min(kb * KEYS + u * 16 + c16, keys - 1) & mask) * RB + X::key_offset(g4));
      } else {
        const char *at = uniform_ptr(page_at(p.kp, pg.x[0]) + int64_t((kb * KEYS) & mask) * RB);
        const uint32_t last = keys - 1 - kb * KEYS;
#pragma unroll
        for (int u = 0; u < U; ++u)
          X::template load_row<SPLIT_KEYS>(kx.x[u], at + (min(uint32_t(u * 16 + c16), last) * RB + X::key_offset(g4)));
      }
    };
    auto load_values = [&](int kb, const Pages &pg) {
      if constexpr (SMALL) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const char *at = page_at(p.vp, pg.x[U + u]) + c16 * (E * ES);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            vx.x[u * 4 + i] = X::template load_value<SPLIT_KEYS>(
                at + (min(kb * KEYS + u * 16 + g4 * 4 + i, keys - 1) & mask) * RB);
        }
      } else {
        const char *at = uniform_ptr(page_at(p.vp, pg.x[0]) + int64_t((kb * KEYS) & mask) * RB);
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
      Pages cur = pages_of(kb), next = pages_of(min(kb + STEP, kb1 - 1));
      load_keys(kb, cur);
      load_values(kb, cur);
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
        cur = next;
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
            const char *row = page_at(p.vp, table_entry(table, key >> p.log2p)) + int64_t(key & mask) * RB;
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

    const bool whole = x.k0 == 0 && x.k1 == x.keys;
    float *rec = p.partials + (int64_t(range) * 2 + (x.k0 == 0 ? 1 : 0)) * p.record_floats;
    // E elements e0 .. of a column of the tile: to the output, or its record.
    auto put = [&](int col, int e0, float top, float sum, float (&o)[E]) {
      if (whole) {
        const int i = (x.col0 + col) / G, head = x.h * G + (x.col0 + col) - i * G;
        const int64_t token = x.start + i;
        const float inv = 1.0f / sum;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] *= inv;
        store_out<ES, E>(static_cast<char *>(p.out) + (token * p.os[0] + head * p.os[1] + e0) * ES, o);
        if (p.lse && e0 == 0) p.lse[token * p.hq + head] = (top + __log2f(sum)) * kLn2;
      } else {
        store_out<4, E>(reinterpret_cast<char *>(rec + col * D + e0), o);
        if (e0 == 0) {
          rec[COLS * D + 2 * col] = top;
          rec[COLS * D + 2 * col + 1] = sum;
        }
      }
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
        const int c = tid >> 4, e0 = (tid & 15) * E, col = t * 16 + c;
        if (col < x.cols) {
          float top = stat[0][c][0];
#pragma unroll
          for (int w = 1; w < kWaves; ++w) top = fmaxf(top, stat[w][c][0]);
          float sum = 0.0f, o[E] = {};
#pragma unroll
          for (int w = 0; w < kWaves; ++w) {
            const float f = fast_exp2(stat[w][c][0] - top);
            sum = fmaf(stat[w][c][1], f, sum);
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = fmaf(area[w][c][e0 + e], f, o[e]);
          }
          put(col, e0, top, sum, o);
        }
      } else if (t * 16 + c16 < cols) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float o[E];
#pragma unroll
          for (int j = 0; j < E; ++j) o[j] = acc[t][j][r];
          put(wave * 16 * NT + t * 16 + c16, (g4 * 4 + r) * E, mx[t], l, o);
        }
      }
    }
    if (x.k0 == 0 && x.k1 < x.keys) {
      cut = true;
      if (tid == 0) describe_unit(p.units + range, x, pos, per, range, G);
    }
    pos += x.k1 - x.k0;
  }
  if (tid == 0 && !cut) p.units[range].pieces = 0;
}

// ---------------------------------------------------------------------------
// Wide tiles (128 columns, bf16): pieces of prompts, turns, long drafts.  Bound by
// the matrix cores and the vector work of the softmax beside them.  One workgroup =
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
constexpr int kWideRange = 1024;   // fewest keys of a workgroup's range
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
  __shared__ int64_t sums[kWaves];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, hb = lane >> 5;
  const int G = p.hq / p.hkv;
  if (blockIdx.x == 0 && p.flags) {
    int32_t f = 0;
    for (int b = tid; b < p.rows; b += kThreads) f |= row_flags(p.cu, p.len, p.total, p.capacity, b, p.max_chunk);
    if (f) raise(p.flags, f);
  }
  const int64_t all = scan_rows(prefix, sums, p.rows, [&](int b) { return row_keys<true>(p, b, G); });
  clear_dropped<2, D>(p);
  const int range = range_of_block(gridDim.x);
  const int64_t per = max((all + gridDim.x - 1) / gridDim.x, int64_t(kWideRange));
  const int64_t lo = range * per, hi = min(lo + per, all);
  bool cut = false;
  int b = lo < hi ? row_at_key(prefix, p.rows, lo) : 0;
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

  for (int64_t pos = lo; pos < hi;) {
    const Piece x = next_piece<true>(p, prefix, b, pos, hi, G);
    b = x.b;
    const int c = wave * 32 + col, ti = (x.col0 + c) / G, head = x.h * G + (x.col0 + c) - ti * G;
    const bool colv = c < x.cols;
    const int64_t token = x.start + ti;
    const int lim = x.n + ti;   // the last key that this column sees
    const int blk0 = (x.k0 + 31) >> 5, nblk = (x.k1 + 31) >> 5;
    // Keys < wave_hi feed this wave, those up to full_end all of its columns.
    const int wcols = min(32, x.cols - wave * 32);
    const int wave_hi = wcols > 0 ? min(x.n + (x.col0 + wave * 32 + wcols - 1) / G + 1, nblk * 32) : 0;
    const int full_end = x.n + (x.col0 + wave * 32) / G;

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

    const int32_t *table = p.table + int64_t(b) * p.max_pages;
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
    const bool whole = x.k0 == 0 && x.k1 == x.keys;
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
        float *rec = p.partials + (int64_t(range) * 2 + (x.k0 == 0 ? 1 : 0)) * p.record_floats;
#pragma unroll
        for (int i = 0; i < NTL; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            *reinterpret_cast<f32x4_t *>(rec + c * D + 32 * i + 8 * j + 4 * hb) =
                f32x4_t{acc[i][4 * j], acc[i][4 * j + 1], acc[i][4 * j + 2], acc[i][4 * j + 3]};
        if (hb == 0) {
          rec[kWideCols * D + 2 * c] = m;
          rec[kWideCols * D + 2 * c + 1] = ls;
        }
      }
    }
    if (x.k0 == 0 && x.k1 < x.keys) {
      cut = true;
      if (tid == 0) describe_unit(p.units + range, x, pos, per, range, G);
    }
    pos += x.k1 - x.k0;
  }
  if (tid == 0 && !cut) p.units[range].pieces = 0;
}

// Joins the records of a unit that was cut: o = sum_i 2^(m_i - M) acc_i / sum_i
// 2^(m_i - M) l_i.  A workgroup per range (one unit at most starts in it and goes
// on) and 8 columns; D / 4 lanes' groups of 4 elements, the groups that columns do
// not need sharing the records.
template <int ES, int D>
__global__ __launch_bounds__(kThreads) void full_combine_kernel(FullParams p, int tile_cols) {
  constexpr int LPG = D / 4, GROUPS = kThreads / LPG, CPW = 8;   // lanes of a group
  const int range = blockIdx.x, col0 = blockIdx.y * CPW;
  const FullUnit u = p.units[range];
  const int cols = min(CPW, u.cols - col0);
  if (u.pieces == 0 || cols <= 0) return;
  __shared__ __align__(16) float part[GROUPS][D];
  const int tid = threadIdx.x, group = tid / LPG, gl = tid % LPG;
  int slices = 1;   // groups per column
  while (slices * 2 * cols <= GROUPS) slices *= 2;
  const int G = p.hq / p.hkv;
  auto record = [&](int i) { return p.partials + (int64_t(range + i) * 2 + (i == 0 ? 1 : 0)) * p.record_floats; };
  for (int first = 0; first < cols; first += GROUPS / slices) {
    const int cc = first + group / slices, slice = group % slices;
    const bool on = cc < cols;
    const int col = col0 + (on ? cc : 0);
    float top = lowest(), sum = 0.0f;
    for (int i = gl; i < u.pieces; i += LPG) {
      const float *ml = record(i) + tile_cols * D + 2 * col;
      const float mn = fmaxf(top, ml[0]);
      sum = sum * fast_exp2(top - mn) + ml[1] * fast_exp2(ml[0] - mn);
      top = mn;
    }
#pragma unroll
    for (int o = 1; o < LPG; o <<= 1) {
      const float to = __shfl_xor(top, o, LPG), so = __shfl_xor(sum, o, LPG), mn = fmaxf(top, to);
      sum = sum * fast_exp2(top - mn) + so * fast_exp2(to - mn);
      top = mn;
    }
    f32x4_t o = f32x4_t{};
#pragma unroll 4
    for (int i = slice; i < u.pieces; i += slices) {
      const float *r = record(i);
      const f32x4_t x = *reinterpret_cast<const f32x4_t *>(r + col * D + 4 * gl);
      const float f = fast_exp2(r[tile_cols * D + 2 * col] - top);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fmaf(x[e], f, o[e]);
    }
    *reinterpret_cast<f32x4_t *>(&part[group][4 * gl]) = o;
    __syncthreads();
    if (on && slice == 0) {
      for (int s = 1; s < slices; ++s) o += *reinterpret_cast<const f32x4_t *>(&part[group + s][4 * gl]);
      const int i = (u.first_col + col) / G, head = u.head + (u.first_col + col) - i * G;
      const int64_t token = u.row_start + i;
      const float inv = 1.0f / sum, f[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
      store_out<ES, 4>(static_cast<char *>(p.out) + (token * p.os[0] + head * p.os[1] + 4 * gl) * ES, f);
      if (p.lse && gl == 0) p.lse[token * p.hq + head] = (top + __log2f(sum)) * kLn2;
    }
    __syncthreads();
  }
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
  // Few tokens: one to a workgroup, their heads shared out, so that the chip is filled.
  const int64_t units = int64_t(p.total) * (p.hq + (paged ? 2 : 1) * p.hkv) * (D * ES / 32);
  const bool few = units < int64_t(2048) * kThreads;
  const int shift = few ? 0 : 2, groups = (p.total + (1 << shift) - 1) >> shift;
  const int shares = few ? static_cast<int>((units / p.total + kThreads - 1) / kThreads) : 1;
  const dim3 grid(groups + (paged ? 1 : 0), shares);
  if (paged) hipLaunchKernelGGL((rotate_kernel<ES, D, true>), grid, dim3(kThreads), 0, s, p, shift);
  else hipLaunchKernelGGL((rotate_kernel<ES, D, false>), grid, dim3(kThreads), 0, s, p, shift);
  return hipGetLastError();
}

template <int ES, int D>
hipError_t attend(const FullParams &p, hipStream_t s) {
  const size_t lds = (size_t(p.rows) + 1) * sizeof(int64_t);
  if constexpr (ES == 2) {
    if (p.tile_cols == kWideCols) hipLaunchKernelGGL((full_wide_kernel<D>), dim3(p.places), dim3(kThreads), lds, s, p);
    else if (p.tile_cols == 32) launch_narrow<ES, D, 2, true>(p, lds, s);
    else launch_narrow<ES, D, 1, true>(p, lds, s);
  } else {
    if (p.tile_cols == 64) launch_narrow<ES, D, 1, false>(p, lds, s);
    else launch_narrow<ES, D, 1, true>(p, lds, s);
  }
  const int cols = static_cast<int>(std::min<int64_t>(p.tile_cols, int64_t(p.max_chunk) * (p.hq / p.hkv)));
  hipLaunchKernelGGL((full_combine_kernel<ES, D>), dim3(p.places, (cols + 7) / 8), dim3(kThreads), 0, s, p, p.tile_cols);
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
