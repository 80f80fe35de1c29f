// Parameters and launchers of the rotation and of full caches (dmc_full.hip).
#pragma once
#include "dmc_internal.h"

namespace dmc {

constexpr int32_t FLAG_BAD_PAGE = 8;   // beside the flags of the compressed caches: page id outside the pool

// Position rotation of packed tensors, and the append to a full cache (dmc_full.hip).
// Tensors are [total, heads, d] with element strides of the token and head axes.
struct RotateParams {
  const void *q, *k, *v;         // v: append only
  void *qo, *ko;                 // ko: rotation only
  int64_t qs[2], ks[2], vs[2], qos[2], kos[2];
  const float *inv_freq;         // [r / 2]
  const int32_t *positions;      // [total] (rotation)
  // append
  const int32_t *cu;             // [rows + 1], nullptr: one token per row
  const int32_t *len;            // [rows], < 0: not in use
  const int32_t *table;          // [rows, max_pages]
  char *kp, *vp;                 // [num_pages][hkv][P][d]
  int32_t *flags;                // optional
  int32_t total, rows, hq, hkv, r, halves, inverse, log2p, max_pages, num_pages, capacity;   // hq 0: no queries
};
// (elem_bytes, head_dim); paged: append, else rotation.
hipError_t launch_rotate(int elem_bytes, int head_dim, bool paged, const RotateParams &p, hipStream_t s);

// Attention of new tokens over a full cache.
// A piece of a unit: keys k0 .. k1 - 1 of the `keys` that tile columns col0 .. col0 +
// cols - 1 of row b and kv head h take; piece `index` of `pieces`, which are those of
// ranges first, first + 1, ...
struct FullPiece {
  int32_t b, n, start, h, col0, cols, keys, k0, k1, first, index, pieces;
};
struct FullParams {
  const void *q;
  void *out;
  int64_t qs[2], os[2];
  float *lse;                    // optional [total, hq]
  const int32_t *cu, *len, *table;
  const char *kp, *vp;
  int32_t *flags;                // optional
  int32_t *counters;             // workspace: [3][places], 0 between calls (one launch)
  FullPiece *cut_units;          // workspace: [places] (two launches)
  int32_t one_launch;
  float *partials;               // workspace: [places][2][record_floats]
  int64_t record_floats;
  float scale_log2;
  uint32_t group_magic;          // a / G = mulhi(a, group_magic) >> group_shift for a < 2^31 (G = 1: group_shift -1)
  int32_t group_shift;
  int32_t total, rows, hq, hkv, log2p, max_pages, num_pages, capacity, max_chunk, places, tile_cols, tile_tokens;
};
// Workgroups of the attention: two to each of 256 compute units (with three, 64 rows of
// up to 1000 keys take 47.7 us instead of 40.1, wide tiles 1044 us instead of 855).
constexpr int kFullPlaces = 512;
// Query columns of a tile: 16 or 32 (bf16) that all waves of a workgroup share; wider
// ones, of whole tokens, once a row has more: 128 (bf16) or 64 (fp32).  Drafts of 4
// tokens, 64/8 heads, 16 rows of up to 8192 keys: 69.5 us with 32 columns, 83.0 with 16,
// 91.7 with 128; fp32 chunks of 64 tokens on 8000, 8 rows of 8/4 heads of 128 (109 us at a
// large fp32 product's rate): 190 us with 64 columns, 290 with 16.
constexpr inline int full_tile_cols(int elem_bytes, int64_t max_chunk, int group) {
  const int64_t cols = max_chunk * group;
  if (elem_bytes == 4) return cols <= 16 || group > 64 ? 16 : 64;
  return cols <= 16 ? 16 : cols <= 32 || group > 128 ? 32 : 128;
}
// Whether the work is small whatever the lengths are (tiles: narrow column tiles of all
// rows): then all tiles are narrow and their records are joined within the launch.
// A row of 900 keys: 11.2 us, in two launches 12.3; 77 tokens on 700, 2 rows of 32/8 heads:
// 21.3 us, with wide tiles in two launches 27.7.  Larger work joined within the launch: 64
// rows of up to 1000 keys 43.9 us against 40.1, 16 rows of up to 24000 152 against 147.
constexpr inline bool full_one_launch(int64_t tiles, int hkv, int64_t capacity) {
  return tiles * hkv * capacity <= int64_t(1) << 18;
}
hipError_t launch_full_attend(int elem_bytes, int head_dim, const FullParams &p, hipStream_t s);

}  // namespace dmc
