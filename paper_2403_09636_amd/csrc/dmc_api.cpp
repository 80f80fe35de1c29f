// Host side of the DMC C ABI: configuration and argument validation,
// workspace layout, per-layer state and kernel launches.
//
// Every validation runs before the first HIP call of an entry point, so an
// invalid request returns its status without touching the device (and can
// be exercised on a machine with no GPU).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <algorithm>
#include <cstring>
#include <new>
#include <string>
#include <vector>

#include "../../include/dmc.h"
#include "dmc_full.h"
#include "dmc_internal.h"

using dmc::align_up;

struct dmc_cache {
  dmc_cache_config cfg;
  dmc::Layout lay;
  char *ws;
  size_t ws_bytes;
  int device;
  int cu_count;
};

namespace {

thread_local std::string g_err;

dmc_status fail(dmc_status s, const char *fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  g_err = buf;
  return s;
}

dmc_status hip_fail(hipError_t e, const char *what) {
  return fail(DMC_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

bool pow2(int64_t x) { return x > 0 && (x & (x - 1)) == 0; }
int ilog2(int64_t x) {
  int r = 0;
  while ((int64_t(1) << r) < x) ++r;
  return r;
}
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

#ifndef DMC_DECODE_WG_PER_CU
#define DMC_DECODE_WG_PER_CU 2
#endif
// Persistent decode grid, counted in workgroups of 4 waves per compute unit
// (the vector-ALU launch packs them into 8-wave workgroups for bf16 caches
// with up to two query heads per kv head), and the largest number of waves a
// decode launch uses.
constexpr int kDecodeWgPerCu = DMC_DECODE_WG_PER_CU;
constexpr int64_t kMaxDecodeWaves = 8192;
constexpr size_t kMaxDecodeLds = 64 * 1024;
constexpr size_t kMaxLdsPerWorkgroup = 160 * 1024;   // gfx950

int elem_bytes(const dmc_cache_config &c) { return c.dtype == DMC_FP32 ? 4 : 2; }

// Units per entry of the decode kernel's slot-space table in LDS: 1 (every
// unit's offset) when that table fits beside the kernel's static LDS, else the
// smallest power of two that makes it fit (exact caches; windowed ones need
// 1); 0 if none up to kMaxSlotGroup does.
int slot_group_for(const dmc_cache_config &c) {
  const int64_t units = int64_t(c.batch) * c.num_kv_heads;
  const int G = c.num_q_heads / c.num_kv_heads;
  const bool v_trans = c.dtype == DMC_BF16 && G >= 4 && c.page_size == 32;
  // windowed caches decode with the full table only
  const int gmax = c.window > 0 ? 1 : dmc::kMaxSlotGroup;
  for (int g = 1; g <= gmax; g <<= 1) {
    const int entries = static_cast<int>((units + g - 1) / g + 1);
    const size_t dyn = dmc::decode_lds_bytes(entries, G, c.head_dim, c.window > 0);
    if (dyn <= kMaxDecodeLds &&
        dyn + dmc::decode_static_lds_bytes(c.head_dim, v_trans) <= kMaxLdsPerWorkgroup)
      return g;
  }
  return 0;
}

dmc_status validate_config(const dmc_cache_config *c) {
  if (!c) return fail(DMC_ERR_INVALID_ARG, "config is NULL");
  if (c->num_layers < 1 || c->batch < 1 || c->num_kv_heads < 1 || c->num_q_heads < 1)
    return fail(DMC_ERR_INVALID_ARG, "layers, batch and head counts must be >= 1");
  if (c->num_q_heads % c->num_kv_heads != 0)
    return fail(DMC_ERR_INVALID_ARG, "num_q_heads (%d) must be a multiple of num_kv_heads (%d)",
                c->num_q_heads, c->num_kv_heads);
  const int G = c->num_q_heads / c->num_kv_heads;
  if (G != 1 && G != 2 && G != 4 && G != 8)
    return fail(DMC_ERR_UNSUPPORTED, "query group size %d not in {1,2,4,8}", G);
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(DMC_ERR_UNSUPPORTED, "head_dim %d not in {64,128}", c->head_dim);
  if (c->dtype != DMC_BF16 && c->dtype != DMC_FP32)
    return fail(DMC_ERR_INVALID_ARG, "unknown dtype %d", c->dtype);
  if (!pow2(c->page_size) || c->page_size < 8 || c->page_size > 65536)
    return fail(DMC_ERR_UNSUPPORTED, "page_size %d must be a power of two in [8,65536]",
                c->page_size);
  if (c->max_slots_per_seq < 1)
    return fail(DMC_ERR_INVALID_ARG, "max_slots_per_seq must be >= 1");
  if (c->num_pages < 1 || c->num_pages >= (int64_t(1) << 31))
    return fail(DMC_ERR_INVALID_ARG, "num_pages %lld outside [1, 2^31)",
                static_cast<long long>(c->num_pages));
  if (!std::isfinite(c->decision_bias)) return fail(DMC_ERR_INVALID_ARG, "decision_bias not finite");
  if (c->omega_src != DMC_OMEGA_LEAD_QHEAD && c->omega_src != DMC_OMEGA_GROUP_MEAN &&
      c->omega_src != DMC_OMEGA_UNIFORM)
    return fail(DMC_ERR_INVALID_ARG, "unknown omega_src %d", c->omega_src);
  if (c->decision_src != DMC_DECISION_PER_HEAD && c->decision_src != DMC_DECISION_SHARED_LAYER)
    return fail(DMC_ERR_INVALID_ARG, "unknown decision_src %d", c->decision_src);
  if (c->window < 0) return fail(DMC_ERR_INVALID_ARG, "window must be >= 0");
  if (c->window > dmc::kMaxWindow)
    return fail(DMC_ERR_UNSUPPORTED, "window %d exceeds %d", c->window, dmc::kMaxWindow);
  if (c->split_tile < 0) return fail(DMC_ERR_INVALID_ARG, "split_tile must be >= 0");
  if (c->max_prompt_len < 0 || c->max_prompt_len > c->max_slots_per_seq)
    return fail(DMC_ERR_INVALID_ARG, "max_prompt_len must be in [0, max_slots_per_seq]");
  const int64_t units = int64_t(c->batch) * c->num_kv_heads;
  if (units > (int64_t(1) << 20)) return fail(DMC_ERR_UNSUPPORTED, "too many units per layer");
  if (slot_group_for(*c) == 0)
    return fail(DMC_ERR_UNSUPPORTED,
                "batch * num_kv_heads = %lld units exceed the decode kernel's LDS slot-space table "
                "(%s)", static_cast<long long>(units),
                c->window > 0 ? "a windowed cache keeps one entry per unit"
                              : "even at 64 units per entry");
  return DMC_OK;
}

dmc::Layout make_layout(const dmc_cache_config &c) {
  dmc::Layout L{};
  const int es = elem_bytes(c);
  L.units = c.batch * c.num_kv_heads;
  L.group = c.num_q_heads / c.num_kv_heads;
  L.maxpages = static_cast<int32_t>((int64_t(c.max_slots_per_seq) + c.page_size - 1) / c.page_size);
  L.split_tile = c.split_tile;
  {
    // ranges <= max(waves, ceil(S / split_tile)) with S <= U * max_slots; one
    // record per (range, unit) piece is indexed range + unit.
    const int64_t S = int64_t(L.units) * (c.max_slots_per_seq + dmc::kDecodeUnitOverhead);
    int64_t ranges = kMaxDecodeWaves;
    if (c.split_tile > 0) ranges = std::max<int64_t>(ranges, (S + c.split_tile - 1) / c.split_tile);
    L.max_records = ranges + L.units + 1;
  }
  L.max_prompt = c.max_prompt_len > 0 ? c.max_prompt_len : c.max_slots_per_seq;
  L.prompt_chunks = (L.max_prompt + 63) / 64;
  L.carry_blocks = (L.max_prompt + 31) / 32;
  L.window = c.window;
  L.slot_group = slot_group_for(c);
  L.page_bytes = int64_t(2) * c.page_size * c.head_dim * es;
  // Grouped-query caches decode on matrix cores with value pages transposed.
  L.v_trans = c.dtype == DMC_BF16 && L.group >= 4 && c.page_size == 32;
  const size_t U = size_t(L.units), NL = size_t(c.num_layers);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = align_up(off + bytes, 256);
    return at;
  };
  L.pool = take(size_t(c.num_pages) * size_t(L.page_bytes));
  L.ptab = take(NL * U * size_t(L.maxpages) * 4);
  L.lens = take(2 * NL * U * 4);
  L.z = take(NL * U * 4);
  L.ctrl = take(sizeof(dmc::Control));
  L.meta = take(U * 2 * 4);
  L.partials = take(size_t(L.max_records) * L.group * (c.head_dim + 4) * 4);
  L.pf_alpha = take(U * size_t(L.max_prompt));
  L.pf_omega = take(U * size_t(L.max_prompt) * 4);
  L.pf_count = take(U * size_t(L.prompt_chunks) * 4);
  L.pf_mask = take(U * size_t(L.prompt_chunks) * 8);
  L.pf_pagebase = take(U * 4);
  L.pf_carry = take(U * size_t(L.carry_blocks) * dmc::carry_stride(c.head_dim) * 4);
  L.win = take(NL * U * size_t(L.window) * 2 * c.head_dim * es);
  L.win_omega = take(NL * U * size_t(L.window) * 4);
  L.win_len = take(L.window > 0 ? NL * U * 4 : 0);
  L.total = off;
  return L;
}

// Runs the enqueue on the cache's device, restoring the caller's afterwards.
struct DeviceGuard {
  int prev = -1;
  bool ok = true;
  explicit DeviceGuard(int dev) {
    if (hipGetDevice(&prev) != hipSuccess) {
      ok = false;
      return;
    }
    if (prev != dev && hipSetDevice(dev) != hipSuccess) ok = false;
  }
  ~DeviceGuard() {
    int cur = -1;
    if (prev >= 0 && hipGetDevice(&cur) == hipSuccess && cur != prev) (void)hipSetDevice(prev);
  }
};

template <typename T>
T *at(const dmc_cache *c, size_t off) {
  return reinterpret_cast<T *>(c->ws + off);
}

// Lengths of one layer: buffer 0 holds the current slot counts (read by every
// kernel); buffer 1 receives the post-step counts of a decode step, which the
// step's combine launch copies back into buffer 0.  A decode call therefore
// always uses the same pair, and a captured call replays correctly.
int32_t *lens_of(const dmc_cache *c, int layer, int which) {
  return at<int32_t>(c, c->lay.lens) + (size_t(which) * c->cfg.num_layers + layer) * c->lay.units;
}

// Token-window ring of one layer (all null when the cache has no window).
dmc::WindowState window_of(const dmc_cache *c, int layer) {
  dmc::WindowState w{};
  const dmc::Layout &L = c->lay;
  w.window = L.window;
  if (L.window > 0) {
    const size_t units = size_t(L.units) * L.window;
    w.ring = c->ws + L.win + size_t(layer) * units * 2 * c->cfg.head_dim * elem_bytes(c->cfg);
    w.omega = at<float>(c, L.win_omega) + size_t(layer) * units;
    w.seg_len = at<int32_t>(c, L.win_len) + size_t(layer) * L.units;
  }
  return w;
}

dmc_status check_layer(const dmc_cache *c, int32_t layer) {
  if (!c) return fail(DMC_ERR_INVALID_ARG, "cache is NULL");
  if (layer < 0 || layer >= c->cfg.num_layers)
    return fail(DMC_ERR_INVALID_ARG, "layer %d outside [0, %d)", layer, c->cfg.num_layers);
  return DMC_OK;
}

dmc_status enqueue_reset(dmc_cache *c, hipStream_t s) {
  dmc::ResetParams p{};
  p.units = c->lay.units;
  p.all_units = p.units * c->cfg.num_layers;
  p.table = p.all_units * c->lay.maxpages;
  p.ptab = at<int32_t>(c, c->lay.ptab);
  p.lens = at<int32_t>(c, c->lay.lens);
  p.z = at<float>(c, c->lay.z);
  p.ctrl = at<dmc::Control>(c, c->lay.ctrl);
  p.meta = at<int32_t>(c, c->lay.meta);
  p.win_len = c->lay.window > 0 ? at<int32_t>(c, c->lay.win_len) : nullptr;
  const hipError_t e = dmc::launch_reset(p, s);
  return e == hipSuccess ? DMC_OK : hip_fail(e, "reset");
}

}  // namespace

extern "C" {

const char *dmc_last_error(void) { return g_err.c_str(); }

size_t dmc_cache_workspace_bytes(const dmc_cache_config *cfg) {
  if (validate_config(cfg) != DMC_OK) return 0;
  return make_layout(*cfg).total;
}

dmc_status dmc_cache_alloc(const dmc_cache_config *cfg, void *workspace, size_t bytes,
                           dmc_stream_t stream, dmc_cache **out) {
  if (!out) return fail(DMC_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  dmc_status st = validate_config(cfg);
  if (st != DMC_OK) return st;
  if (!workspace) return fail(DMC_ERR_INVALID_ARG, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(workspace) & 255u)
    return fail(DMC_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  const dmc::Layout lay = make_layout(*cfg);
  if (bytes < lay.total)
    return fail(DMC_ERR_INVALID_ARG, "workspace has %zu bytes, needs %zu", bytes, lay.total);
  int dev = 0, cus = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (e != hipSuccess) return hip_fail(e, "hipDeviceGetAttribute");
  dmc_cache *c = new (std::nothrow) dmc_cache();
  if (!c) return fail(DMC_ERR_INVALID_ARG, "out of host memory");
  c->cfg = *cfg;
  c->lay = lay;
  c->ws = static_cast<char *>(workspace);
  c->ws_bytes = bytes;
  c->device = dev;
  c->cu_count = cus > 0 ? cus : 256;
  // Set-up of dmc_decode_step_static: the device address of the library's
  // static scratch on this (current) device, resolved once per device.
  void *scratch = nullptr;
  e = dmc::static_scratch(&scratch);
  if (e != hipSuccess) {
    delete c;
    return hip_fail(e, "static scratch address");
  }
  st = enqueue_reset(c, static_cast<hipStream_t>(stream));
  if (st != DMC_OK) {
    delete c;
    return st;
  }
  *out = c;
  return DMC_OK;
}

dmc_status dmc_cache_free(dmc_cache *cache) {
  if (!cache) return fail(DMC_ERR_INVALID_ARG, "cache is NULL");
  delete cache;
  return DMC_OK;
}

dmc_status dmc_cache_reset(dmc_cache *cache, dmc_stream_t stream) {
  if (!cache) return fail(DMC_ERR_INVALID_ARG, "cache is NULL");
  DeviceGuard g(cache->device);
  if (!g.ok) return fail(DMC_ERR_HIP, "cannot select the cache's device");
  return enqueue_reset(cache, static_cast<hipStream_t>(stream));
}

namespace {

// Persistent decode grid of a cache: workgroups of 4 waves, kDecodeWgPerCu per
// compute unit (the matrix-core launch halves it when its LDS ring allows one;
// the vector-ALU launch may pack the same waves into larger workgroups).
int decode_grid(const dmc_cache *cache) {
  return static_cast<int>(
      std::min<int64_t>(int64_t(cache->cu_count) * kDecodeWgPerCu, kMaxDecodeWaves / 4));
}

// Shared checks and parameter set-up of the two decode entry points; the
// split-K records (partials, meta) are filled in by the caller.
dmc_status decode_params(dmc_cache *cache, int32_t layer, const void *q, const void *k,
                         const void *v, void *out, int32_t *slot_index, dmc::DecodeParams *out_p) {
  dmc_status st = check_layer(cache, layer);
  if (st != DMC_OK) return st;
  if (!q || !k || !v || !out) return fail(DMC_ERR_INVALID_ARG, "q, k, v and out must be non-NULL");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out))
    return fail(DMC_ERR_INVALID_ARG, "q, k, v and out must be 16-byte aligned");
  const dmc_cache_config &c = cache->cfg;
  const dmc::Layout &L = cache->lay;
  dmc::DecodeParams &p = *out_p;
  p = dmc::DecodeParams{};
  p.pool = cache->ws + L.pool;
  p.page_bytes = L.page_bytes;
  p.num_pages = c.num_pages;
  p.ptab = at<int32_t>(cache, L.ptab) + size_t(layer) * L.units * L.maxpages;
  p.len_in = lens_of(cache, layer, 0);
  p.len_out = lens_of(cache, layer, 1);
  p.z = at<float>(cache, L.z) + size_t(layer) * L.units;
  p.ctrl = at<dmc::Control>(cache, L.ctrl);
  p.q = q;
  p.k = k;
  p.v = v;
  p.out = out;
  p.slot_index = slot_index;
  p.win = window_of(cache, layer);
  p.c = c.decision_bias;
  p.scale_log2 = static_cast<float>(1.4426950408889634 / std::sqrt(double(c.head_dim)));
  p.units = L.units;
  p.hkv = c.num_kv_heads;
  p.hq = c.num_q_heads;
  p.compute_units = cache->cu_count;
  p.maxpages = L.maxpages;
  p.max_slots = c.max_slots_per_seq;
  p.log2p = ilog2(c.page_size);
  p.split_tile = L.split_tile;
  p.omega_src = c.omega_src;
  p.decision_src = c.decision_src;
  p.slot_group = L.slot_group;
  return DMC_OK;
}

dmc_status decode_launch(dmc_cache *cache, const dmc::DecodeParams &p, dmc_stream_t stream) {
  hipError_t e = dmc::launch_decode(elem_bytes(cache->cfg), cache->cfg.head_dim, cache->lay.group,
                                    cache->lay.v_trans, p, decode_grid(cache),
                                    static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "decode launch");
  return DMC_OK;
}

// Bytes of split-K records one decode launch of this cache can use: the
// per-unit table (first record, count) and one record of G x (d + 4) fp32 per
// (range, unit) piece, indexed range + unit.  Ranges are at most the launch's
// waves, or ceil(S / split_tile) with S <= units * (max_slots_per_seq + the
// decode kernels' virtual positions per unit).
size_t decode_records_bytes(const dmc_cache *cache, size_t *meta_bytes) {
  const dmc::Layout &L = cache->lay;
  int64_t ranges = int64_t(decode_grid(cache)) * 4;
  if (L.split_tile > 0) {
    const int64_t S = int64_t(L.units) * (cache->cfg.max_slots_per_seq + dmc::kDecodeUnitOverhead);
    ranges = std::max<int64_t>(ranges, (S + L.split_tile - 1) / L.split_tile);
  }
  *meta_bytes = align_up(size_t(L.units) * 2 * 4, 256);
  return *meta_bytes + size_t(ranges + L.units) * L.group * (cache->cfg.head_dim + 4) * 4;
}

}  // namespace

dmc_status dmc_decode_step(dmc_cache *cache, int32_t layer, const void *q, const void *k,
                           const void *v, void *out, int32_t *slot_index, dmc_stream_t stream) {
  dmc::DecodeParams p;
  dmc_status st = decode_params(cache, layer, q, k, v, out, slot_index, &p);
  if (st != DMC_OK) return st;
  p.partials = at<float>(cache, cache->lay.partials);
  p.meta = at<int32_t>(cache, cache->lay.meta);
  DeviceGuard g(cache->device);
  if (!g.ok) return fail(DMC_ERR_HIP, "cannot select the cache's device");
  return decode_launch(cache, p, stream);
}

dmc_status dmc_decode_step_static(dmc_cache *cache, int32_t layer, const void *q, const void *k,
                                  const void *v, void *out, int32_t *slot_index,
                                  dmc_stream_t stream) {
  dmc::DecodeParams p;
  dmc_status st = decode_params(cache, layer, q, k, v, out, slot_index, &p);
  if (st != DMC_OK) return st;
  size_t meta_bytes = 0;
  const size_t need = decode_records_bytes(cache, &meta_bytes);
  if (need > dmc::kStaticScratchBytes)
    return fail(DMC_ERR_UNSUPPORTED,
                "decode records of this cache need %zu bytes, more than the %zu-byte static "
                "scratch of dmc_decode_step_static (use dmc_decode_step)",
                need, dmc::kStaticScratchBytes);
  DeviceGuard g(cache->device);
  if (!g.ok) return fail(DMC_ERR_HIP, "cannot select the cache's device");
  char *scratch = nullptr;
  hipError_t e = dmc::static_scratch(reinterpret_cast<void **>(&scratch));
  if (e != hipSuccess) return hip_fail(e, "static scratch address");
  p.meta = reinterpret_cast<int32_t *>(scratch);
  p.partials = reinterpret_cast<float *>(scratch + meta_bytes);
  return decode_launch(cache, p, stream);
}

namespace {

// Shared argument checks and parameter set-up of the two prompt entry points.
dmc_status prefill_params(dmc_cache *cache, int32_t layer, const void *k, const int64_t k_strides[3],
                          const void *v, const int64_t v_strides[3], const void *q,
                          const int64_t q_strides[3], int32_t n, const int32_t *prompt_lens,
                          int32_t *slot_index, bool full_q, dmc::PrefillParams *out) {
  dmc_status st = check_layer(cache, layer);
  if (st != DMC_OK) return st;
  const dmc_cache_config &c = cache->cfg;
  const dmc::Layout &L = cache->lay;
  if (n < 0 || n > L.max_prompt)
    return fail(DMC_ERR_INVALID_ARG, "prompt length %d outside [0, %d]", n, L.max_prompt);
  if (n > 0) {
    if (!k || !v || !q) return fail(DMC_ERR_INVALID_ARG, "k, v and q must be non-NULL");
    if (!k_strides || !v_strides || !q_strides)
      return fail(DMC_ERR_INVALID_ARG, "stride arrays must be non-NULL");
    if (!aligned16(k) || !aligned16(v))
      return fail(DMC_ERR_INVALID_ARG, "k and v must be 16-byte aligned");
    if (full_q && !aligned16(q)) return fail(DMC_ERR_INVALID_ARG, "q must be 16-byte aligned");
    for (int i = 0; i < 3; ++i) {
      if (k_strides[i] < 0 || v_strides[i] < 0 || q_strides[i] < 0)
        return fail(DMC_ERR_INVALID_ARG, "strides must be non-negative");
      if (k_strides[i] % 8 || v_strides[i] % 8)
        return fail(DMC_ERR_INVALID_ARG, "k and v strides must be multiples of 8 elements");
      if (full_q && q_strides[i] % 8)
        return fail(DMC_ERR_INVALID_ARG, "q strides must be multiples of 8 elements");
    }
    // the compaction addresses up to 64 consecutive tokens from one base with
    // 32-bit offsets
    const int64_t es = c.dtype == DMC_FP32 ? 4 : 2, lim = int64_t(1) << 25;
    if (k_strides[1] * es >= lim || v_strides[1] * es >= lim || q_strides[1] * es >= lim)
      return fail(DMC_ERR_UNSUPPORTED, "k, v and q token strides must be below 32 MiB");
  }
  dmc::PrefillParams &p = *out;
  p = dmc::PrefillParams{};
  p.pool = cache->ws + L.pool;
  p.page_bytes = L.page_bytes;
  p.num_pages = c.num_pages;
  p.ptab = at<int32_t>(cache, L.ptab) + size_t(layer) * L.units * L.maxpages;
  p.len = lens_of(cache, layer, 0);
  p.z = at<float>(cache, L.z) + size_t(layer) * L.units;
  p.ctrl = at<dmc::Control>(cache, L.ctrl);
  p.k = k;
  p.v = v;
  p.q = q;
  for (int i = 0; i < 3; ++i) {
    p.ks[i] = n > 0 ? k_strides[i] : 0;
    p.vs[i] = n > 0 ? v_strides[i] : 0;
    p.qs[i] = n > 0 ? q_strides[i] : 0;
  }
  p.prompt_lens = prompt_lens;
  p.slot_index = slot_index;
  p.alpha = at<uint8_t>(cache, L.pf_alpha);
  p.omega = at<float>(cache, L.pf_omega);
  p.count = at<int32_t>(cache, L.pf_count);
  p.mask = at<uint64_t>(cache, L.pf_mask);
  p.page_base = at<int32_t>(cache, L.pf_pagebase);
  p.carry = nullptr;
  p.win = window_of(cache, layer);
  p.c = c.decision_bias;
  p.n = n;
  p.units = L.units;
  p.hkv = c.num_kv_heads;
  p.hq = c.num_q_heads;
  p.maxpages = L.maxpages;
  p.log2p = ilog2(c.page_size);
  p.omega_src = c.omega_src;
  p.decision_src = c.decision_src;
  p.max_prompt = L.max_prompt;
  p.prompt_chunks = L.prompt_chunks;
  p.carry_blocks = L.carry_blocks;
  return DMC_OK;
}

}  // namespace

dmc_status dmc_prefill_compress(dmc_cache *cache, int32_t layer, const void *k,
                                const int64_t k_strides[3], const void *v,
                                const int64_t v_strides[3], const void *q,
                                const int64_t q_strides[3], int32_t n,
                                const int32_t *prompt_lens, int32_t *slot_index,
                                dmc_stream_t stream) {
  dmc::PrefillParams p;
  dmc_status st = prefill_params(cache, layer, k, k_strides, v, v_strides, q, q_strides, n,
                                 prompt_lens, slot_index, false, &p);
  if (st != DMC_OK) return st;
  DeviceGuard g(cache->device);
  if (!g.ok) return fail(DMC_ERR_HIP, "cannot select the cache's device");
  hipError_t e = dmc::launch_prefill(elem_bytes(cache->cfg), cache->cfg.head_dim, cache->lay.v_trans,
                                     p, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "prefill launch");
  return DMC_OK;
}

dmc_status dmc_prefill_attend(dmc_cache *cache, int32_t layer, const void *k,
                              const int64_t k_strides[3], const void *v,
                              const int64_t v_strides[3], const void *q,
                              const int64_t q_strides[3], int32_t n,
                              const int32_t *prompt_lens, void *out,
                              const int64_t out_strides[3], int32_t *slot_index,
                              dmc_stream_t stream) {
  dmc::PrefillParams p;
  dmc_status st = prefill_params(cache, layer, k, k_strides, v, v_strides, q, q_strides, n,
                                 prompt_lens, slot_index, true, &p);
  if (st != DMC_OK) return st;
  if (n > 0) {
    if (!out || !out_strides) return fail(DMC_ERR_INVALID_ARG, "out and out_strides must be non-NULL");
    if (!aligned16(out)) return fail(DMC_ERR_INVALID_ARG, "out must be 16-byte aligned");
    for (int i = 0; i < 3; ++i)
      if (out_strides[i] < 0 || out_strides[i] % 8)
        return fail(DMC_ERR_INVALID_ARG, "out strides must be non-negative multiples of 8");
  }
  const dmc_cache_config &c = cache->cfg;
  const dmc::Layout &L = cache->lay;
  if (c.dtype == DMC_BF16 && (int64_t(n) + c.page_size - 1) / c.page_size > dmc::kPromptMaxPages)
    return fail(DMC_ERR_UNSUPPORTED, "prompt of %d tokens exceeds %d pages per unit", n,
                dmc::kPromptMaxPages);
  // Windowed open states need no carry records (they span at most w tokens).
  p.carry = L.window > 0 ? nullptr : at<float>(cache, L.pf_carry);
  dmc::PromptParams a{};
  a.pool = p.pool;
  a.page_bytes = p.page_bytes;
  a.ptab = p.ptab;
  a.q = q;
  a.k = k;
  a.v = v;
  for (int i = 0; i < 3; ++i) {
    a.qs[i] = p.qs[i];
    a.ks[i] = p.ks[i];
    a.vs[i] = p.vs[i];
    a.os[i] = n > 0 ? out_strides[i] : 0;
  }
  a.out = out;
  a.prompt_lens = prompt_lens;
  a.alpha = p.alpha;
  a.omega = p.omega;
  a.count = p.count;
  a.page_base = p.page_base;
  a.carry = p.carry;
  a.scale_log2 = static_cast<float>(1.4426950408889634 / std::sqrt(double(c.head_dim)));
  a.n = n;
  a.units = L.units;
  a.hkv = c.num_kv_heads;
  a.hq = c.num_q_heads;
  a.maxpages = L.maxpages;
  a.log2p = p.log2p;
  a.max_prompt = L.max_prompt;
  a.prompt_chunks = L.prompt_chunks;
  a.carry_blocks = L.carry_blocks;
  a.window = L.window;
  DeviceGuard g(cache->device);
  if (!g.ok) return fail(DMC_ERR_HIP, "cannot select the cache's device");
  const hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e = dmc::launch_prefill(elem_bytes(c), c.head_dim, L.v_trans, p, s);
  if (e != hipSuccess) return hip_fail(e, "prefill launch");
  e = dmc::launch_prompt_attend(elem_bytes(c), c.head_dim, L.group, L.v_trans, a, p.ctrl, s);
  if (e != hipSuccess) return hip_fail(e, "prompt attention launch");
  return DMC_OK;
}

dmc_status dmc_cache_lengths(const dmc_cache *cache, int32_t layer, int32_t *lengths,
                             dmc_stream_t stream) {
  dmc_status st = check_layer(cache, layer);
  if (st != DMC_OK) return st;
  if (!lengths) return fail(DMC_ERR_INVALID_ARG, "lengths is NULL");
  DeviceGuard g(cache->device);
  if (!g.ok) return fail(DMC_ERR_HIP, "cannot select the cache's device");
  hipError_t e = dmc::launch_copy_i32(lengths, lens_of(cache, layer, 0),
                                      cache->lay.units, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "lengths copy");
  return DMC_OK;
}

static dmc::DenseParams dense_params(const dmc_cache *cache, int32_t layer, int32_t dense_slots) {
  const dmc::Layout &L = cache->lay;
  dmc::DenseParams p{};
  p.pool = cache->ws + L.pool;
  p.page_bytes = L.page_bytes;
  p.num_pages = cache->cfg.num_pages;
  p.ptab = at<int32_t>(cache, L.ptab) + size_t(layer) * L.units * L.maxpages;
  p.len = lens_of(cache, layer, 0);
  p.z = at<float>(cache, L.z) + size_t(layer) * L.units;
  p.ctrl = at<dmc::Control>(cache, L.ctrl);
  p.page_base = at<int32_t>(cache, L.pf_pagebase);
  p.dense_slots = dense_slots;
  p.units = L.units;
  p.maxpages = L.maxpages;
  p.log2p = ilog2(cache->cfg.page_size);
  p.max_slots = cache->cfg.max_slots_per_seq;
  return p;
}

dmc_status dmc_cache_export(const dmc_cache *cache, int32_t layer, void *k_dense, void *v_dense,
                            int32_t dense_slots, float *z, dmc_stream_t stream) {
  dmc_status st = check_layer(cache, layer);
  if (st != DMC_OK) return st;
  if (dense_slots < 0) return fail(DMC_ERR_INVALID_ARG, "dense_slots must be >= 0");
  if (!z || (dense_slots > 0 && (!k_dense || !v_dense)))
    return fail(DMC_ERR_INVALID_ARG, "k_dense, v_dense and z must be non-NULL");
  if (!aligned16(k_dense) || !aligned16(v_dense))
    return fail(DMC_ERR_INVALID_ARG, "dense tensors must be 16-byte aligned");
  dmc::DenseParams p = dense_params(cache, layer, dense_slots);
  p.kd = k_dense;
  p.vd = v_dense;
  p.z_out = z;
  DeviceGuard g(cache->device);
  if (!g.ok) return fail(DMC_ERR_HIP, "cannot select the cache's device");
  hipError_t e = dmc::launch_export(elem_bytes(cache->cfg), cache->cfg.head_dim, cache->lay.v_trans, p,
                                    static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "export launch");
  return DMC_OK;
}

dmc_status dmc_cache_import(dmc_cache *cache, int32_t layer, const void *k_dense,
                            const void *v_dense, int32_t dense_slots, const int32_t *lengths,
                            const float *z, dmc_stream_t stream) {
  dmc_status st = check_layer(cache, layer);
  if (st != DMC_OK) return st;
  if (dense_slots < 0) return fail(DMC_ERR_INVALID_ARG, "dense_slots must be >= 0");
  if (!lengths || !z || (dense_slots > 0 && (!k_dense || !v_dense)))
    return fail(DMC_ERR_INVALID_ARG, "k_dense, v_dense, lengths and z must be non-NULL");
  if (!aligned16(k_dense) || !aligned16(v_dense))
    return fail(DMC_ERR_INVALID_ARG, "dense tensors must be 16-byte aligned");
  if (cache->lay.window > 0)
    return fail(DMC_ERR_UNSUPPORTED,
                "a cache with a window keeps its open segments' raw tokens; slots cannot supply them");
  dmc::DenseParams p = dense_params(cache, layer, dense_slots);
  p.kd = const_cast<void *>(k_dense);
  p.vd = const_cast<void *>(v_dense);
  p.lengths_in = lengths;
  p.z_in = z;
  DeviceGuard g(cache->device);
  if (!g.ok) return fail(DMC_ERR_HIP, "cannot select the cache's device");
  hipError_t e = dmc::launch_import(elem_bytes(cache->cfg), cache->cfg.head_dim, cache->lay.v_trans, p,
                                    static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "import launch");
  return DMC_OK;
}

namespace {

dmc_status validate_train(const dmc_train_config *c) {
  if (!c) return fail(DMC_ERR_INVALID_ARG, "config is NULL");
  if (c->batch < 1 || c->seq_len < 1 || c->num_q_heads < 1 || c->num_kv_heads < 1)
    return fail(DMC_ERR_INVALID_ARG, "batch, seq_len and head counts must be >= 1");
  if (c->num_q_heads % c->num_kv_heads != 0)
    return fail(DMC_ERR_INVALID_ARG, "num_q_heads (%d) must be a multiple of num_kv_heads (%d)",
                c->num_q_heads, c->num_kv_heads);
  const int G = c->num_q_heads / c->num_kv_heads;
  if (G != 1 && G != 2 && G != 4 && G != 8)
    return fail(DMC_ERR_UNSUPPORTED, "query group size %d not in {1,2,4,8}", G);
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(DMC_ERR_UNSUPPORTED, "head_dim %d not in {64,128}", c->head_dim);
  if (c->dtype != DMC_BF16 && c->dtype != DMC_FP32)
    return fail(DMC_ERR_INVALID_ARG, "unknown dtype %d", c->dtype);
  if (!std::isfinite(c->decision_bias)) return fail(DMC_ERR_INVALID_ARG, "decision_bias not finite");
  if (!(c->temperature > 0.0f) || !std::isfinite(c->temperature))
    return fail(DMC_ERR_INVALID_ARG, "temperature must be a finite value > 0");
  if (c->window < 1 || c->window > dmc::kMaxWindow)
    return fail(DMC_ERR_INVALID_ARG, "training window %d outside [1, %d]", c->window, dmc::kMaxWindow);
  if (c->omega_src != DMC_OMEGA_LEAD_QHEAD && c->omega_src != DMC_OMEGA_UNIFORM)
    return fail(DMC_ERR_UNSUPPORTED, "training omega_src must be LEAD_QHEAD or UNIFORM");
  const int64_t rows = int64_t(c->batch) * c->seq_len * c->num_q_heads;
  if (rows > (int64_t(1) << 31) / c->head_dim)
    return fail(DMC_ERR_UNSUPPORTED, "tensors larger than 2^31 elements");
  return DMC_OK;
}

int train_elem_bytes(const dmc_train_config &c) { return c.dtype == DMC_FP32 ? 4 : 2; }

// Device that holds a buffer, for entry points whose configuration names none.
dmc_status memory_device(const void *ptr, const char *what, int *dev) {
  hipPointerAttribute_t attr{};
  hipError_t e = hipPointerGetAttributes(&attr, ptr);
  if (e != hipSuccess) return hip_fail(e, "hipPointerGetAttributes");
  if (attr.type != hipMemoryTypeDevice)
    return fail(DMC_ERR_INVALID_ARG, "%s is not device memory", what);
  *dev = attr.device;
  return DMC_OK;
}

dmc::TrainLayout train_layout_of(const dmc_train_config &c) {
  return dmc::train_layout(c.batch, c.seq_len, c.num_q_heads, c.num_kv_heads, c.head_dim,
                           train_elem_bytes(c), c.window);
}

// Common checks and parameter set-up of the two training entry points.
dmc_status train_params(const dmc_train_config *cfg, const void *q, const void *k, const void *v,
                        const float *noise, void *ws, size_t bytes, dmc::TrainParams *p) {
  dmc_status st = validate_train(cfg);
  if (st != DMC_OK) return st;
  if (!q || !k || !v || !noise || !ws)
    return fail(DMC_ERR_INVALID_ARG, "q, k, v, noise and workspace must be non-NULL");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v))
    return fail(DMC_ERR_INVALID_ARG, "q, k and v must be 16-byte aligned");
  if (reinterpret_cast<uintptr_t>(ws) & 255u)
    return fail(DMC_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  const dmc::TrainLayout L = train_layout_of(*cfg);
  if (bytes < L.total)
    return fail(DMC_ERR_INVALID_ARG, "workspace has %zu bytes, needs %zu", bytes, L.total);
  char *w = static_cast<char *>(ws);
  *p = dmc::TrainParams{};
  p->q = q;
  p->k = k;
  p->v = v;
  p->noise = noise;
  p->ks = w + L.ks;
  p->vs = w + L.vs;
  p->alpha = reinterpret_cast<float *>(w + L.alpha);
  p->omega = reinterpret_cast<float *>(w + L.omega);
  p->z = reinterpret_cast<float *>(w + L.z);
  p->mask = reinterpret_cast<float *>(w + L.mask);
  p->lse = reinterpret_cast<float *>(w + L.lse);
  p->dsum = reinterpret_cast<float *>(w + L.dsum);
  p->dks = reinterpret_cast<float *>(w + L.dks);
  p->dvs = reinterpret_cast<float *>(w + L.dvs);
  p->dmask = reinterpret_cast<float *>(w + L.dmask);
  p->qs = reinterpret_cast<float *>(w + L.qs);
  p->e = reinterpret_cast<float *>(w + L.e);
  p->c = cfg->decision_bias;
  p->tau = cfg->temperature;
  p->scale_log2 = static_cast<float>(1.4426950408889634 / std::sqrt(double(cfg->head_dim)));
  p->batch = cfg->batch;
  p->n = cfg->seq_len;
  p->hq = cfg->num_q_heads;
  p->hkv = cfg->num_kv_heads;
  p->window = cfg->window;
  p->omega_src = cfg->omega_src;
  return DMC_OK;
}

}  // namespace

size_t dmc_train_workspace_bytes(const dmc_train_config *cfg) {
  if (validate_train(cfg) != DMC_OK) return 0;
  return train_layout_of(*cfg).total;
}

dmc_status dmc_train_forward(const dmc_train_config *cfg, const void *q, const void *k,
                             const void *v, const float *noise, void *out, float *alpha,
                             void *ws, size_t bytes, dmc_stream_t stream) {
  dmc::TrainParams p;
  dmc_status st = train_params(cfg, q, k, v, noise, ws, bytes, &p);
  if (st != DMC_OK) return st;
  if (!out) return fail(DMC_ERR_INVALID_ARG, "out must be non-NULL");
  if (!aligned16(out)) return fail(DMC_ERR_INVALID_ARG, "out must be 16-byte aligned");
  p.out = out;
  p.alpha_out = alpha;
  int dev = 0;
  st = memory_device(ws, "the workspace", &dev);
  if (st != DMC_OK) return st;
  DeviceGuard g(dev);   // enqueue on the workspace's device, restoring the caller's
  if (!g.ok) return fail(DMC_ERR_HIP, "cannot select the workspace's device");
  hipError_t e = dmc::launch_train_forward(train_elem_bytes(*cfg), cfg->head_dim,
                                           cfg->num_q_heads / cfg->num_kv_heads, p,
                                           static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "training forward launch");
  return DMC_OK;
}

dmc_status dmc_train_backward(const dmc_train_config *cfg, const void *q, const void *k,
                              const void *v, const float *noise, const void *out,
                              const void *dout, const float *dalpha, void *dq, void *dk, void *dv,
                              void *ws, size_t bytes, dmc_stream_t stream) {
  dmc::TrainParams p;
  dmc_status st = train_params(cfg, q, k, v, noise, ws, bytes, &p);
  if (st != DMC_OK) return st;
  if (!out || !dout || !dq || !dk || !dv)
    return fail(DMC_ERR_INVALID_ARG, "out, dout, dq, dk and dv must be non-NULL");
  if (!aligned16(out) || !aligned16(dout) || !aligned16(dq) || !aligned16(dk) || !aligned16(dv))
    return fail(DMC_ERR_INVALID_ARG, "out, dout, dq, dk and dv must be 16-byte aligned");
  p.out = const_cast<void *>(out);
  p.dout = dout;
  p.dalpha = dalpha;
  p.dq = dq;
  p.dk = dk;
  p.dv = dv;
  int dev = 0;
  st = memory_device(ws, "the workspace", &dev);
  if (st != DMC_OK) return st;
  DeviceGuard g(dev);
  if (!g.ok) return fail(DMC_ERR_HIP, "cannot select the workspace's device");
  hipError_t e = dmc::launch_train_backward(train_elem_bytes(*cfg), cfg->head_dim,
                                            cfg->num_q_heads / cfg->num_kv_heads, p,
                                            static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "training backward launch");
  return DMC_OK;
}

// A packed tensor [rows, heads, d]: pointer and strides.  An input that is read
// 32 tokens from one base has bounded token strides; an output's rows may not
// overlap.
struct Packed {
  const char *name;
  const void *ptr;
  const int64_t *st;
  int32_t heads;
  bool bounded, output;
};

static dmc_status check_packed(const Packed &t, int64_t rows, int head_dim, int es) {
  if (!t.ptr || !t.st) return fail(DMC_ERR_INVALID_ARG, "%s and its strides must be non-NULL", t.name);
  if (!aligned16(t.ptr)) return fail(DMC_ERR_INVALID_ARG, "%s must be 16-byte aligned", t.name);
  for (int i = 0; i < 2; ++i)
    if (t.st[i] < 0 || t.st[i] % 8)
      return fail(DMC_ERR_INVALID_ARG, "%s strides must be non-negative multiples of 8", t.name);
  // (divided, not multiplied: strides may be anything)
  if (t.bounded && t.st[0] >= (int64_t(1) << 25) / es)
    return fail(DMC_ERR_UNSUPPORTED, "%s token stride must be below 32 MiB", t.name);
  const int64_t far = (int64_t(1) << 58) / (rows + t.heads);
  if (t.st[0] > far || t.st[1] > far)
    return fail(DMC_ERR_INVALID_ARG, "%s strides exceed the address space", t.name);
  if (t.output && rows > 1 && t.st[0] < t.st[1] * (t.heads - 1) + head_dim &&
      (t.heads == 1 || t.st[1] < t.st[0] * (rows - 1) + head_dim || t.st[0] < head_dim))
    return fail(DMC_ERR_INVALID_ARG, "the rows of %s overlap", t.name);
  if (t.output && t.heads > 1 && t.st[1] < head_dim)
    return fail(DMC_ERR_INVALID_ARG, "the rows of %s overlap", t.name);
  return DMC_OK;
}

constexpr int32_t kMaxPackedTokens = 1 << 28;

static dmc_status validate_causal(const dmc_causal_config *c) {
  if (!c) return fail(DMC_ERR_INVALID_ARG, "config is NULL");
  if (c->num_q_heads < 1 || c->num_kv_heads < 1)
    return fail(DMC_ERR_INVALID_ARG, "head counts must be >= 1");
  if (c->num_q_heads % c->num_kv_heads != 0)
    return fail(DMC_ERR_INVALID_ARG, "num_q_heads (%d) must be a multiple of num_kv_heads (%d)",
                c->num_q_heads, c->num_kv_heads);
  if (c->num_q_heads > 4096) return fail(DMC_ERR_UNSUPPORTED, "more than 4096 query heads");
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(DMC_ERR_UNSUPPORTED, "head_dim %d not in {64,128}", c->head_dim);
  if (c->dtype != DMC_BF16 && c->dtype != DMC_FP32)
    return fail(DMC_ERR_INVALID_ARG, "unknown dtype %d", c->dtype);
  return DMC_OK;
}

static dmc_status check_packed_counts(int32_t num_seqs, int32_t total) {
  if (total < 0 || num_seqs < 0) return fail(DMC_ERR_INVALID_ARG, "token and sequence counts must be >= 0");
  if (total > kMaxPackedTokens || num_seqs > kMaxPackedTokens)
    return fail(DMC_ERR_UNSUPPORTED, "more than %d tokens or sequences", kMaxPackedTokens);
  return DMC_OK;
}

static size_t causal_stats_bytes(const dmc_causal_config &c, int32_t total) {
  return align_up(size_t(c.num_q_heads) * (size_t(total) + 32) * 8, 256);
}
// Bytes of `parts` parts of `heads` rows of `floats` for each of `total` tokens.
static size_t causal_part_bytes(int32_t total, int parts, int heads, int floats) {
  return parts > 1 ? align_up(size_t(parts) * total * heads * floats * 4, 256) : 0;
}
// The most of that for up to `total` tokens in any number of sequences: fewer tokens
// may be cut into more parts, but parts times tiles stay within `places`.
static size_t causal_most_part_bytes(int32_t total, int max_parts, int places, int tile, int heads, int floats) {
  size_t most = 0;
  for (int parts = 2; parts <= max_parts; ++parts) {
    const int64_t tokens = std::min<int64_t>(total, places / (int64_t(parts) * heads) * tile);
    if (tokens > 0) most = std::max(most, causal_part_bytes(static_cast<int32_t>(tokens), parts, heads, floats));
  }
  return most;
}
static size_t causal_workspace(const dmc_causal_config &c, int32_t total) {
  const bool bf16 = c.dtype == DMC_BF16;
  return causal_stats_bytes(c, total) +
         2 * causal_most_part_bytes(total, dmc::kMaxKeyParts, dmc::kPartPlaces, bf16 ? 128 : 32, c.num_kv_heads,
                                    c.head_dim) +
         (bf16 ? causal_most_part_bytes(total, dmc::kMaxQueryParts, dmc::kQueryPartPlaces, 128, c.num_q_heads,
                                        c.head_dim + 4)
               : 0);
}

static void copy_strides(int64_t (&dst)[2], const int64_t *src) {
  dst[0] = src[0];
  dst[1] = src[1];
}

static void causal_params(const dmc_causal_config &c, const int32_t *cu, int32_t seqs, int32_t total, void *ws,
                          dmc::CausalParams *p) {
  p->cu = cu;
  p->seqs = seqs;
  p->total = total;
  p->hq = c.num_q_heads;
  p->hkv = c.num_kv_heads;
  p->stat_stride = int64_t(total) + 32;
  p->scale_log2 = static_cast<float>(1.4426950408889634 / std::sqrt(double(c.head_dim)));
  const dmc::CausalParts parts = dmc::causal_parts(c.dtype == DMC_FP32 ? 4 : 2, c.num_q_heads, c.num_kv_heads, seqs, total);
  p->parts = parts.keys;
  p->query_parts = parts.queries;
  char *w = static_cast<char *>(ws);
  const size_t keys = causal_part_bytes(total, parts.keys, c.num_kv_heads, c.head_dim);
  p->stats = reinterpret_cast<float *>(w);
  w += causal_stats_bytes(c, total);
  p->part_k = reinterpret_cast<float *>(w);
  p->part_v = reinterpret_cast<float *>(w + keys);
  p->part_q = reinterpret_cast<float *>(w + 2 * keys);
}

// Checks of the workspace of a causal call.
static dmc_status check_causal_workspace(const dmc_causal_config &c, int32_t total, const void *ws, size_t bytes) {
  if (!ws) return fail(DMC_ERR_INVALID_ARG, "workspace must be non-NULL");
  if (reinterpret_cast<uintptr_t>(ws) & 255u)
    return fail(DMC_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  if (bytes < causal_workspace(c, total))
    return fail(DMC_ERR_INVALID_ARG, "workspace has %zu bytes, needs %zu", bytes, causal_workspace(c, total));
  return DMC_OK;
}

// Whether a launch with one workgroup per head and tile (of at least 32 tokens) fits a grid.
static bool causal_grid_fits(const dmc_causal_config &c, int32_t seqs, int32_t total) {
  const int64_t tiles = int64_t(total) / 32 + seqs;
  return tiles * c.num_q_heads <= 0x7fffffff;
}

size_t dmc_causal_workspace_bytes(const dmc_causal_config *cfg, int32_t total) {
  if (validate_causal(cfg) != DMC_OK || check_packed_counts(0, total) != DMC_OK) return 0;
  return causal_workspace(*cfg, total);
}

dmc_status dmc_causal_forward(const dmc_causal_config *cfg, const void *q, const int64_t q_strides[2],
                              const void *k, const int64_t k_strides[2], const void *v,
                              const int64_t v_strides[2], const int32_t *cu, int32_t num_seqs,
                              int32_t total, void *out, const int64_t out_strides[2], float *lse,
                              void *ws, size_t bytes, dmc_stream_t stream) {
  dmc_status st = validate_causal(cfg);
  if (st == DMC_OK) st = check_packed_counts(num_seqs, total);
  if (st != DMC_OK) return st;
  if (total == 0 || num_seqs == 0) return DMC_OK;
  const int es = cfg->dtype == DMC_FP32 ? 4 : 2, hq = cfg->num_q_heads, hkv = cfg->num_kv_heads;
  const Packed tensors[] = {{"q", q, q_strides, hq, true, false},
                            {"k", k, k_strides, hkv, true, false},
                            {"v", v, v_strides, hkv, true, false},
                            {"out", out, out_strides, hq, false, true}};
  for (const Packed &t : tensors) {
    st = check_packed(t, total, cfg->head_dim, es);
    if (st != DMC_OK) return st;
  }
  if (!cu || !lse) return fail(DMC_ERR_INVALID_ARG, "cu_seqlens and lse must be non-NULL");
  st = check_causal_workspace(*cfg, total, ws, bytes);
  if (st != DMC_OK) return st;
  if (!causal_grid_fits(*cfg, num_seqs, total))
    return fail(DMC_ERR_UNSUPPORTED, "too many tokens and sequences for one launch");
  dmc::CausalParams p{};
  causal_params(*cfg, cu, num_seqs, total, ws, &p);
  p.q = q;
  p.k = k;
  p.v = v;
  p.out = out;
  p.lse = lse;
  copy_strides(p.qs, q_strides);
  copy_strides(p.ks, k_strides);
  copy_strides(p.vs, v_strides);
  copy_strides(p.os, out_strides);
  int dev = 0;
  st = memory_device(ws, "the workspace", &dev);
  if (st != DMC_OK) return st;
  DeviceGuard g(dev);
  if (!g.ok) return fail(DMC_ERR_HIP, "cannot select the tensors' device");
  hipError_t e = dmc::launch_causal_forward(es, cfg->head_dim, p, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "causal forward launch");
  return DMC_OK;
}

dmc_status dmc_causal_backward(const dmc_causal_config *cfg, const void *q, const int64_t q_strides[2],
                               const void *k, const int64_t k_strides[2], const void *v,
                               const int64_t v_strides[2], const int32_t *cu, int32_t num_seqs,
                               int32_t total, const void *out, const int64_t out_strides[2],
                               const float *lse, const void *dout, const int64_t dout_strides[2],
                               void *dq, const int64_t dq_strides[2], void *dk,
                               const int64_t dk_strides[2], void *dv, const int64_t dv_strides[2],
                               void *ws, size_t bytes, dmc_stream_t stream) {
  dmc_status st = validate_causal(cfg);
  if (st == DMC_OK) st = check_packed_counts(num_seqs, total);
  if (st != DMC_OK) return st;
  if (total == 0 || num_seqs == 0) return DMC_OK;
  const int es = cfg->dtype == DMC_FP32 ? 4 : 2, hq = cfg->num_q_heads, hkv = cfg->num_kv_heads;
  const Packed tensors[] = {{"q", q, q_strides, hq, true, false},
                            {"k", k, k_strides, hkv, true, false},
                            {"v", v, v_strides, hkv, true, false},
                            {"out", out, out_strides, hq, false, false},
                            {"dout", dout, dout_strides, hq, true, false},
                            {"dq", dq, dq_strides, hq, false, true},
                            {"dk", dk, dk_strides, hkv, false, true},
                            {"dv", dv, dv_strides, hkv, false, true}};
  for (const Packed &t : tensors) {
    st = check_packed(t, total, cfg->head_dim, es);
    if (st != DMC_OK) return st;
  }
  if (!cu || !lse) return fail(DMC_ERR_INVALID_ARG, "cu_seqlens and lse must be non-NULL");
  st = check_causal_workspace(*cfg, total, ws, bytes);
  if (st != DMC_OK) return st;
  if (!causal_grid_fits(*cfg, num_seqs, total))
    return fail(DMC_ERR_UNSUPPORTED, "too many tokens and sequences for one launch");
  dmc::CausalParams p{};
  causal_params(*cfg, cu, num_seqs, total, ws, &p);
  p.q = q;
  p.k = k;
  p.v = v;
  p.out = const_cast<void *>(out);
  p.lse = const_cast<float *>(lse);
  p.dout = dout;
  p.dq = dq;
  p.dk = dk;
  p.dv = dv;
  copy_strides(p.qs, q_strides);
  copy_strides(p.ks, k_strides);
  copy_strides(p.vs, v_strides);
  copy_strides(p.os, out_strides);
  copy_strides(p.dos, dout_strides);
  copy_strides(p.dqs, dq_strides);
  copy_strides(p.dks, dk_strides);
  copy_strides(p.dvs, dv_strides);
  int dev = 0;
  st = memory_device(ws, "the workspace", &dev);
  if (st != DMC_OK) return st;
  DeviceGuard g(dev);
  if (!g.ok) return fail(DMC_ERR_HIP, "cannot select the tensors' device");
  hipError_t e = dmc::launch_causal_backward(es, cfg->head_dim, p, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "causal backward launch");
  return DMC_OK;
}

// Workspace of the chunk calls: byte offsets of its sections (256-byte aligned).
struct ChunkLayout {
  size_t state_k, state_v, closed_k, closed_v, before, starts, carry, visible, unit_order, piece_base, pieces, record_base,
      old_len, old_z, partials, total;
};

static ChunkLayout chunk_layout(const dmc_cache *c, int32_t total) {
  const dmc_cache_config &cfg = c->cfg;
  const size_t es = elem_bytes(cfg), d = cfg.head_dim, H = cfg.num_kv_heads, U = c->lay.units, B = cfg.batch;
  const size_t blocks32 = size_t(total) / 32 + B, blocks64 = size_t(total) / 64 + B;
  ChunkLayout L{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = align_up(off + bytes, 256);
    return at;
  };
  L.state_k = take(H * total * d * es);
  L.state_v = take(H * total * d * es);
  L.closed_k = take(H * blocks32 * 32 * d * es);
  L.closed_v = take(H * blocks32 * 32 * d * es);
  L.before = take(H * total * 4);
  L.starts = take(H * blocks64 * 4);
  L.carry = take(H * blocks64 * dmc::carry_stride(cfg.head_dim) * 4);
  L.visible = take(U * 4);
  L.unit_order = take((U + 7) / 8 * 8 * 8 * 4);
  L.piece_base = take(((U + 7) / 8 + 1) * 8 * 4);
  L.pieces = take(U * 4);
  L.record_base = take(U * 4);
  L.old_len = take(U * 4);
  L.old_z = take(U * 4);
  // (wide tiles' records, which narrow ones fit as well)
  L.partials = take(size_t(4) * c->cu_count * (cfg.dtype == DMC_BF16 ? 128 : 32) * (d + 4) * 4);
  L.total = off;
  return L;
}

static dmc_status check_chunk_sizes(const dmc_cache *c, int32_t total, int32_t max_chunk) {
  if (!c) return fail(DMC_ERR_INVALID_ARG, "cache is NULL");
  if (c->lay.window > 0)
    return fail(DMC_ERR_UNSUPPORTED, "chunks on a cache with a window are not supported");
  if (total < 0) return fail(DMC_ERR_INVALID_ARG, "total_tokens must be >= 0");
  if (max_chunk < 1) return fail(DMC_ERR_INVALID_ARG, "max_chunk must be >= 1");
  if (total > (1 << 24)) return fail(DMC_ERR_UNSUPPORTED, "more than %d tokens in a call", 1 << 24);
  // grids: a workgroup per 64-token block or column tile (of 4 tokens or more) and kv head; heads in grid.y
  const int64_t tiles = int64_t(total) / 4 + c->cfg.batch;
  if (c->cfg.num_kv_heads > 65535 || tiles * c->cfg.num_kv_heads + 4 * c->cu_count > 0x7fffffff)
    return fail(DMC_ERR_UNSUPPORTED, "too many tokens, rows and heads for one launch");
  return DMC_OK;
}

// Checks and parameters that both chunk calls share.
static dmc_status chunk_params(const dmc_cache *c, int32_t layer, const void *k, const int64_t *k_strides, const void *v,
                               const int64_t *v_strides, const void *q, const int64_t *q_strides, const int32_t *cu,
                               int32_t total, int32_t max_chunk, void *ws, size_t bytes, dmc::ChunkParams *out) {
  dmc_status st = check_layer(c, layer);
  if (st == DMC_OK) st = check_chunk_sizes(c, total, max_chunk);
  if (st != DMC_OK) return st;
  const dmc_cache_config &cfg = c->cfg;
  const dmc::Layout &L = c->lay;
  const int es = elem_bytes(cfg);
  if (total > 0) {
    for (const Packed &t : {Packed{"k", k, k_strides, cfg.num_kv_heads, true, false},
                            Packed{"v", v, v_strides, cfg.num_kv_heads, true, false}}) {
      st = check_packed(t, total, cfg.head_dim, es);
      if (st != DMC_OK) return st;
    }
    if (!q || !q_strides) return fail(DMC_ERR_INVALID_ARG, "q and its strides must be non-NULL");
    if (q_strides[0] < 0 || q_strides[1] < 0) return fail(DMC_ERR_INVALID_ARG, "q strides must be non-negative");
    if (q_strides[0] >= (int64_t(1) << 25) / es || q_strides[1] > (int64_t(1) << 40))
      return fail(DMC_ERR_UNSUPPORTED, "q token stride must be below 32 MiB");
    if (!cu || !ws) return fail(DMC_ERR_INVALID_ARG, "cu_seqlens and workspace must be non-NULL");
    if (reinterpret_cast<uintptr_t>(ws) & 255u)
      return fail(DMC_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  }
  const ChunkLayout W = chunk_layout(c, total);
  if (total > 0 && bytes < W.total)
    return fail(DMC_ERR_INVALID_ARG, "workspace has %zu bytes, needs %zu", bytes, W.total);
  dmc::ChunkParams &p = *out;
  p = dmc::ChunkParams{};
  p.pool = c->ws + L.pool;
  p.page_bytes = L.page_bytes;
  p.num_pages = cfg.num_pages;
  p.ptab = at<int32_t>(c, L.ptab) + size_t(layer) * L.units * L.maxpages;
  p.len = lens_of(c, layer, 0);
  p.z = at<float>(c, L.z) + size_t(layer) * L.units;
  p.ctrl = at<dmc::Control>(c, L.ctrl);
  p.q = q;
  p.k = k;
  p.v = v;
  if (total > 0) {
    copy_strides(p.qs, q_strides);
    copy_strides(p.ks, k_strides);
    copy_strides(p.vs, v_strides);
  }
  p.cu = cu;
  char *w = static_cast<char *>(ws);
  p.state_k = w + W.state_k;
  p.state_v = w + W.state_v;
  p.closed_k = w + W.closed_k;
  p.closed_v = w + W.closed_v;
  p.before = reinterpret_cast<int32_t *>(w + W.before);
  p.starts = reinterpret_cast<int32_t *>(w + W.starts);
  p.carry = reinterpret_cast<float *>(w + W.carry);
  p.visible = reinterpret_cast<int32_t *>(w + W.visible);
  p.unit_order = reinterpret_cast<int32_t *>(w + W.unit_order);
  p.piece_base = reinterpret_cast<int32_t *>(w + W.piece_base);
  p.pieces = reinterpret_cast<int32_t *>(w + W.pieces);
  p.record_base = reinterpret_cast<int32_t *>(w + W.record_base);
  p.old_len = reinterpret_cast<int32_t *>(w + W.old_len);
  p.old_z = reinterpret_cast<float *>(w + W.old_z);
  p.partials = reinterpret_cast<float *>(w + W.partials);
  p.c = cfg.decision_bias;
  p.scale_log2 = static_cast<float>(1.4426950408889634 / std::sqrt(double(cfg.head_dim)));
  p.rows = cfg.batch;
  p.total = total;
  p.max_chunk = max_chunk;
  p.units = L.units;
  p.hq = cfg.num_q_heads;
  p.hkv = cfg.num_kv_heads;
  p.maxpages = L.maxpages;
  p.max_slots = cfg.max_slots_per_seq;
  p.log2p = ilog2(cfg.page_size);
  p.omega_src = cfg.omega_src;
  p.decision_src = cfg.decision_src;
  p.blocks64 = total / 64 + cfg.batch;
  p.blocks32 = total / 32 + cfg.batch;
  p.piece_min = dmc::kChunkPieceMin;
  return DMC_OK;
}

size_t dmc_chunk_workspace_bytes(const dmc_cache *cache, int32_t total, int32_t max_chunk) {
  if (check_chunk_sizes(cache, total, max_chunk) != DMC_OK) return 0;
  return chunk_layout(cache, total).total;
}

dmc_status dmc_chunk_attend(const dmc_cache *cache, int32_t layer, const void *q, const int64_t q_strides[2],
                            const void *k, const int64_t k_strides[2], const void *v, const int64_t v_strides[2],
                            const int32_t *cu, int32_t total, int32_t max_chunk, void *out,
                            const int64_t out_strides[2], void *ws, size_t bytes, dmc_stream_t stream) {
  dmc::ChunkParams p;
  dmc_status st = chunk_params(cache, layer, k, k_strides, v, v_strides, q, q_strides, cu, total, max_chunk, ws, bytes, &p);
  if (st != DMC_OK) return st;
  if (total == 0) return DMC_OK;
  const dmc_cache_config &c = cache->cfg;
  for (const Packed &t : {Packed{"q", q, q_strides, c.num_q_heads, true, false},
                          Packed{"out", out, out_strides, c.num_q_heads, false, true}}) {
    st = check_packed(t, total, c.head_dim, elem_bytes(c));
    if (st != DMC_OK) return st;
  }
  p.out = out;
  copy_strides(p.os, out_strides);
  const bool wide = dmc::chunk_wide(elem_bytes(c), cache->lay.group, max_chunk,
                                    int64_t(cache->lay.units) * c.max_slots_per_seq);
  p.tile_shift = dmc::chunk_tile_shift(cache->lay.group, wide);
  const dmc::ChunkSplit split = dmc::chunk_split(cache->cu_count, c.batch, c.num_kv_heads, cache->lay.group, c.max_slots_per_seq,
                                                 total, max_chunk, p.tile_shift, wide);
  p.fixed_parts = split.fixed_parts;
  p.piece_budget = split.piece_budget;
  DeviceGuard g(cache->device);
  if (!g.ok) return fail(DMC_ERR_HIP, "cannot select the cache's device");
  hipError_t e = dmc::launch_chunk_attend(elem_bytes(c), c.head_dim, cache->lay.group, cache->lay.v_trans, wide, p,
                                          static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "chunk attention launch");
  return DMC_OK;
}

dmc_status dmc_chunk_append(dmc_cache *cache, int32_t layer, const void *k, const int64_t k_strides[2],
                            const void *v, const int64_t v_strides[2], const void *q, const int64_t q_strides[2],
                            const int32_t *cu, const int32_t *accepted, int32_t total, int32_t max_chunk,
                            int32_t *slot_index, void *ws, size_t bytes, dmc_stream_t stream) {
  dmc::ChunkParams p;
  dmc_status st = chunk_params(cache, layer, k, k_strides, v, v_strides, q, q_strides, cu, total, max_chunk, ws, bytes, &p);
  if (st != DMC_OK) return st;
  if (total == 0) return DMC_OK;
  p.accepted = accepted;
  p.slot_index = slot_index;
  const dmc_cache_config &c = cache->cfg;
  DeviceGuard g(cache->device);
  if (!g.ok) return fail(DMC_ERR_HIP, "cannot select the cache's device");
  hipError_t e = dmc::launch_chunk_append(elem_bytes(c), c.head_dim, cache->lay.v_trans, p,
                                          static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "chunk append launch");
  return DMC_OK;
}

// Full caches and the position rotation.
static dmc_status validate_heads(int32_t hq, int32_t hkv, int32_t head_dim, int32_t dtype, int32_t rotary_dim,
                                 int32_t rotary_pairs) {
  if (hq < 1 || hkv < 1) return fail(DMC_ERR_INVALID_ARG, "head counts must be >= 1");
  if (hq > 4096 || hkv > 4096) return fail(DMC_ERR_UNSUPPORTED, "more than 4096 heads");
  if (head_dim != 64 && head_dim != 128) return fail(DMC_ERR_UNSUPPORTED, "head_dim %d not in {64,128}", head_dim);
  if (dtype != DMC_BF16 && dtype != DMC_FP32) return fail(DMC_ERR_INVALID_ARG, "unknown dtype %d", dtype);
  if (rotary_dim < 0 || rotary_dim > head_dim || rotary_dim % 16 != 0)
    return fail(DMC_ERR_INVALID_ARG, "rotary_dim %d is not a multiple of 16 in [0, %d]", rotary_dim, head_dim);
  if (rotary_pairs != DMC_PAIRS_HALVES && rotary_pairs != DMC_PAIRS_ADJACENT)
    return fail(DMC_ERR_INVALID_ARG, "unknown rotary_pairs %d", rotary_pairs);
  return DMC_OK;
}

static dmc_status validate_full(const dmc_full_config *c) {
  if (!c) return fail(DMC_ERR_INVALID_ARG, "config is NULL");
  dmc_status st = validate_heads(c->num_q_heads, c->num_kv_heads, c->head_dim, c->dtype, c->rotary_dim, c->rotary_pairs);
  if (st != DMC_OK) return st;
  if (c->num_q_heads % c->num_kv_heads != 0)
    return fail(DMC_ERR_INVALID_ARG, "num_q_heads (%d) must be a multiple of num_kv_heads (%d)",
                c->num_q_heads, c->num_kv_heads);
  if (c->batch < 1 || c->max_pages < 1 || c->num_pages < 1)
    return fail(DMC_ERR_INVALID_ARG, "batch, max_pages and num_pages must be >= 1");
  if (c->batch > 4096) return fail(DMC_ERR_UNSUPPORTED, "more than 4096 rows");
  if (!pow2(c->page_size) || c->page_size < 8 || c->page_size > 65536)
    return fail(DMC_ERR_INVALID_ARG, "page_size %d is not a power of two in [8, 65536]", c->page_size);
  if (int64_t(c->max_pages) * c->page_size > (int64_t(1) << 30))
    return fail(DMC_ERR_UNSUPPORTED, "rows of more than 2^30 tokens");
  return DMC_OK;
}

// (a launch has less than 2^32 threads: 256 for each token)
constexpr int32_t kMaxRotatedTokens = 1 << 23;

// The rows and tokens of a call on a full cache.
static dmc_status check_full_rows(const dmc_full_config &c, const int32_t *cu, int32_t total, const int32_t *lengths,
                                  const int32_t *table, const void *k_pages, const void *v_pages) {
  if (total < 0) return fail(DMC_ERR_INVALID_ARG, "total_tokens must be >= 0");
  if (int64_t(total) * (c.num_q_heads + 2 * c.num_kv_heads) * c.head_dim > (int64_t(1) << 36) || total > kMaxRotatedTokens)
    return fail(DMC_ERR_UNSUPPORTED, "too many tokens for one call");
  if (!cu && total != 0 && total != c.batch)
    return fail(DMC_ERR_INVALID_ARG, "%d tokens without cu_seqlens, one for each of %d rows expected", total, c.batch);
  if (total == 0) return DMC_OK;
  if (!lengths || !table || !k_pages || !v_pages)
    return fail(DMC_ERR_INVALID_ARG, "lengths, page_table, k_pages and v_pages must be non-NULL");
  if (!aligned16(k_pages) || !aligned16(v_pages))
    return fail(DMC_ERR_INVALID_ARG, "k_pages and v_pages must be 16-byte aligned");
  return DMC_OK;
}

static dmc_status run_rotation(int es, int head_dim, bool paged, const dmc::RotateParams &p, dmc_stream_t stream) {
  int dev = 0;
  dmc_status st = memory_device(p.k, "k", &dev);
  if (st != DMC_OK) return st;
  DeviceGuard g(dev);
  if (!g.ok) return fail(DMC_ERR_HIP, "cannot select the tensors' device");
  hipError_t e = dmc::launch_rotate(es, head_dim, paged, p, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, paged ? "append launch" : "rotation launch");
  return DMC_OK;
}

dmc_status dmc_rotate(const dmc_rotary_config *cfg, const void *q, const int64_t q_strides[2], const void *k,
                      const int64_t k_strides[2], const int32_t *positions, const float *inv_freq, int32_t total,
                      int32_t inverse, void *q_out, const int64_t q_out_strides[2], void *k_out,
                      const int64_t k_out_strides[2], dmc_stream_t stream) {
  if (!cfg) return fail(DMC_ERR_INVALID_ARG, "config is NULL");
  dmc_status st = validate_heads(cfg->num_q_heads, cfg->num_kv_heads, cfg->head_dim, cfg->dtype, cfg->rotary_dim,
                                 cfg->rotary_pairs);
  if (st == DMC_OK) st = check_packed_counts(0, total);
  if (st != DMC_OK) return st;
  if (total > kMaxRotatedTokens) return fail(DMC_ERR_UNSUPPORTED, "more than %d tokens in one call", kMaxRotatedTokens);
  if (total == 0) return DMC_OK;
  const int es = cfg->dtype == DMC_FP32 ? 4 : 2;
  for (const Packed &t : {Packed{"q", q, q_strides, cfg->num_q_heads, false, false},
                          Packed{"k", k, k_strides, cfg->num_kv_heads, false, false},
                          Packed{"q_out", q_out, q_out_strides, cfg->num_q_heads, false, true},
                          Packed{"k_out", k_out, k_out_strides, cfg->num_kv_heads, false, true}}) {
    st = check_packed(t, total, cfg->head_dim, es);
    if (st != DMC_OK) return st;
  }
  if (!positions || (cfg->rotary_dim > 0 && !inv_freq))
    return fail(DMC_ERR_INVALID_ARG, "positions and inv_freq must be non-NULL");
  dmc::RotateParams p{};
  p.q = q;
  p.k = k;
  p.qo = q_out;
  p.ko = k_out;
  copy_strides(p.qs, q_strides);
  copy_strides(p.ks, k_strides);
  copy_strides(p.qos, q_out_strides);
  copy_strides(p.kos, k_out_strides);
  p.inv_freq = inv_freq;
  p.positions = positions;
  p.total = total;
  p.hq = cfg->num_q_heads;
  p.hkv = cfg->num_kv_heads;
  p.r = cfg->rotary_dim;
  p.halves = cfg->rotary_pairs == DMC_PAIRS_HALVES;
  p.inverse = inverse != 0;
  return run_rotation(es, cfg->head_dim, false, p, stream);
}

dmc_status dmc_full_append(const dmc_full_config *cfg, const void *k, const int64_t k_strides[2], const void *v,
                           const int64_t v_strides[2], const void *q, const int64_t q_strides[2],
                           const float *inv_freq, const int32_t *cu, int32_t total, const int32_t *lengths,
                           const int32_t *table, void *k_pages, void *v_pages, void *q_out,
                           const int64_t q_out_strides[2], int32_t *flags, dmc_stream_t stream) {
  dmc_status st = validate_full(cfg);
  if (st == DMC_OK) st = check_full_rows(*cfg, cu, total, lengths, table, k_pages, v_pages);
  if (st != DMC_OK || total == 0) return st;
  const int es = cfg->dtype == DMC_FP32 ? 4 : 2;
  for (const Packed &t : {Packed{"k", k, k_strides, cfg->num_kv_heads, false, false},
                          Packed{"v", v, v_strides, cfg->num_kv_heads, false, false},
                          Packed{"q", q, q_strides, cfg->num_q_heads, false, false},
                          Packed{"q_out", q_out, q_out_strides, cfg->num_q_heads, false, true}}) {
    if (!q && t.name[0] == 'q') continue;
    st = check_packed(t, total, cfg->head_dim, es);
    if (st != DMC_OK) return st;
  }
  if (cfg->rotary_dim > 0 && !inv_freq) return fail(DMC_ERR_INVALID_ARG, "inv_freq must be non-NULL");
  dmc::RotateParams p{};
  p.k = k;
  p.v = v;
  copy_strides(p.ks, k_strides);
  copy_strides(p.vs, v_strides);
  if (q) {
    p.q = q;
    p.qo = q_out;
    copy_strides(p.qs, q_strides);
    copy_strides(p.qos, q_out_strides);
    p.hq = cfg->num_q_heads;
  }
  p.inv_freq = inv_freq;
  p.cu = cu;
  p.len = lengths;
  p.table = table;
  p.kp = static_cast<char *>(k_pages);
  p.vp = static_cast<char *>(v_pages);
  p.flags = flags;
  p.total = total;
  p.rows = cfg->batch;
  p.hkv = cfg->num_kv_heads;
  p.r = cfg->rotary_dim;
  p.halves = cfg->rotary_pairs == DMC_PAIRS_HALVES;
  p.log2p = ilog2(cfg->page_size);
  p.max_pages = cfg->max_pages;
  p.num_pages = cfg->num_pages;
  p.capacity = cfg->max_pages * cfg->page_size;
  return run_rotation(es, cfg->head_dim, true, p, stream);
}

static dmc_status check_full_sizes(const dmc_full_config *c, int32_t total, int32_t max_chunk) {
  dmc_status st = validate_full(c);
  if (st != DMC_OK) return st;
  if (total < 0) return fail(DMC_ERR_INVALID_ARG, "total_tokens must be >= 0");
  if (max_chunk < 1) return fail(DMC_ERR_INVALID_ARG, "max_chunk must be >= 1");
  if (int64_t(std::max(total, max_chunk)) * c->num_q_heads > (int64_t(1) << 30) || max_chunk > (1 << 24))
    return fail(DMC_ERR_UNSUPPORTED, "too many tokens and heads for one call");
  return DMC_OK;
}

static_assert(DMC_FULL_COUNTER_BYTES >= dmc::kFullPlaces * 3 * sizeof(int32_t), "counters");

static int64_t full_record_floats(int tile_cols, int head_dim) { return int64_t(tile_cols) * (head_dim + 2); }

struct FullLayout {
  int tile_cols;
  size_t counters, cut_units, partials, total;
};

static FullLayout full_layout(const dmc_full_config &c, int32_t max_chunk) {
  FullLayout L{};
  L.tile_cols = dmc::full_tile_cols(c.dtype == DMC_FP32 ? 4 : 2, max_chunk, c.num_q_heads / c.num_kv_heads);
  L.counters = 0;
  L.cut_units = DMC_FULL_COUNTER_BYTES;
  L.partials = L.cut_units + align_up(size_t(dmc::kFullPlaces) * sizeof(dmc::FullPiece), 256);
  L.total = L.partials + align_up(size_t(dmc::kFullPlaces) * 2 * full_record_floats(L.tile_cols, c.head_dim) * 4, 256);
  return L;
}

size_t dmc_full_workspace_bytes(const dmc_full_config *cfg, int32_t total, int32_t max_chunk) {
  if (check_full_sizes(cfg, total, max_chunk) != DMC_OK) return 0;
  return full_layout(*cfg, max_chunk).total;
}

dmc_status dmc_full_attend(const dmc_full_config *cfg, const void *q, const int64_t q_strides[2], const int32_t *cu,
                           int32_t total, int32_t max_chunk, const int32_t *lengths, const int32_t *table,
                           const void *k_pages, const void *v_pages, void *out, const int64_t out_strides[2],
                           float *lse, int32_t *flags, void *ws, size_t bytes, dmc_stream_t stream) {
  dmc_status st = check_full_sizes(cfg, total, max_chunk);
  if (st == DMC_OK) st = check_full_rows(*cfg, cu, total, lengths, table, k_pages, v_pages);
  if (st != DMC_OK || total == 0) return st;
  const int es = cfg->dtype == DMC_FP32 ? 4 : 2;
  for (const Packed &t : {Packed{"q", q, q_strides, cfg->num_q_heads, false, false},
                          Packed{"out", out, out_strides, cfg->num_q_heads, false, true}}) {
    st = check_packed(t, total, cfg->head_dim, es);
    if (st != DMC_OK) return st;
  }
  if (!cu) max_chunk = 1;
  const FullLayout L = full_layout(*cfg, max_chunk);
  if (!ws) return fail(DMC_ERR_INVALID_ARG, "workspace must be non-NULL");
  if (reinterpret_cast<uintptr_t>(ws) & 255u) return fail(DMC_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  if (bytes < L.total) return fail(DMC_ERR_INVALID_ARG, "workspace has %zu bytes, needs %zu", bytes, L.total);
  dmc::FullParams p{};
  p.q = q;
  p.out = out;
  copy_strides(p.qs, q_strides);
  copy_strides(p.os, out_strides);
  p.lse = lse;
  p.cu = cu;
  p.len = lengths;
  p.table = table;
  p.kp = static_cast<const char *>(k_pages);
  p.vp = static_cast<const char *>(v_pages);
  p.flags = flags;
  p.counters = reinterpret_cast<int32_t *>(static_cast<char *>(ws) + L.counters);
  p.cut_units = reinterpret_cast<dmc::FullPiece *>(static_cast<char *>(ws) + L.cut_units);
  p.partials = reinterpret_cast<float *>(static_cast<char *>(ws) + L.partials);
  p.scale_log2 = static_cast<float>(1.4426950408889634 / std::sqrt(double(cfg->head_dim)));
  p.total = total;
  p.rows = cfg->batch;
  p.hq = cfg->num_q_heads;
  p.hkv = cfg->num_kv_heads;
  p.log2p = ilog2(cfg->page_size);
  p.max_pages = cfg->max_pages;
  p.num_pages = cfg->num_pages;
  p.capacity = cfg->max_pages * cfg->page_size;
  p.max_chunk = max_chunk;
  p.places = dmc::kFullPlaces;
  const int G = cfg->num_q_heads / cfg->num_kv_heads;
  const int narrow = std::min(L.tile_cols, es == 4 ? 16 : 32);
  const int64_t tiles = cu ? int64_t(total) * G / narrow + cfg->batch : int64_t(cfg->batch) * ((G + narrow - 1) / narrow);
  p.one_launch = dmc::full_one_launch(tiles, cfg->num_kv_heads, p.capacity);
  p.tile_cols = p.one_launch ? narrow : L.tile_cols;
  p.tile_tokens = std::max(1, p.tile_cols / G);
  p.record_floats = full_record_floats(p.tile_cols, cfg->head_dim);
  p.group_shift = ilog2(G) - 1;
  p.group_magic = G > 1 ? static_cast<uint32_t>(((uint64_t(1) << (31 + ilog2(G))) + G - 1) / G) : 0;
  int dev = 0;
  st = memory_device(ws, "the workspace", &dev);
  if (st != DMC_OK) return st;
  DeviceGuard g(dev);
  if (!g.ok) return fail(DMC_ERR_HIP, "cannot select the workspace's device");
  hipError_t e = dmc::launch_full_attend(es, cfg->head_dim, p, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "full attention launch");
  return DMC_OK;
}

static dmc_status read_control(dmc_cache *cache, dmc_stream_t stream, dmc::Control *out) {
  DeviceGuard g(cache->device);
  if (!g.ok) return fail(DMC_ERR_HIP, "cannot select the cache's device");
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e = hipStreamSynchronize(s);
  if (e != hipSuccess) return hip_fail(e, "hipStreamSynchronize");
  e = hipMemcpy(out, cache->ws + cache->lay.ctrl, sizeof(dmc::Control), hipMemcpyDeviceToHost);
  if (e != hipSuccess) return hip_fail(e, "reading the control block");
  return DMC_OK;
}

dmc_status dmc_cache_check(dmc_cache *cache, dmc_stream_t stream) {
  if (!cache) return fail(DMC_ERR_INVALID_ARG, "cache is NULL");
  dmc::Control ctl{};
  dmc_status st = read_control(cache, stream, &ctl);
  if (st != DMC_OK) return st;
  if (ctl.flags & (dmc::FLAG_POOL_EXHAUSTED | dmc::FLAG_SLOTS_EXHAUSTED))
    return fail(DMC_ERR_CAPACITY, "cache capacity exhausted (flags 0x%x: %s%s)", ctl.flags,
                (ctl.flags & dmc::FLAG_POOL_EXHAUSTED) ? "page pool " : "",
                (ctl.flags & dmc::FLAG_SLOTS_EXHAUSTED) ? "slots per unit" : "");
  if (ctl.flags & dmc::FLAG_BAD_LENGTH)
    return fail(DMC_ERR_INVALID_ARG, "an imported or prompt length was out of range");
  return DMC_OK;
}

dmc_status dmc_cache_pages_used(dmc_cache *cache, int64_t *pages_out, dmc_stream_t stream) {
  if (!cache || !pages_out) return fail(DMC_ERR_INVALID_ARG, "cache and pages_out must be non-NULL");
  dmc::Control ctl{};
  dmc_status st = read_control(cache, stream, &ctl);
  if (st != DMC_OK) return st;
  const unsigned long long used = ctl.pages_used;
  const unsigned long long cap = static_cast<unsigned long long>(cache->cfg.num_pages);
  *pages_out = static_cast<int64_t>(used < cap ? used : cap);
  return DMC_OK;
}

}  // extern "C"
