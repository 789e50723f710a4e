// C entry points of the paged K/V cache: argument checks and launches.  They
// need no context and keep no state between calls: the shapes come with the
// cache descriptor, scratch memory and stream with the call.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "gmc.h"
#include "gmc_cache.h"
#include "gmc_cache_grid.h"
#include "gmc_path.h"

namespace {

using namespace gmc;

long long ll(int64_t x) { return static_cast<long long>(x); }
bool misaligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; }

// The kernels' view of a checked descriptor.
int check_cache(const char* fn, const gmc_cache* c, CacheView* out) {
  if (!c) return set_error(GMC_ERR_ARG, "%s: cache is NULL", fn);
  if (c->dtype != GMC_F32 && c->dtype != GMC_BF16) return set_error(GMC_ERR_ARG, "%s: dtype=%d unknown", fn, c->dtype);
  if (c->n_kv_heads < 1 || c->n_q_heads < 1 || c->n_q_heads > GMC_CACHE_MAX_HEADS || c->n_q_heads % c->n_kv_heads != 0)
    return set_error(GMC_ERR_ARG, "%s: n_kv_heads=%d must divide n_q_heads=%d in [1, %d]", fn, c->n_kv_heads,
                     c->n_q_heads, GMC_CACHE_MAX_HEADS);
  if (c->head_dim < 32 || c->head_dim > 256 || c->head_dim % 32 != 0)
    return set_error(GMC_ERR_ARG, "%s: head_dim=%d must be a multiple of 32 in [32, 256]", fn, c->head_dim);
  if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)) != 0)
    return set_error(GMC_ERR_ARG, "%s: page_size=%d must be a power of two in [16, 1024]", fn, c->page_size);
  if (c->n_seq < 1 || c->n_seq > 65535) return set_error(GMC_ERR_ARG, "%s: n_seq=%lld out of [1, 65535]", fn, ll(c->n_seq));
  if (c->n_pages < 1 || c->n_pages > (1ll << 31) - 1)
    return set_error(GMC_ERR_ARG, "%s: n_pages=%lld out of [1, 2^31)", fn, ll(c->n_pages));
  if (c->max_pages < 1 || ll(c->max_pages) * c->page_size > (1ll << 24))
    return set_error(GMC_ERR_ARG, "%s: max_pages=%d must be at least 1, and at most 2^24 slots a sequence", fn, c->max_pages);
  if (!c->k_pages || !c->v_pages || !c->page_table || !c->lens) return set_error(GMC_ERR_ARG, "%s: null cache pointer", fn);
  if (misaligned(c->k_pages, 16) || misaligned(c->v_pages, 16))
    return set_error(GMC_ERR_ARG, "%s: pages must be 16-byte aligned", fn);
  if (c->slot_pos && !c->seen) return set_error(GMC_ERR_ARG, "%s: slot_pos needs seen", fn);
  CacheView& v = *out;
  v.k = c->k_pages; v.v = c->v_pages; v.table = c->page_table; v.lens = c->lens; v.seen = c->seen;
  v.slot_pos = c->slot_pos; v.weights = c->weights;
  v.n_pages = c->n_pages; v.n_seq = static_cast<int>(c->n_seq); v.max_pages = c->max_pages;
  v.page = c->page_size; v.shift = __builtin_ctz(c->page_size); v.cap = c->max_pages * c->page_size;
  v.hq = c->n_q_heads; v.hkv = c->n_kv_heads; v.hg = c->n_q_heads / c->n_kv_heads; v.dh = c->head_dim;
  v.dtype = c->dtype;
  return GMC_OK;
}

size_t elem(const CacheView& c) { return c.dtype == GMC_F32 ? 4 : 2; }

// Rows of `width` elements, `stride` apart, in 16-byte pieces.
int check_rows(const char* fn, const char* name, const CacheView& c, const void* p, int64_t stride, int64_t width) {
  if (!p) return set_error(GMC_ERR_ARG, "%s: %s is NULL", fn, name);
  if (misaligned(p, 16) || stride < width || stride * elem(c) % 16 != 0 || stride > (1ll << 24))
    return set_error(GMC_ERR_ARG, "%s: %s must be 16-byte aligned with rows a multiple of 16 bytes and %lld to 2^24 "
                     "elements apart (stride=%lld)", fn, name, ll(width), ll(stride));
  return GMC_OK;
}

// starts / max_new / rows of the new tokens.
int check_new(const char* fn, const CacheView& c, const int32_t* starts, int64_t max_new, int64_t rows) {
  if (max_new < 1 || max_new > c.cap)
    return set_error(GMC_ERR_ARG, "%s: max_new=%lld out of [1, %d] (the slots of a sequence)", fn, ll(max_new), c.cap);
  if (rows < 1 || rows > (1ll << 31) - 1) return set_error(GMC_ERR_ARG, "%s: rows=%lld out of [1, 2^31)", fn, ll(rows));
  if (!starts && rows != max_new * c.n_seq)
    return set_error(GMC_ERR_ARG, "%s: without starts rows=%lld must be n_seq * max_new = %lld", fn, ll(rows),
                     ll(max_new) * c.n_seq);
  return GMC_OK;
}

int check_attend(const char* fn, const CacheView& c, const void* q, int64_t q_stride, float scale, int64_t window,
                 int64_t sinks, const void* out) {
  const int rc = check_rows(fn, "q", c, q, q_stride, static_cast<int64_t>(c.hq) * c.dh);
  if (rc != GMC_OK) return rc;
  if (!std::isfinite(scale)) return set_error(GMC_ERR_ARG, "%s: scale=%g must be finite", fn, static_cast<double>(scale));
  if (window < 0 || sinks < 0 || window > INT32_MAX || sinks > INT32_MAX)
    return set_error(GMC_ERR_ARG, "%s: window=%lld and sinks=%lld must be in [0, 2^31)", fn, ll(window), ll(sinks));
  if (!out || misaligned(out, 16)) return set_error(GMC_ERR_ARG, "%s: out is NULL or not 16-byte aligned", fn);
  return GMC_OK;
}

// (what is launched for a prefill is fewer than 2^32 threads, and the kernel counts rows in 32 bits)
int check_blocks(const char* fn, const CacheView& c, int64_t max_new) {
  if ((max_new * c.hg + 127) / 128 * c.hkv * c.n_seq > kPreMaxBlocks)
    return set_error(GMC_ERR_ARG, "%s: more than 2^23 blocks of 128 queries (max_new=%lld, n_seq=%d); split the call",
                     fn, ll(max_new), c.n_seq);
  return GMC_OK;
}

AttendArgs attend_args(const void* q, int64_t q_stride, int64_t rows, const int32_t* starts, int64_t max_new,
                       float scale, int64_t window, int64_t sinks, void* out, float* lse) {
  AttendArgs a{};
  a.q = q; a.q_stride = q_stride; a.rows = rows; a.starts = starts; a.max_new = static_cast<int>(max_new);
  a.scale = scale; a.window = static_cast<int>(window); a.sinks = static_cast<int>(sinks); a.out = out; a.lse = lse;
  return a;
}

int check_workspace(const char* fn, const void* ws, int64_t bytes, int64_t need) {
  if (need > 0 && (!ws || misaligned(ws, 256)))
    return set_error(GMC_ERR_ARG, "%s: workspace is NULL or not 256-byte aligned", fn);
  if (bytes < need)
    return set_error(GMC_ERR_CAPACITY, "%s: the workspace holds %lld bytes, the call needs %lld", fn, ll(bytes), ll(need));
  return GMC_OK;
}

// Launches on the stream's own device, whichever is current.
template <typename F>
int on_stream(const char* fn, void* stream, F launch) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  int current = 0, dev = 0;
  hipError_t err = hipGetDevice(&current);
  if (err != hipSuccess) return set_error(GMC_ERR_HIP, "%s: no HIP device (%s)", fn, hipGetErrorString(err));
  dev = current;
  if (st) {
    err = hipStreamGetDevice(st, &dev);
    if (err == hipSuccess && dev != current) err = hipSetDevice(dev);
  }
  if (err == hipSuccess) {
    err = launch(st);
    if (dev != current) (void)hipSetDevice(current);
  }
  if (err != hipSuccess) return set_error(GMC_ERR_HIP, "%s: %s", fn, hipGetErrorString(err));
  return GMC_OK;
}

// The kernels' view of a checked descriptor of 4 bits: codes as pages.
int check_cache4(const char* fn, const gmc_cache4* c, CacheView* out, CacheScales* scales) {
  if (!c) return set_error(GMC_ERR_ARG, "%s: cache is NULL", fn);
  gmc_cache d{};
  d.dtype = c->dtype; d.n_q_heads = c->n_q_heads; d.n_kv_heads = c->n_kv_heads; d.head_dim = c->head_dim;
  d.page_size = c->page_size; d.max_pages = c->max_pages; d.n_pages = c->n_pages; d.n_seq = c->n_seq;
  d.k_pages = c->k_codes; d.v_pages = c->v_codes; d.page_table = c->page_table; d.lens = c->lens;
  const int rc = check_cache(fn, &d, out);
  if (rc != GMC_OK) return rc;
  if (!c->k_scales || !c->v_scales || misaligned(c->k_scales, 16) || misaligned(c->v_scales, 16))
    return set_error(GMC_ERR_ARG, "%s: scales are NULL or not 16-byte aligned", fn);
  scales->k = static_cast<uint8_t*>(c->k_scales);
  scales->v = static_cast<uint8_t*>(c->v_scales);
  scales->bytes = scale_bytes(c->head_dim);
  return GMC_OK;
}

int check_rotary(const char* fn, const CacheView& c, const gmc_rotary* r, RotaryView* out) {
  if (!r->cos || !r->sin || misaligned(r->cos, 16) || misaligned(r->sin, 16))
    return set_error(GMC_ERR_ARG, "%s: the rotary tables are NULL or not 16-byte aligned", fn);
  if (r->n_pos < 1 || r->n_pos > (1ll << 31) - 1)
    return set_error(GMC_ERR_ARG, "%s: n_pos=%lld out of [1, 2^31)", fn, ll(r->n_pos));
  if (r->rot_dim < 16 || r->rot_dim % 16 != 0 || r->rot_dim > c.dh)
    return set_error(GMC_ERR_ARG, "%s: rot_dim=%d must be a multiple of 16 in [16, %d]", fn, r->rot_dim, c.dh);
  if (r->interleaved != 0 && r->interleaved != 1)
    return set_error(GMC_ERR_ARG, "%s: interleaved=%d must be 0 or 1", fn, r->interleaved);
  const int32_t* s = r->sections;
  const bool none = s[0] == 0 && s[1] == 0 && s[2] == 0;
  if (!none) {
    for (int i = 0; i < 3; ++i)
      if (s[i] < 0 || s[i] > c.dh || s[i] % 4 != 0)
        return set_error(GMC_ERR_ARG, "%s: sections[%d]=%d must be a multiple of 4, not negative", fn, i, s[i]);
    if (s[0] + s[1] + s[2] != r->rot_dim / 2)
      return set_error(GMC_ERR_ARG, "%s: sections hold %d pairs, rot_dim=%d has %d", fn, s[0] + s[1] + s[2], r->rot_dim,
                       r->rot_dim / 2);
  }
  RotaryView& v = *out;
  v.cos = r->cos; v.sin = r->sin; v.n_pos = static_cast<int>(r->n_pos); v.rot = r->rot_dim;
  v.interleaved = r->interleaved;
  v.axes = none ? 1 : 3;
  v.t_end = none ? r->rot_dim : s[0];
  v.h_end = none ? r->rot_dim : s[0] + s[1];
  return GMC_OK;
}

// The new rows of an append.
int check_append(const char* fn, const CacheView& c, const void* k, const void* v, int64_t k_stride, int64_t v_stride,
                 int64_t rows, const int32_t* starts, const int32_t* src, int64_t max_new) {
  const int64_t width = static_cast<int64_t>(c.hkv) * c.dh;
  int rc = check_rows(fn, "k", c, k, k_stride, width);
  if (rc != GMC_OK) return rc;
  if ((rc = check_rows(fn, "v", c, v, v_stride, width)) != GMC_OK) return rc;
  if (src && starts) return set_error(GMC_ERR_ARG, "%s: src and starts must not both be set", fn);
  if (src && (rows < c.n_seq || rows % c.n_seq != 0))
    return set_error(GMC_ERR_ARG, "%s: with src rows=%lld must be a multiple of n_seq=%d", fn, ll(rows), c.n_seq);
  return check_new(fn, c, starts, max_new, src ? max_new * c.n_seq : rows);
}

// An append with rotation, queries or 4 bits.
int append_rotary(const char* fn, const CacheView& c, const CacheScales* scales, const gmc_rotary* rotary, const void* k,
                  const void* v, int64_t k_stride, int64_t v_stride, int64_t rows, const int32_t* starts,
                  const int32_t* src, int64_t max_new, const int32_t* pos, const void* q, int64_t q_stride, void* q_out,
                  void* stream) {
  int rc = check_append(fn, c, k, v, k_stride, v_stride, rows, starts, src, max_new);
  if (rc != GMC_OK) return rc;
  RotaryView r{};
  if (rotary) {
    if ((rc = check_rotary(fn, c, rotary, &r)) != GMC_OK) return rc;
  } else if (pos || q || q_out) {
    return set_error(GMC_ERR_ARG, "%s: pos, q and q_out need rotary", fn);
  }
  if (!q != !q_out) return set_error(GMC_ERR_ARG, "%s: q and q_out must both be set or both be NULL", fn);
  if (q) {
    const int64_t width = static_cast<int64_t>(c.hq) * c.dh;
    if ((rc = check_rows(fn, "q", c, q, q_stride, width)) != GMC_OK) return rc;
    if (misaligned(q_out, 16)) return set_error(GMC_ERR_ARG, "%s: q_out is not 16-byte aligned", fn);
    if (q == q_out && (src || (rows > 1 && q_stride != width)))
      return set_error(GMC_ERR_ARG, "%s: q_out may be q only without src and with rows of q %lld elements apart", fn,
                       ll(width));
  }
  RotaryArgs a{};
  a.k = k; a.v = v; a.q = q; a.k_stride = k_stride; a.v_stride = v_stride; a.q_stride = q_stride; a.rows = rows;
  a.per_seq = rows / c.n_seq;
  a.starts = starts; a.src = src; a.pos = pos; a.max_new = static_cast<int>(max_new); a.q_out = q_out;
  return on_stream(fn, stream, [&](hipStream_t st) {
    return launch_cache_append_rotary(c, scales, rotary ? &r : nullptr, a, st);
  });
}

int64_t round256(int64_t x) { return (x + 255) / 256 * 256; }

int64_t decode_bytes(const CacheView& c, bool accumulate) { return round256(decode_scratch_bytes(c, accumulate)); }
int64_t decode4_bytes(const CacheView& c) { return round256(decode4_scratch_bytes(c)); }
int64_t prefill_bytes(const CacheView& c, int64_t max_new, bool four_bits = false) {
  return round256(prefill_scratch_bytes(c, static_cast<int>(max_new), four_bits));
}
int64_t evict_bytes(const CacheView& c) { return round256(evict_scratch_bytes(c)); }

}  // namespace

extern "C" {

int gmc_cache_append(const gmc_cache* cache, const void* k, const void* v, int64_t k_stride, int64_t v_stride,
                     int64_t rows, const int32_t* starts, const int32_t* src, int64_t max_new, void* stream) {
  const char* fn = "gmc_cache_append";
  CacheView c;
  int rc = check_cache(fn, cache, &c);
  if (rc != GMC_OK) return rc;
  if ((rc = check_append(fn, c, k, v, k_stride, v_stride, rows, starts, src, max_new)) != GMC_OK) return rc;
  return on_stream(fn, stream, [&](hipStream_t st) {
    return launch_cache_append(c, k, v, k_stride, v_stride, rows, starts, src, static_cast<int>(max_new), st);
  });
}

int64_t gmc_cache_decode_bytes(const gmc_cache* cache, int32_t accumulate) {
  CacheView c;
  const int rc = check_cache("gmc_cache_decode_bytes", cache, &c);
  return rc != GMC_OK ? rc : decode_bytes(c, accumulate != 0);
}

int gmc_cache_decode(const gmc_cache* cache, const void* q, int64_t q_stride, float scale, int64_t window,
                     int64_t sinks, int32_t accumulate, void* out, float* lse, void* workspace,
                     int64_t workspace_bytes, void* stream) {
  const char* fn = "gmc_cache_decode";
  CacheView c;
  int rc = check_cache(fn, cache, &c);
  if (rc != GMC_OK) return rc;
  if ((rc = check_attend(fn, c, q, q_stride, scale, window, sinks, out)) != GMC_OK) return rc;
  if (accumulate && !c.weights) return set_error(GMC_ERR_ARG, "%s: accumulate needs the cache's weights", fn);
  rc = check_workspace(fn, workspace, workspace_bytes, decode_bytes(c, accumulate != 0));
  if (rc != GMC_OK) return rc;
  const AttendArgs a = attend_args(q, q_stride, c.n_seq, nullptr, 1, scale, window, sinks, out, lse);
  return on_stream(fn, stream, [&](hipStream_t st) {
    return launch_cache_decode(c, a, accumulate != 0, workspace, st);
  });
}

int64_t gmc_cache_prefill_bytes(const gmc_cache* cache, int64_t max_new) {
  CacheView c;
  const int rc = check_cache("gmc_cache_prefill_bytes", cache, &c);
  if (rc != GMC_OK) return rc;
  if (max_new < 1 || max_new > c.cap)
    return set_error(GMC_ERR_ARG, "gmc_cache_prefill_bytes: max_new=%lld out of [1, %d]", ll(max_new), c.cap);
  return prefill_bytes(c, max_new);
}

int gmc_cache_prefill(const gmc_cache* cache, const void* q, int64_t q_stride, int64_t rows, const int32_t* starts,
                      int64_t max_new, float scale, int64_t window, int64_t sinks, void* out, float* lse,
                      void* workspace, int64_t workspace_bytes, void* stream) {
  const char* fn = "gmc_cache_prefill";
  CacheView c;
  int rc = check_cache(fn, cache, &c);
  if (rc != GMC_OK) return rc;
  if ((rc = check_attend(fn, c, q, q_stride, scale, window, sinks, out)) != GMC_OK) return rc;
  if ((rc = check_new(fn, c, starts, max_new, rows)) != GMC_OK) return rc;
  if ((rc = check_blocks(fn, c, max_new)) != GMC_OK) return rc;
  if ((rc = check_workspace(fn, workspace, workspace_bytes, prefill_bytes(c, max_new))) != GMC_OK) return rc;
  const AttendArgs a = attend_args(q, q_stride, rows, starts, max_new, scale, window, sinks, out, lse);
  return on_stream(fn, stream, [&](hipStream_t st) { return launch_cache_prefill(c, a, workspace, st); });
}

int64_t gmc_cache_evict_bytes(const gmc_cache* cache, int64_t budget) {
  CacheView c;
  const int rc = check_cache("gmc_cache_evict_bytes", cache, &c);
  if (rc != GMC_OK) return rc;
  if (budget < 1) return set_error(GMC_ERR_ARG, "gmc_cache_evict_bytes: budget=%lld must be at least 1", ll(budget));
  return budget >= c.cap ? 0 : evict_bytes(c);
}

int gmc_cache_evict(const gmc_cache* cache, int64_t budget, int64_t sinks, int64_t recent, void* workspace,
                    int64_t workspace_bytes, void* stream) {
  const char* fn = "gmc_cache_evict";
  CacheView c;
  int rc = check_cache(fn, cache, &c);
  if (rc != GMC_OK) return rc;
  if (!c.weights || !c.slot_pos)
    return set_error(GMC_ERR_ARG, "%s: needs the cache's weights, slot_pos and seen", fn);
  if (budget < 1 || sinks < 0 || recent < 0 || sinks > budget || recent > budget - sinks)
    return set_error(GMC_ERR_ARG, "%s: need budget >= 1 and sinks + recent <= budget, none negative (budget=%lld "
                     "sinks=%lld recent=%lld)", fn, ll(budget), ll(sinks), ll(recent));
  if (budget >= c.cap) return GMC_OK;   // no sequence can hold more
  if (ll(c.n_seq) * c.hkv > evict_max_groups(c))
    return set_error(GMC_ERR_ARG, "%s: more than %lld caches of a head (n_seq=%d, n_kv_heads=%d); split the call", fn,
                     evict_max_groups(c), c.n_seq, c.hkv);
  rc = check_workspace(fn, workspace, workspace_bytes, evict_bytes(c));
  if (rc != GMC_OK) return rc;
  return on_stream(fn, stream, [&](hipStream_t st) {
    return launch_cache_evict(c, static_cast<int>(budget), static_cast<int>(sinks), static_cast<int>(recent),
                              workspace, st);
  });
}

int gmc_cache_append_rotary(const gmc_cache* cache, const gmc_rotary* rotary, const void* k, const void* v,
                            int64_t k_stride, int64_t v_stride, int64_t rows, const int32_t* starts,
                            const int32_t* src, int64_t max_new, const int32_t* pos, const void* q, int64_t q_stride,
                            void* q_out, void* stream) {
  const char* fn = "gmc_cache_append_rotary";
  CacheView c;
  const int rc = check_cache(fn, cache, &c);
  if (rc != GMC_OK) return rc;
  if (!rotary) return set_error(GMC_ERR_ARG, "%s: rotary is NULL", fn);
  return append_rotary(fn, c, nullptr, rotary, k, v, k_stride, v_stride, rows, starts, src, max_new, pos, q, q_stride,
                       q_out, stream);
}

int gmc_cache4_append(const gmc_cache4* cache, const gmc_rotary* rotary, const void* k, const void* v,
                      int64_t k_stride, int64_t v_stride, int64_t rows, const int32_t* starts, const int32_t* src,
                      int64_t max_new, const int32_t* pos, const void* q, int64_t q_stride, void* q_out,
                      void* stream) {
  const char* fn = "gmc_cache4_append";
  CacheView c;
  CacheScales s;
  const int rc = check_cache4(fn, cache, &c, &s);
  if (rc != GMC_OK) return rc;
  return append_rotary(fn, c, &s, rotary, k, v, k_stride, v_stride, rows, starts, src, max_new, pos, q, q_stride, q_out,
                       stream);
}

int gmc_cache4_read(const gmc_cache4* cache, int64_t rows, const int32_t* starts, int64_t max_new, void* k_out,
                    void* v_out, void* stream) {
  const char* fn = "gmc_cache4_read";
  CacheView c;
  CacheScales s;
  int rc = check_cache4(fn, cache, &c, &s);
  if (rc != GMC_OK) return rc;
  if ((rc = check_new(fn, c, starts, max_new, rows)) != GMC_OK) return rc;
  if (!k_out || !v_out || misaligned(k_out, 16) || misaligned(v_out, 16))
    return set_error(GMC_ERR_ARG, "%s: k_out or v_out is NULL or not 16-byte aligned", fn);
  return on_stream(fn, stream, [&](hipStream_t st) {
    return launch_cache4_read(c, s, rows, starts, static_cast<int>(max_new), k_out, v_out, st);
  });
}

int64_t gmc_cache4_prefill_bytes(const gmc_cache4* cache, int64_t max_new) {
  const char* fn = "gmc_cache4_prefill_bytes";
  CacheView c;
  CacheScales s;
  const int rc = check_cache4(fn, cache, &c, &s);
  if (rc != GMC_OK) return rc;
  if (max_new < 1 || max_new > c.cap)
    return set_error(GMC_ERR_ARG, "%s: max_new=%lld out of [1, %d]", fn, ll(max_new), c.cap);
  return prefill_bytes(c, max_new, true);
}

int gmc_cache4_prefill(const gmc_cache4* cache, const void* q, int64_t q_stride, int64_t rows, const int32_t* starts,
                       int64_t max_new, float scale, int64_t window, int64_t sinks, void* out, float* lse,
                       void* workspace, int64_t workspace_bytes, void* stream) {
  const char* fn = "gmc_cache4_prefill";
  CacheView c;
  CacheScales s;
  int rc = check_cache4(fn, cache, &c, &s);
  if (rc != GMC_OK) return rc;
  if ((rc = check_attend(fn, c, q, q_stride, scale, window, sinks, out)) != GMC_OK) return rc;
  if ((rc = check_new(fn, c, starts, max_new, rows)) != GMC_OK) return rc;
  if ((rc = check_blocks(fn, c, max_new)) != GMC_OK) return rc;
  if ((rc = check_workspace(fn, workspace, workspace_bytes, prefill_bytes(c, max_new, true))) != GMC_OK) return rc;
  const AttendArgs a = attend_args(q, q_stride, rows, starts, max_new, scale, window, sinks, out, lse);
  return on_stream(fn, stream, [&](hipStream_t st) { return launch_cache4_prefill(c, s, a, workspace, st); });
}

int64_t gmc_cache4_decode_bytes(const gmc_cache4* cache) {
  CacheView c;
  CacheScales s;
  const int rc = check_cache4("gmc_cache4_decode_bytes", cache, &c, &s);
  return rc != GMC_OK ? rc : decode4_bytes(c);
}

int gmc_cache4_decode(const gmc_cache4* cache, const void* q, int64_t q_stride, float scale, int64_t window,
                      int64_t sinks, void* out, float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  const char* fn = "gmc_cache4_decode";
  CacheView c;
  CacheScales s;
  int rc = check_cache4(fn, cache, &c, &s);
  if (rc != GMC_OK) return rc;
  if ((rc = check_attend(fn, c, q, q_stride, scale, window, sinks, out)) != GMC_OK) return rc;
  if ((rc = check_workspace(fn, workspace, workspace_bytes, decode4_bytes(c))) != GMC_OK) return rc;
  const AttendArgs a = attend_args(q, q_stride, c.n_seq, nullptr, 1, scale, window, sinks, out, lse);
  return on_stream(fn, stream, [&](hipStream_t st) { return launch_cache4_decode(c, s, a, workspace, st); });
}

}  // extern "C"
