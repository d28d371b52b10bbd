// C ABI of the batched serving step: rotary positions, the paged cache, attention over it, sampling.
// Host-side validation and dispatch; nothing is enqueued unless every argument check passes.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <string>

#include "sirius.h"
#include "common.h"
#include "kernels.h"
#include "paged.h"

namespace {

constexpr int kMaxTokens = 1 << 20;  // tokens per call
constexpr int kMaxHeads = 4096;
constexpr int kMaxSeqs = 65535;
constexpr long kMaxGrid = (1 << 24) - 1;  // workgroups of 256 threads: a launch has fewer than 2^32 threads

int fail(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  sirius::set_last_error(buf);
  return code;
}

int hip_status(hipError_t e, const char* what) {
  if (e == hipSuccess) return SIRIUS_OK;
  return fail(SIRIUS_EHIP, "%s: HIP error %d (%s)", what, (int)e, hipGetErrorString(e));
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_ptr(const char* fn, const void* p, const char* name) {
  if (p == nullptr) return fail(SIRIUS_EINVAL, "%s: %s is NULL", fn, name);
  if (!aligned16(p)) return fail(SIRIUS_EINVAL, "%s: %s is not 16-byte aligned", fn, name);
  return SIRIUS_OK;
}

int check_dtype(const char* fn, int t, const char* name) {
  if (t == SIRIUS_F32 || t == SIRIUS_BF16) return SIRIUS_OK;
  return fail(SIRIUS_EINVAL, "%s: %s=%d is neither SIRIUS_F32 nor SIRIUS_BF16", fn, name, t);
}

// Rows of `heads` heads, tokens ld elements apart.
int check_rows(const char* fn, const void* p, const char* name, int heads, int hd, int64_t ld) {
  int rc = check_ptr(fn, p, name);
  if (rc) return rc;
  if (ld < (int64_t)heads * hd || ld % 8 != 0 || ld > ((int64_t)1 << 31))
    return fail(SIRIUS_EINVAL, "%s: the stride %lld of %s must be a multiple of 8, at least heads*head_dim=%lld", fn,
                (long long)ld, name, (long long)heads * hd);
  return SIRIUS_OK;
}

int check_heads(const char* fn, int n, const char* name) {
  if (n < 1 || n > kMaxHeads) return fail(SIRIUS_EINVAL, "%s: %s=%d outside [1, %d]", fn, name, n, kMaxHeads);
  return SIRIUS_OK;
}

int check_head_dim(const char* fn, int hd) {
  if (hd < 8 || hd > 128 || hd % 8 != 0)
    return fail(SIRIUS_EINVAL, "%s: head_dim=%d must be a multiple of 8 in [8, 128]", fn, hd);
  return SIRIUS_OK;
}

int check_rotation(const char* fn, const sirius_rotation* r, int hd, sirius::RopeCall& c) {
  c.mscale = 1.f;
  c.eps = -1.f;
  if (r == nullptr) return SIRIUS_OK;
  if (r->rot_dim < 0 || r->rot_dim > hd || r->rot_dim % 2 != 0)
    return fail(SIRIUS_EINVAL, "%s: rot_dim=%d must be even, in [0, head_dim=%d]", fn, r->rot_dim, hd);
  if (r->rot_dim > 0 && r->freqs == nullptr) return fail(SIRIUS_EINVAL, "%s: freqs is NULL", fn);
  if (!std::isfinite(r->mscale)) return fail(SIRIUS_EINVAL, "%s: mscale must be finite", fn);
  if (std::isnan(r->norm_eps) || std::isinf(r->norm_eps)) return fail(SIRIUS_EINVAL, "%s: norm_eps must be finite", fn);
  if (!aligned16(r->freqs) || !aligned16(r->q_weight) || !aligned16(r->k_weight))
    return fail(SIRIUS_EINVAL, "%s: freqs and the norm weights must be 16-byte aligned", fn);
  c.freqs = r->freqs;
  c.qw = r->q_weight;
  c.kw = r->k_weight;
  c.rot = r->rot_dim;
  c.inter = r->interleaved != 0;
  c.mscale = r->mscale;
  c.eps = r->norm_eps;
  return SIRIUS_OK;
}

int check_paged_sizes(const char* fn, const sirius_paged* c) {
  if (c == nullptr) return fail(SIRIUS_EINVAL, "%s: cache is NULL", fn);
  int rc;
  if ((rc = check_heads(fn, c->n_kv_heads, "n_kv_heads")) || (rc = check_head_dim(fn, c->head_dim))) return rc;
  if (c->B < 0 || c->B > kMaxSeqs) return fail(SIRIUS_EINVAL, "%s: B=%d outside [0, %d]", fn, c->B, kMaxSeqs);
  if (c->T < 0 || c->T > kMaxTokens) return fail(SIRIUS_EINVAL, "%s: T=%d outside [0, 2^20]", fn, c->T);
  if (c->page_size < 8 || c->page_size > sirius::kMaxPageSize || c->page_size % 8 != 0)
    return fail(SIRIUS_EINVAL, "%s: page_size=%d must be a multiple of 8 in [8, %d]", fn, c->page_size, sirius::kMaxPageSize);
  if (c->n_pages < 1) return fail(SIRIUS_EINVAL, "%s: n_pages=%d must be >= 1", fn, c->n_pages);
  if (c->max_pages < 1 || (int64_t)c->max_pages * c->page_size > sirius::kMaxPagedRows)
    return fail(SIRIUS_EINVAL, "%s: max_pages=%d of %d rows: 1 to 2^20 rows per sequence", fn, c->max_pages, c->page_size);
  if (c->max_n < 0 || c->max_n > kMaxTokens) return fail(SIRIUS_EINVAL, "%s: max_n=%d outside [0, 2^20]", fn, c->max_n);
  if (c->tok_start == nullptr && (int64_t)c->B * c->max_n != c->T)
    return fail(SIRIUS_EINVAL, "%s: T=%d tokens are not B=%d times max_n=%d (no tok_start)", fn, c->T, c->B, c->max_n);
  return SIRIUS_OK;
}

int check_paged_ptrs(const char* fn, const sirius_paged* c) {
  int rc;
  if ((rc = check_ptr(fn, c->k_pages, "k_pages")) || (rc = check_ptr(fn, c->v_pages, "v_pages"))) return rc;
  if (c->page_table == nullptr || c->cache_pos == nullptr)
    return fail(SIRIUS_EINVAL, "%s: page_table or cache_pos is NULL", fn);
  return SIRIUS_OK;
}

sirius::PagedView view(const sirius_paged* c) {
  sirius::PagedView v{};
  v.k_pages = c->k_pages;
  v.v_pages = c->v_pages;
  v.table = c->page_table;
  v.pos = c->cache_pos;
  v.start = c->tok_start;
  v.B = c->B;
  v.T = c->T;
  v.n = c->max_n;
  v.n_pages = c->n_pages;
  v.page_size = c->page_size;
  v.max_pages = c->max_pages;
  v.page_magic = (uint32_t)((((uint64_t)1 << 32) + c->page_size - 1) / c->page_size);
  return v;
}

}  // namespace

extern "C" {

int sirius_rope_freqs(double* freqs, int rot_dim, double theta, int scaling, double factor, double low, double high,
                      double orig_len) {
  const char* fn = "sirius_rope_freqs";
  if (freqs == nullptr) return fail(SIRIUS_EINVAL, "%s: freqs is NULL", fn);
  if (rot_dim < 2 || rot_dim > 128 || rot_dim % 2 != 0)
    return fail(SIRIUS_EINVAL, "%s: rot_dim=%d must be even, in [2, 128]", fn, rot_dim);
  if (!std::isfinite(theta) || !(theta > 1.0)) return fail(SIRIUS_EINVAL, "%s: theta must be finite and > 1", fn);
  if (scaling < SIRIUS_ROPE_PLAIN || scaling > SIRIUS_ROPE_RAMP) return fail(SIRIUS_EINVAL, "%s: unknown scaling %d", fn, scaling);
  if (scaling != SIRIUS_ROPE_PLAIN && (!std::isfinite(factor) || !(factor >= 1.0)))
    return fail(SIRIUS_EINVAL, "%s: factor must be finite and >= 1", fn);
  const bool parts = scaling == SIRIUS_ROPE_SMOOTH || scaling == SIRIUS_ROPE_RAMP;
  if (parts && (!(low >= 0.0) || !(high > low) || !std::isfinite(high) || !(orig_len >= 1.0) || !std::isfinite(orig_len)))
    return fail(SIRIUS_EINVAL, "%s: need 0 <= low < high and orig_len >= 1, all finite", fn);
  if (scaling == SIRIUS_ROPE_RAMP && !(low > 0.0)) return fail(SIRIUS_EINVAL, "%s: the ramp needs low > 0", fn);
  if (scaling == SIRIUS_ROPE_BASE && rot_dim == 2) return fail(SIRIUS_EINVAL, "%s: BASE needs rot_dim > 2", fn);
  const double two_pi = 6.283185307179586476925;
  if (scaling == SIRIUS_ROPE_BASE) theta *= std::pow(factor, rot_dim / (rot_dim - 2.0));
  auto index = [&](double turns) { return rot_dim * std::log(orig_len / (two_pi * turns)) / (2.0 * std::log(theta)); };
  double first = 0.0, last = 1.0;
  if (scaling == SIRIUS_ROPE_RAMP) {
    first = std::min(std::max(std::floor(index(high)), 0.0), rot_dim - 1.0);
    last = std::min(std::max(std::ceil(index(low)), 0.0), rot_dim - 1.0);
    if (last <= first) last = first + 1e-3;  // a step
  }
  for (int j = 0; j < rot_dim / 2; ++j) {
    const double f = std::pow(theta, -2.0 * j / rot_dim);
    double keep = 1.0;  // the share of f that stays unscaled
    if (scaling == SIRIUS_ROPE_LINEAR) keep = 0.0;
    if (scaling == SIRIUS_ROPE_SMOOTH) keep = (orig_len * f / two_pi - low) / (high - low);
    if (scaling == SIRIUS_ROPE_RAMP) keep = 1.0 - (j - first) / (last - first);
    keep = std::min(std::max(keep, 0.0), 1.0);
    freqs[j] = keep == 1.0 ? f : f * (keep + (1.0 - keep) / factor);
  }
  return SIRIUS_OK;
}

int sirius_rope(const void* q, int q_dtype, int64_t ldq, const void* k, int k_dtype, int64_t ldk, const int32_t* positions,
                int T, int H, int Hkv, int head_dim, const sirius_rotation* rotation, void* q_out, uint16_t* k_out,
                void* stream) {
  const char* fn = "sirius_rope";
  int rc;
  if ((rc = check_head_dim(fn, head_dim))) return rc;
  if (T < 0 || T > kMaxTokens) return fail(SIRIUS_EINVAL, "%s: T=%d outside [0, 2^20]", fn, T);
  sirius::RopeCall c{};
  if (rotation == nullptr) return fail(SIRIUS_EINVAL, "%s: rotation is NULL", fn);
  if ((rc = check_rotation(fn, rotation, head_dim, c))) return rc;
  if ((rc = check_dtype(fn, q_dtype, "q_dtype")) || (rc = check_dtype(fn, k_dtype, "k_dtype"))) return rc;
  if (T == 0) return SIRIUS_OK;
  if (q == nullptr && k == nullptr) return fail(SIRIUS_EINVAL, "%s: q and k are both NULL", fn);
  if (positions == nullptr) return fail(SIRIUS_EINVAL, "%s: positions is NULL", fn);
  if (q != nullptr && ((rc = check_heads(fn, H, "H")) || (rc = check_rows(fn, q, "q", H, head_dim, ldq)) ||
                       (rc = check_ptr(fn, q_out, "q_out"))))
    return rc;
  if (k != nullptr && ((rc = check_heads(fn, Hkv, "Hkv")) || (rc = check_rows(fn, k, "k", Hkv, head_dim, ldk)) ||
                       (rc = check_ptr(fn, k_out, "k_out"))))
    return rc;
  c.q = q; c.k = k;
  c.q_bf16 = q_dtype == SIRIUS_BF16; c.k_bf16 = k_dtype == SIRIUS_BF16;
  c.ldq = ldq; c.ldk = ldk;
  c.positions = positions;
  c.T = T; c.H = H; c.Hkv = Hkv; c.hd = head_dim;
  c.q_out = q_out; c.k_out = k_out;
  return hip_status(sirius::launch_rope(c, static_cast<hipStream_t>(stream)), fn);
}

int sirius_kv_append(const void* q, int q_dtype, int64_t ldq, const void* k, const void* v, int kv_dtype, int64_t ldk,
                     int64_t ldv, const sirius_paged* cache, const int32_t* positions, int H,
                     const sirius_rotation* rotation, void* q_out, void* stream) {
  const char* fn = "sirius_kv_append";
  int rc;
  if ((rc = check_paged_sizes(fn, cache))) return rc;
  sirius::RopeCall c{};
  if ((rc = check_rotation(fn, rotation, cache->head_dim, c))) return rc;
  if ((rc = check_dtype(fn, q_dtype, "q_dtype")) || (rc = check_dtype(fn, kv_dtype, "kv_dtype"))) return rc;
  if (cache->T == 0 || cache->B == 0) return SIRIUS_OK;
  if ((rc = check_paged_ptrs(fn, cache))) return rc;
  const int hd = cache->head_dim, Hkv = cache->n_kv_heads;
  if (q != nullptr && ((rc = check_heads(fn, H, "H")) || (rc = check_rows(fn, q, "q", H, hd, ldq)) ||
                       (rc = check_ptr(fn, q_out, "q_out"))))
    return rc;
  if ((rc = check_rows(fn, k, "k", Hkv, hd, ldk)) || (rc = check_rows(fn, v, "v", Hkv, hd, ldv))) return rc;
  if (sirius::kv_append_grid(cache->T, Hkv) > kMaxGrid) return fail(SIRIUS_EINVAL, "%s: T=%d tokens of %d heads are too many", fn, cache->T, Hkv);
  c.q = q; c.k = k; c.v = v;
  c.q_bf16 = q_dtype == SIRIUS_BF16; c.k_bf16 = kv_dtype == SIRIUS_BF16;
  c.ldq = ldq; c.ldk = ldk; c.ldv = ldv;
  c.positions = positions;
  c.T = cache->T; c.H = H; c.Hkv = Hkv; c.hd = hd;
  c.q_out = q_out;
  return hip_status(sirius::launch_kv_append(c, view(cache), static_cast<hipStream_t>(stream)), fn);
}

int sirius_attn_paged(const void* q, int q_dtype, int64_t ldq, const sirius_paged* cache, int H, float scale,
                      float softcap, const float* slopes, int window, const uint64_t* mask, void* out, void* ws,
                      size_t ws_bytes, void* stream) {
  const char* fn = "sirius_attn_paged";
  int rc;
  if ((rc = check_paged_sizes(fn, cache))) return rc;
  const int hd = cache->head_dim, Hkv = cache->n_kv_heads;
  if ((rc = check_dtype(fn, q_dtype, "q_dtype")) || (rc = check_heads(fn, H, "H"))) return rc;
  if (H % Hkv != 0) return fail(SIRIUS_EINVAL, "%s: H=%d must be a multiple of n_kv_heads=%d", fn, H, Hkv);
  if (!(scale >= 0.f) || std::isinf(scale)) return fail(SIRIUS_EINVAL, "%s: scale must be finite and >= 0", fn);
  if (!(softcap >= 0.f) || std::isinf(softcap)) return fail(SIRIUS_EINVAL, "%s: softcap must be finite and >= 0", fn);
  if (window < 0) return fail(SIRIUS_EINVAL, "%s: window=%d < 0", fn, window);
  if (mask != nullptr && cache->max_n > 64) return fail(SIRIUS_EINVAL, "%s: a mask needs max_n=%d <= 64", fn, cache->max_n);
  if (cache->T == 0 || cache->B == 0) return SIRIUS_OK;
  if ((rc = check_paged_ptrs(fn, cache)) || (rc = check_rows(fn, q, "q", H, hd, ldq)) || (rc = check_ptr(fn, out, "out")) ||
      (rc = check_ptr(fn, ws, "ws")))
    return rc;
  const int64_t rows = (int64_t)(H / Hkv) * cache->max_n;
  if (rows > INT32_MAX / 256) return fail(SIRIUS_EINVAL, "%s: too many query rows per call", fn);
  const sirius::PagedAttnLayout L = sirius::paged_attn_layout(cache->B, cache->max_n, H, Hkv, hd, q_dtype == SIRIUS_BF16);
  if (sirius::paged_attn_grid(view(cache), Hkv, L) > kMaxGrid) return fail(SIRIUS_EINVAL, "%s: too many query rows per call", fn);
  if (ws_bytes < L.total) return fail(SIRIUS_EWORKSPACE, "%s: workspace %zu bytes < %zu needed", fn, ws_bytes, L.total);
  sirius::PagedAttnCall c{};
  c.q = q;
  c.q_bf16 = q_dtype == SIRIUS_BF16;
  c.ldq = ldq;
  c.H = H; c.Hkv = Hkv; c.hd = hd;
  c.scale = scale > 0.f ? scale : (float)(1.0 / std::sqrt((double)hd));
  c.cap = softcap > 0.f ? std::max(softcap, FLT_MIN) : 0.f;  // 1 / cap stays finite (a score of 0 times it, 0)
  c.slopes = slopes;
  c.window = window;
  c.mask = mask;
  c.out = out;
  return hip_status(sirius::launch_attn_paged(c, view(cache), static_cast<char*>(ws), L, static_cast<hipStream_t>(stream)), fn);
}

int sirius_sample(const float* logits, int64_t ld, int B, int V, const float* u, const float* temperature,
                  const int32_t* top_k, const float* top_p, const float* min_p, int32_t* token, int32_t* kept, float* prob,
                  void* ws, size_t ws_bytes, void* stream) {
  const char* fn = "sirius_sample";
  if (B < 0 || B > kMaxSeqs) return fail(SIRIUS_EINVAL, "%s: B=%d outside [0, %d]", fn, B, kMaxSeqs);
  if (V < 1 || V > (1 << 24)) return fail(SIRIUS_EINVAL, "%s: V=%d outside [1, 2^24]", fn, V);
  if (ld < V || ld > ((int64_t)1 << 31)) return fail(SIRIUS_EINVAL, "%s: rows of V=%d are %lld apart", fn, V, (long long)ld);
  if (B == 0) return SIRIUS_OK;
  int rc;
  if ((rc = check_ptr(fn, logits, "logits")) || (rc = check_ptr(fn, ws, "ws"))) return rc;
  if (u == nullptr || token == nullptr) return fail(SIRIUS_EINVAL, "%s: u or token is NULL", fn);
  if (sirius::sample_grid(B, V) > kMaxGrid) return fail(SIRIUS_EINVAL, "%s: B=%d rows of V=%d are too many", fn, B, V);
  const sirius::SampleLayout L = sirius::sample_layout(B, V);
  if (ws_bytes < L.total) return fail(SIRIUS_EWORKSPACE, "%s: workspace %zu bytes < %zu needed", fn, ws_bytes, L.total);
  const sirius::SampleCall c{logits, (long)ld, B, V, u, temperature, top_k, top_p, min_p, token, kept, prob};
  return hip_status(sirius::launch_sample(c, static_cast<char*>(ws), L, static_cast<hipStream_t>(stream)), fn);
}

}  // extern "C"
