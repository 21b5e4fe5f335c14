// Entry points of the operators of a transformer layer: argument checks, workspaces, launches.  Nothing is enqueued before every argument is checked.
#include <cmath>
#include <exception>

#include "layer.h"

namespace prism {
namespace {

constexpr long long MAX_ROWS = (1ll << 31) - 1;
constexpr long long MAX_GROUPS = (1ll << 24) - 1;   // workgroups of 256 in a launch, which takes fewer than 2^32 work-items

int refuse(const char* why, int rc = PRISM_EINVAL) {
  set_last_error(why);
  return rc;
}

int launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? (int)PRISM_OK : refuse(hipGetErrorString(e), PRISM_EHIP);
}

// A C entry lets no exception out
template <typename F> int guarded(F&& f) {
  try {
    set_last_error("");
    return f();
  } catch (const std::exception& e) {
    try { set_last_error(e.what()); } catch (...) {}
    return PRISM_ENOMEM;
  } catch (...) {
    return PRISM_EHIP;
  }
}

bool is_type(int dt) { return dt == PRISM_F32 || dt == PRISM_BF16; }
bool aligned_to(const void* p, int size) { return ((uintptr_t)p & (uintptr_t)(size - 1)) == 0; }

template <typename... S> bool negative(const S&... s) { return ((s.batch < 0 || s.token < 0 || s.head < 0) || ...); }

int check(const prism_norm_rope_desc* d, int dt) {
  if (!d || !is_type(dt)) return refuse("null description or unknown type");
  if (d->batch < 0 || d->len < 0 || d->q_heads < 0 || d->k_heads < 0 || d->head_dim < 1) return refuse("negative size, or a head without entries");
  if (d->rot_dim < 0 || d->rot_dim > d->head_dim || d->rot_dim % 2) return refuse("rot_dim has to be even and at most head_dim");
  if (d->rot_dim > 0 && !d->inv_freq) return refuse("rot_dim without inv_freq");
  if (!std::isfinite(d->scale) || (d->norm && !(d->eps >= 0.0f && std::isfinite(d->eps)))) return refuse("scale or eps is not finite, or eps negative");
  if (!d->positions && (long long)d->start + d->len - 1 > 0x7FFFFFFFll) return refuse("the last position is past 2^31 - 1");
  if (!d->norm && (d->q_weight || d->k_weight)) return refuse("weights without the norm");
  if (negative(d->q, d->k, d->q_out, d->k_out, d->dq, d->dk)) return refuse("a stride is negative");
  if (d->head_dim > PRISM_MAX_NORM_HEAD) return refuse("head_dim is over PRISM_MAX_NORM_HEAD", PRISM_EUNSUPPORTED);
  if ((long long)d->batch * d->len > MAX_ROWS / (d->q_heads + (long long)d->k_heads + 1)) return refuse("more than 2^31 - 1 heads in a call", PRISM_EUNSUPPORTED);
  return PRISM_OK;
}
bool empty(const prism_norm_rope_desc& d) { return d.batch == 0 || d.len == 0 || (d.q_heads == 0 && d.k_heads == 0); }

int check(const prism_attention_desc* d, int dt) {
  if (!d || !is_type(dt)) return refuse("null description or unknown type");
  if (d->batch < 0 || d->q_len < 0 || d->k_len < 0 || d->q_heads < 0 || d->k_heads < 0 || d->head_dim < 1) return refuse("negative size, or a head without entries");
  if (d->k_heads ? d->q_heads == 0 || d->q_heads % d->k_heads : d->q_heads) return refuse("q_heads has to be a multiple of k_heads");
  if (!(d->scale > 0.0f) || !std::isfinite(d->scale)) return refuse("scale has to be positive and finite");
  if (!(d->softcap >= 0.0f) || !std::isfinite(d->softcap)) return refuse("softcap has to be finite and not negative");
  // the factors that scores are taken times: an infinite one would make NaN of a score of 0, a subnormal one of a cap loses digits
  const float log2e = 1.4426950408889634f;
  if (!std::isfinite(d->scale * log2e) || (d->softcap > 0.0f && !(std::isnormal(d->scale / d->softcap) && std::isnormal(d->softcap * log2e))))
    return refuse("scale log2(e), scale / softcap or softcap log2(e) is out of the range of fp32");
  if (!d->q_doc != !d->k_doc) return refuse("q_doc and k_doc go together");
  if (d->prefix && !d->causal) return refuse("a prefix needs the causal mask");
  if (negative(d->q, d->k, d->v, d->out, d->dout, d->dq, d->dk, d->dv)) return refuse("a stride is negative");
  if (d->head_dim > PRISM_MAX_ATTENTION_HEAD) return refuse("head_dim is over PRISM_MAX_ATTENTION_HEAD", PRISM_EUNSUPPORTED);
  if (!d->k_heads || !d->batch) return PRISM_OK;
  const long long G = d->q_heads / d->k_heads, R = G * d->q_len, pairs = (long long)d->batch * d->k_heads;
  if (R > MAX_ROWS - 256 || d->k_len > MAX_ROWS - 256 || pairs * R > MAX_ROWS / 4 || pairs * d->k_len > MAX_ROWS / 4)
    return refuse("the rows of a call and the keys of a call (their heads counted) may be 2^29 at most", PRISM_EUNSUPPORTED);
  if (pairs * ((R + 127) / 128) > MAX_GROUPS || pairs * (((long long)d->k_len + 127) / 128) > MAX_GROUPS)
    return refuse("more than 2^24 - 1 tiles of 128 rows or keys in a call", PRISM_EUNSUPPORTED);
  return PRISM_OK;
}
// no result at all (keys without queries have gradients: zero)
bool empty(const prism_attention_desc& d, bool backward) { return d.batch == 0 || d.q_heads == 0 || (d.q_len == 0 && (!backward || d.k_len == 0)); }

}  // namespace
}  // namespace prism

using namespace prism;

extern "C" {

int prism_dropout(const void* x, const void* residual, void* y, int64_t count, prism_dtype dt, double p, uint64_t seed, uint32_t offset, void* stream) {
  return guarded([&]() -> int {
    if (!is_type(dt) || count < 0) return refuse("unknown type or a negative count");
    if (!(p >= 0.0 && p < 1.0)) return refuse("p has to be at least 0 and below 1");
    const unsigned limit = (unsigned)std::nearbyint(p * 65536.0);
    if (limit > 65535u) return refuse("p rounds to 1 in 16 bits");
    if (count > (1ll << 60)) return refuse("more than 2^60 elements", PRISM_EUNSUPPORTED);
    if (count == 0) return PRISM_OK;
    if (!x || !y) return refuse("null pointer");
    const int size = dt == PRISM_F32 ? 4 : 2;
    if (!aligned_to(x, size) || !aligned_to(residual, size) || !aligned_to(y, size)) return refuse("a pointer is not aligned to the element size");
    const int rc = launch_dropout(x, residual, y, count, (int)dt, limit, seed, offset, (hipStream_t)stream);
    return rc == PRISM_OK ? launched() : rc;
  });
}

int prism_qk_norm_rope(const void* q, const void* k, void* q_out, void* k_out, prism_dtype dt, const prism_norm_rope_desc* d, void* stream) {
  return guarded([&]() -> int {
    int rc = check(d, (int)dt);
    if (rc != PRISM_OK || empty(*d)) return rc;
    if ((d->q_heads && (!q || !q_out)) || (d->k_heads && (!k || !k_out))) return refuse("null pointer");
    const int size = dt == PRISM_F32 ? 4 : 2;
    for (const void* x : {q, k, (const void*)q_out, (const void*)k_out})
      if (!aligned_to(x, size)) return refuse("a pointer is not aligned to the element size");
    rc = launch_norm_rope(q, k, q_out, k_out, (int)dt, *d, (hipStream_t)stream);
    return rc == PRISM_OK ? launched() : rc;
  });
}

int prism_qk_norm_rope_backward(const void* dq_out, const void* dk_out, const void* q, const void* k, void* dq, void* dk, float* dq_weight, float* dk_weight,
                                prism_dtype dt, const prism_norm_rope_desc* d, void* stream) {
  return guarded([&]() -> int {
    int rc = check(d, (int)dt);
    if (rc != PRISM_OK || empty(*d)) return rc;
    if (!d->norm && (dq_weight || dk_weight)) return refuse("gradients of weights without the norm");
    if ((d->q_heads && (!dq_out || !dq || (d->norm && !q))) || (d->k_heads && (!dk_out || !dk || (d->norm && !k)))) return refuse("null pointer");
    const int size = dt == PRISM_F32 ? 4 : 2;
    for (const void* x : {dq_out, dk_out, q, k, (const void*)dq, (const void*)dk})
      if (!aligned_to(x, size)) return refuse("a pointer is not aligned to the element size");
    char* ws = nullptr;
    const size_t bytes = dq_weight || dk_weight ? norm_rope_backward_bytes(*d) : 0;
    if (bytes) {
      rc = layer_workspace(bytes, d->workspace, d->workspace_bytes, (hipStream_t)stream, &ws);
      if (rc != PRISM_OK) return rc;
    }
    rc = launch_norm_rope_backward(dq_out, dk_out, q, k, dq, dk, dq_weight, dk_weight, (int)dt, *d, (float*)ws, (hipStream_t)stream);
    return rc == PRISM_OK ? launched() : rc;
  });
}

int prism_attention(const void* q, const void* k, const void* v, void* out, float* lse, prism_dtype dt, const prism_attention_desc* d, void* stream) {
  return guarded([&]() -> int {
    int rc = check(d, (int)dt);
    if (rc != PRISM_OK || empty(*d, false)) return rc;
    if (!q || !out || (d->k_len && (!k || !v))) return refuse("null pointer");
    const int size = dt == PRISM_F32 ? 4 : 2;
    for (const void* x : {q, k, v, (const void*)out})
      if (!aligned_to(x, size)) return refuse("a pointer is not aligned to the element size");
    char* ws = nullptr;
    const size_t bytes = attention_plan(*d, (int)dt, false).total;
    if (bytes) {
      rc = layer_workspace(bytes, d->workspace, d->workspace_bytes, (hipStream_t)stream, &ws);
      if (rc != PRISM_OK) return rc;
    }
    rc = launch_attention(q, k, v, out, lse, (int)dt, *d, ws, (hipStream_t)stream);
    return rc == PRISM_OK ? launched() : rc;
  });
}

int prism_attention_backward(const void* dout, const void* q, const void* k, const void* v, const void* out, const float* lse, void* dq, void* dk, void* dv,
                             prism_dtype dt, const prism_attention_desc* d, void* stream) {
  return guarded([&]() -> int {
    int rc = check(d, (int)dt);
    if (rc != PRISM_OK || empty(*d, true)) return rc;
    if ((d->q_len && (!dout || !q || !out || !lse || !dq)) || (d->k_len && (!k || !v || !dk || !dv))) return refuse("null pointer");
    const int size = dt == PRISM_F32 ? 4 : 2;
    for (const void* x : {dout, q, k, v, out, (const void*)dq, (const void*)dk, (const void*)dv})
      if (!aligned_to(x, size)) return refuse("a pointer is not aligned to the element size");
    char* ws = nullptr;
    rc = layer_workspace(attention_plan(*d, (int)dt, true).total, d->workspace, d->workspace_bytes, (hipStream_t)stream, &ws);
    if (rc != PRISM_OK) return rc;
    rc = launch_attention_backward(dout, q, k, v, out, lse, dq, dk, dv, (int)dt, *d, ws, (hipStream_t)stream);
    return rc == PRISM_OK ? launched() : rc;
  });
}

int prism_norm_rope_workspace_bytes(prism_dtype dt, const prism_norm_rope_desc* d, size_t* out_bytes) {
  return guarded([&]() -> int {
    if (!out_bytes) return refuse("null pointer");
    const int rc = check(d, (int)dt);
    if (rc == PRISM_OK) *out_bytes = empty(*d) ? 0 : norm_rope_backward_bytes(*d);
    return rc;
  });
}

int prism_attention_workspace_bytes(prism_dtype dt, const prism_attention_desc* d, int backward, size_t* out_bytes) {
  return guarded([&]() -> int {
    if (!out_bytes) return refuse("null pointer");
    const int rc = check(d, (int)dt);
    if (rc == PRISM_OK) *out_bytes = empty(*d, backward != 0) ? 0 : attention_plan(*d, (int)dt, backward != 0).total;
    return rc;
  });
}

}  // extern "C"
