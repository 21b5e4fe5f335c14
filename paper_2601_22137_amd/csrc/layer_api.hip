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

int size_of(int dt) { return dt == PRISM_F32 ? 4 : 2; }
// negative, or so long that the rows end past 2^60 elements
template <typename... S> bool bad_stride(long long rows, S... s) { return ((s < 0 || (s > 0 && rows > (1ll << 60) / s)) || ...); }

// Rows of a result that lie over one another
bool overlap(long long rows, long long width, long long stride) { return rows > 1 && stride < width; }
constexpr const char* OVERLAP = "rows of a result lie over one another";

int check(const prism_embedding_desc* d, int dt) {
  if (!d || !is_type(dt)) return refuse("null description or unknown type");
  if (d->count < 0 || d->rows < 0 || d->width < 1) return refuse("negative size, or rows without entries");
  if (!std::isfinite(d->scale)) return refuse("scale is not finite");
  if (bad_stride(d->rows, d->table_stride) || bad_stride(d->count, d->out_stride)) return refuse("a stride is negative, or an array ends past 2^60 elements");
  if (d->count > (1ll << 30) || d->rows > (1ll << 27) || d->width > (1 << 24)) return refuse("more than 2^30 tokens, 2^27 rows or 2^24 entries of a row", PRISM_EUNSUPPORTED);
  return PRISM_OK;
}

int check(const prism_layer_norm_desc* d, int dt) {
  if (!d || !is_type(dt)) return refuse("null description or unknown type");
  if (d->rows < 0 || d->width < 1) return refuse("negative size, or rows without entries");
  if (!(d->eps >= 0.0f) || !std::isfinite(d->eps)) return refuse("eps has to be finite and not negative");
  if (bad_stride(d->rows, d->x, d->residual, d->total, d->y, d->dy, d->dtotal, d->dx)) return refuse("a stride is negative, or an array ends past 2^60 elements");
  if (d->width > PRISM_MAX_NORM_WIDTH) return refuse("width is over PRISM_MAX_NORM_WIDTH", PRISM_EUNSUPPORTED);
  if (d->rows > MAX_ROWS) return refuse("more than 2^31 - 1 rows", PRISM_EUNSUPPORTED);
  return PRISM_OK;
}

int check(const prism_logits_desc* d, int dt, bool loss) {
  if (!d || !is_type(dt)) return refuse("null description or unknown type");
  if (d->rows < 0 || d->vocabulary < 1) return refuse("negative size, or rows without logits");
  // (the rest of a rounded factor has to be a normal number too)
  if (!(d->scale >= std::ldexp(1.0, -100) && d->scale <= std::ldexp(1.0, 100))) return refuse("scale has to be between 2^-100 and 2^100");
  if (bad_stride(d->rows, d->logits_stride, d->dlogits_stride)) return refuse("a stride is negative, or an array ends past 2^60 elements");
  if (loss) {
    if (!(d->clip_low >= 0.0 && d->clip_low <= 1.0) || !(d->clip_high >= 0.0) || !std::isfinite(d->clip_high)) return refuse("clip_low has to be in 0 .. 1, clip_high finite and not negative");
    if (!(d->kl >= 0.0) || !std::isfinite(d->kl)) return refuse("kl has to be finite and not negative");
    if (d->kl > 0.0 && !d->ref_logp) return refuse("kl without ref_logp");
  }
  if (d->rows > MAX_ROWS || d->vocabulary > (1 << 30)) return refuse("more than 2^31 - 1 rows or 2^30 logits of a row", PRISM_EUNSUPPORTED);
  return PRISM_OK;
}

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

int prism_embedding(const void* table, const void* tokens, void* out, prism_dtype dt, const prism_embedding_desc* d, void* stream) {
  return guarded([&]() -> int {
    const int rc = check(d, (int)dt);
    if (rc != PRISM_OK || d->count == 0) return rc;
    if (!tokens || !out || (d->rows && !table)) return refuse("null pointer");
    if (overlap(d->count, d->width, d->out_stride)) return refuse(OVERLAP);
    if (!aligned_to(table, size_of(dt)) || !aligned_to(out, size_of(dt)) || !aligned_to(tokens, d->wide_tokens ? 8 : 4)) return refuse("a pointer is not aligned to the element size");
    launch_embedding(table, tokens, out, (int)dt, *d, (hipStream_t)stream);
    return launched();
  });
}

int prism_embedding_backward(const void* dout, const void* tokens, void* dtable, prism_dtype dt, const prism_embedding_desc* d, void* stream) {
  return guarded([&]() -> int {
    int rc = check(d, (int)dt);
    if (rc != PRISM_OK || d->rows == 0) return rc;
    if (!dtable || (d->count && (!tokens || !dout))) return refuse("null pointer");
    if (overlap(d->rows, d->width, d->table_stride)) return refuse(OVERLAP);
    if (!aligned_to(dtable, size_of(dt)) || !aligned_to(dout, size_of(dt)) || !aligned_to(tokens, d->wide_tokens ? 8 : 4)) return refuse("a pointer is not aligned to the element size");
    char* ws = nullptr;
    rc = layer_workspace(embedding_plan(*d, (int)dt).total, d->workspace, d->workspace_bytes, (hipStream_t)stream, &ws);
    if (rc != PRISM_OK) return rc;
    launch_embedding_backward(dout, tokens, dtable, (int)dt, *d, ws, (hipStream_t)stream);
    return launched();
  });
}

int prism_embedding_workspace_bytes(prism_dtype dt, const prism_embedding_desc* d, size_t* out_bytes) {
  return guarded([&]() -> int {
    if (!out_bytes) return refuse("null pointer");
    const int rc = check(d, (int)dt);
    if (rc == PRISM_OK) *out_bytes = d->rows ? embedding_plan(*d, (int)dt).total : 0;
    return rc;
  });
}

int prism_layer_norm(const void* x, const void* residual, const float* weight, const float* bias, void* y, void* total, float* stats, prism_dtype dt,
                     const prism_layer_norm_desc* d, void* stream) {
  return guarded([&]() -> int {
    const int rc = check(d, (int)dt);
    if (rc != PRISM_OK || d->rows == 0) return rc;
    if (!x || !y) return refuse("null pointer");
    if (!residual != !total) return refuse("residual and total go together");
    if (y == total) return refuse("y and total are the same array");
    if (overlap(d->rows, d->width, d->y) || (total && overlap(d->rows, d->width, d->total))) return refuse(OVERLAP);
    for (const void* p : {x, residual, (const void*)y, (const void*)total})
      if (!aligned_to(p, size_of(dt))) return refuse("a pointer is not aligned to the element size");
    for (const void* p : {(const void*)weight, (const void*)bias})
      if (!aligned_to(p, 4)) return refuse("a pointer is not aligned to the element size");
    if (!aligned_to(stats, 8)) return refuse("stats are not aligned to 8 bytes");
    launch_layer_norm(x, residual, weight, bias, y, total, stats, (int)dt, *d, (hipStream_t)stream);
    return launched();
  });
}

int prism_layer_norm_backward(const void* dy, const void* total, const float* stats, const float* weight, const void* dtotal, void* dx, float* dweight, float* dbias,
                              prism_dtype dt, const prism_layer_norm_desc* d, void* stream) {
  return guarded([&]() -> int {
    int rc = check(d, (int)dt);
    if (rc != PRISM_OK) return rc;
    if (d->rows && (!dy || !total || !stats || !dx)) return refuse("null pointer");
    if (overlap(d->rows, d->width, d->dx)) return refuse(OVERLAP);
    for (const void* p : {dy, total, dtotal, (const void*)dx})
      if (!aligned_to(p, size_of(dt))) return refuse("a pointer is not aligned to the element size");
    for (const void* p : {(const void*)weight, (const void*)dweight, (const void*)dbias})
      if (!aligned_to(p, 4)) return refuse("a pointer is not aligned to the element size");
    if (!aligned_to(stats, 8)) return refuse("stats are not aligned to 8 bytes");
    if (d->rows == 0 && !dweight && !dbias) return PRISM_OK;
    char* ws = nullptr;
    if (dweight || dbias) {      // (of no rows: zeros)
      rc = layer_workspace(layer_norm_backward_bytes(*d, (int)dt) + 256, d->workspace, d->workspace_bytes, (hipStream_t)stream, &ws);
      if (rc != PRISM_OK) return rc;
    }
    launch_layer_norm_backward(dy, total, stats, weight, dtotal, dx, dweight, dbias, (int)dt, *d, (float*)ws, (hipStream_t)stream);
    return launched();
  });
}

int prism_layer_norm_workspace_bytes(prism_dtype dt, const prism_layer_norm_desc* d, size_t* out_bytes) {
  return guarded([&]() -> int {
    if (!out_bytes) return refuse("null pointer");
    const int rc = check(d, (int)dt);
    if (rc == PRISM_OK) *out_bytes = layer_norm_backward_bytes(*d, (int)dt) + 256;
    return rc;
  });
}

int prism_token_logprob(const void* logits, const void* tokens, float* logp, float* lse, prism_dtype dt, const prism_logits_desc* d, void* stream) {
  return guarded([&]() -> int {
    const int rc = check(d, (int)dt, false);
    if (rc != PRISM_OK || d->rows == 0) return rc;
    if (!logits || !tokens) return refuse("null pointer");
    if (!aligned_to(logits, size_of(dt)) || !aligned_to(tokens, d->wide_tokens ? 8 : 4) || !aligned_to(logp, 4) || !aligned_to(lse, 4))
      return refuse("a pointer is not aligned to the element size");
    launch_logprob(logits, tokens, logp, lse, (int)dt, *d, (hipStream_t)stream);
    return launched();
  });
}

int prism_token_logprob_backward(const float* dlogp, const void* logits, const void* tokens, const float* lse, void* dlogits, prism_dtype dt,
                                 const prism_logits_desc* d, void* stream) {
  return guarded([&]() -> int {
    const int rc = check(d, (int)dt, false);
    if (rc != PRISM_OK || d->rows == 0) return rc;
    if (!dlogp || !logits || !tokens || !lse || !dlogits) return refuse("null pointer");
    if (overlap(d->rows, d->vocabulary, d->dlogits_stride)) return refuse(OVERLAP);
    if (!aligned_to(logits, size_of(dt)) || !aligned_to(dlogits, size_of(dt)) || !aligned_to(tokens, d->wide_tokens ? 8 : 4) || !aligned_to(dlogp, 4) || !aligned_to(lse, 4))
      return refuse("a pointer is not aligned to the element size");
    launch_logprob_backward(dlogp, logits, tokens, lse, dlogits, (int)dt, *d, (hipStream_t)stream);
    return launched();
  });
}

int prism_policy_loss(const void* logits, const void* tokens, float* loss, float* logp, float* lse, float* dlogp, void* dlogits, prism_dtype dt,
                      const prism_logits_desc* d, void* stream) {
  return guarded([&]() -> int {
    int rc = check(d, (int)dt, true);
    if (rc != PRISM_OK) return rc;
    if (!loss || (d->rows && (!logits || !tokens))) return refuse("null pointer");
    if (dlogits && overlap(d->rows, d->vocabulary, d->dlogits_stride)) return refuse(OVERLAP);
    if (!aligned_to(logits, size_of(dt)) || !aligned_to(dlogits, size_of(dt)) || !aligned_to(tokens, d->wide_tokens ? 8 : 4)) return refuse("a pointer is not aligned to the element size");
    for (const void* p : {(const void*)loss, (const void*)logp, (const void*)lse, (const void*)dlogp, (const void*)d->advantages, (const void*)d->old_logp,
                          (const void*)d->ref_logp, (const void*)d->weights})
      if (!aligned_to(p, 4)) return refuse("a pointer is not aligned to the element size");
    char* ws = nullptr;
    rc = layer_workspace(policy_loss_bytes(*d), d->workspace, d->workspace_bytes, (hipStream_t)stream, &ws);
    if (rc != PRISM_OK) return rc;
    launch_policy_loss(logits, tokens, loss, logp, lse, dlogp, dlogits, (int)dt, *d, ws, (hipStream_t)stream);
    return launched();
  });
}

int prism_policy_loss_workspace_bytes(const prism_logits_desc* d, size_t* out_bytes) {
  return guarded([&]() -> int {
    if (!out_bytes) return refuse("null pointer");
    const int rc = check(d, PRISM_F32, true);
    if (rc == PRISM_OK) *out_bytes = policy_loss_bytes(*d);
    return rc;
  });
}

}  // extern "C"
