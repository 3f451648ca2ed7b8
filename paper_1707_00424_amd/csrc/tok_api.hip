// C-ABI entry points of the token-model operators: every check of arguments is made here, on the host, before a launch.
#include <stdio.h>

#include "tok.h"

namespace {

struct Check {
  const char *who;
  parle_status status = PARLE_OK;
  // Keeps the first failure; texts name the call and the rule.
  Check &that(bool ok, parle_status s, const char *rule) {
    if (!ok && status == PARLE_OK) {
      status = s;
      char text[160];
      snprintf(text, sizeof(text), "%s: %s", who, rule);
      parle_internal_set_error(text);
    }
    return *this;
  }
  Check &field(bool ok, const char *rule) { return that(ok, PARLE_EINVAL, rule); }
  Check &given(const void *p, const char *name) {
    that(p != nullptr, PARLE_EINVAL, name);
    return that(aligned_to(p, 16), PARLE_EALIGN, "a pointer is not 16-byte aligned");
  }
  Check &maybe(const void *p) { return that(aligned_to(p, 16), PARLE_EALIGN, "a pointer is not 16-byte aligned"); }
  Check &scratch(const void *p, int64_t have, int64_t need) {
    that(need == 0 || p, PARLE_EINVAL, "scratch is NULL").maybe(p);
    return that(have >= need, PARLE_ESIZE, "scratch_bytes is less than the call needs");
  }
  parle_status launched(hipError_t e) {
    if (e == hipSuccess) return PARLE_OK;
    that(false, PARLE_EHIP, hipGetErrorString(e));
    return PARLE_EHIP;
  }
};

// Rows, columns, tokens: a launch counts its threads in x in 32 bits, 1024 for a row at most, and a tile of 256 rows of codes is
// addressed with 32-bit offsets.
constexpr long long kMostRows = 1LL << 22;
constexpr long long kMostElems = 1LL << 40;

bool good(Check &c, const parle_embed_desc *d) {
  c.field(d, "desc is NULL");
  if (c.status) return false;
  c.field((d->dtype | 1) == 1 && (d->table_dtype | 1) == 1, "dtype and table_dtype are 0 or 1")
      .field(d->n >= 1 && d->n <= 65535, "1 <= n <= 65535")
      .field(d->tokens >= 0 && d->vocab >= 1 && d->dim >= 1, "tokens >= 0, vocab >= 1, dim >= 1")
      .field(d->table_stride >= (int64_t)d->vocab * d->dim, "table_stride is less than vocab * dim");
  if (c.status) return false;
  c.that(d->vocab <= kMostRows && d->table_stride <= kMostElems / d->n, PARLE_ESIZE, "vocab exceeds 2^22 or n * table_stride 2^40")
      .that(d->tokens <= kMostRows && d->dim <= kMostRows, PARLE_ESIZE, "tokens or dim exceeds 2^22")
      .that((long long)d->n * d->tokens <= kMostElems / d->dim, PARLE_ESIZE, "n * tokens * dim exceeds 2^40");
  return c.status == PARLE_OK;
}
bool good(Check &c, const parle_norm_desc *d) {
  c.field(d, "desc is NULL");
  if (c.status) return false;
  c.field((d->dtype | 1) == 1 && (d->w_dtype | 1) == 1, "dtype and w_dtype are 0 or 1")
      .field(d->n >= 1 && d->n <= 65535, "1 <= n <= 65535")
      .field(d->rows >= 0 && d->dim >= 1, "rows >= 0, dim >= 1")
      .field(d->w_stride >= d->dim, "w_stride is less than dim")
      .field(d->eps >= 0.f && d->eps < 3e38f, "eps is negative or not finite");
  if (c.status) return false;
  c.that(d->rows <= kMostRows && d->dim <= kMostRows, PARLE_ESIZE, "rows or dim exceeds 2^22")
      .that(d->rows < kMostRows || d->dim <= 4096, PARLE_ESIZE, "rows of more than 4096 elements exceed 2^22 - 1")
      .that(d->w_stride <= kMostElems / d->n && (long long)d->n * d->rows <= kMostElems / d->dim, PARLE_ESIZE,
            "a tensor exceeds 2^40 elements");
  return c.status == PARLE_OK;
}
bool good(Check &c, const parle_quant_desc *d) {
  c.field(d, "desc is NULL");
  if (c.status) return false;
  c.field((d->dtype | 1) == 1, "dtype is 0 or 1")
      .field(d->block == 1 || d->block == 128, "block is 1 or 128")
      .field(d->n >= 1 && d->n <= 65535, "1 <= n <= 65535")
      .field(d->rows >= 0 && d->cols >= 1, "rows >= 0, cols >= 1")
      .field(d->ld >= d->cols, "ld is less than cols");
  if (c.status) return false;
  c.that(d->rows <= kMostRows && d->cols <= kMostRows, PARLE_ESIZE, "rows or cols exceeds 2^22")
      .that(d->ld <= kMostElems / (d->rows + 1), PARLE_ESIZE, "rows * ld exceeds 2^40");
  if (c.status) return false;
  c.field(d->n == 1 || d->rows == 0 || d->stride >= (d->rows - 1) * d->ld + d->cols, "stride is less than a replica's rows")
      .that(d->stride <= kMostElems / d->n && d->stride >= 0, PARLE_ESIZE, "n * stride exceeds 2^40");
  return c.status == PARLE_OK;
}
bool good(Check &c, const parle_fp8_desc *d) {
  c.field(d, "desc is NULL");
  if (c.status) return false;
  c.field((d->out_dtype | 1) == 1 && (d->accumulate | 1) == 1, "out_dtype and accumulate are 0 or 1")
      .field(d->b_block == 1 || d->b_block == 128, "b_block is 1 or 128")
      .field(d->n >= 1 && d->n <= 65535, "1 <= n <= 65535")
      .field(d->rows >= 0 && d->cols >= 1 && d->depth >= 0, "rows >= 0, cols >= 1, depth >= 0")
      .field(d->ld_out >= d->cols, "ld_out is less than cols");
  if (c.status) return false;
  c.that(d->rows <= kMostRows && d->cols <= kMostRows && d->depth <= kMostRows, PARLE_ESIZE, "rows, cols or depth exceeds 2^22")
      .that(d->ld_out <= kMostElems / (d->rows + 1), PARLE_ESIZE, "rows * ld_out exceeds 2^40");
  if (c.status) return false;
  c.field(d->n == 1 || d->rows == 0 || d->out_stride >= (d->rows - 1) * d->ld_out + d->cols, "out_stride is less than a replica's rows")
      .that(d->out_stride <= kMostElems / d->n && d->out_stride >= 0, PARLE_ESIZE, "n * out_stride exceeds 2^40");
  return c.status == PARLE_OK;
}
bool good(Check &c, const parle_logprob_desc *d) {
  c.field(d, "desc is NULL");
  if (c.status) return false;
  c.field((d->dtype | 1) == 1, "dtype is 0 or 1")
      .field(d->n >= 1 && d->n <= 65535, "1 <= n <= 65535")
      .field(d->rows >= 0 && d->classes >= 1, "rows >= 0, classes >= 1")
      .field(d->top >= 0 && d->top <= PARLE_LOGPROB_MAX_TOP, "0 <= top <= PARLE_LOGPROB_MAX_TOP")
      .field(d->ld >= d->classes, "ld is less than classes");
  if (c.status) return false;
  c.that(d->classes <= kMostRows, PARLE_ESIZE, "classes exceeds 2^22")
      .that((long long)d->n * d->rows <= kMostRows && d->ld <= kMostElems / ((long long)d->n * d->rows + 1), PARLE_ESIZE,
            "n * rows exceeds 2^22 or the logits 2^40 elements");
  return c.status == PARLE_OK;
}

// Rows `ld` apart and replicas `stride` apart of a tensor of rows of `width` elements.
bool good_rows(Check &c, int n, int rows, long long width, int64_t ld, int64_t stride, const char *narrow, const char *close) {
  c.field(ld >= width, narrow).that(ld <= kMostElems / ((long long)rows + 1), PARLE_ESIZE, "rows of a replica exceed 2^40 elements");
  if (c.status) return false;
  c.field(n == 1 || rows == 0 || stride >= (rows - 1) * ld + width, close)
      .that(stride >= 0 && stride <= kMostElems / n, PARLE_ESIZE, "a tensor exceeds 2^40 elements");
  return c.status == PARLE_OK;
}
bool good(Check &c, const parle_rope_desc *d) {
  c.field(d, "desc is NULL");
  if (c.status) return false;
  c.field((d->dtype | 1) == 1 && (d->interleaved | 1) == 1 && (d->inverse | 1) == 1, "dtype, interleaved and inverse are 0 or 1")
      .field(d->n >= 1 && d->n <= 65535, "1 <= n <= 65535")
      .field(d->tokens >= 0 && d->heads >= 1 && d->dim >= 1, "tokens >= 0, heads >= 1, dim >= 1")
      .field(d->axes >= 1 && d->axes <= PARLE_ROPE_MAX_AXES, "1 <= axes <= PARLE_ROPE_MAX_AXES");
  if (c.status) return false;
  long long pairs = 0;
  for (int i = 0; i < d->axes; ++i) {
    c.field(d->pairs[i] >= 0, "pairs of an axis are negative");
    pairs += d->pairs[i];
  }
  c.field(2 * pairs <= d->dim, "pairs are more than half of dim");
  c.that(d->tokens <= kMostRows && d->dim <= 4096 && (long long)d->heads * d->dim <= kMostRows, PARLE_ESIZE,
         "tokens or heads * dim exceeds 2^22, or dim 4096");
  if (c.status) return false;
  const long long width = (long long)d->heads * d->dim;
  return good_rows(c, d->n, d->tokens, width, d->ld, d->stride, "ld is less than heads * dim", "stride is less than a replica's rows") &&
         good_rows(c, d->n, d->tokens, width, d->ld_out, d->out_stride, "ld_out is less than heads * dim",
                   "out_stride is less than a replica's rows");
}
// What the attention calls share.
bool good_heads(Check &c, int dtype, int heads, int kv_heads, int dim, int window, int sinks, float scale) {
  c.field((dtype | 1) == 1, "dtype is 0 or 1")
      .field(heads >= 1 && kv_heads >= 1 && heads % kv_heads == 0, "heads is a multiple of kv_heads, both at least 1")
      .field(dim >= 8 && dim % 8 == 0, "dim is a multiple of 8")
      .field(window >= 0 && sinks >= 0, "window >= 0, sinks >= 0")
      .field(scale > 0.f && scale < 3e38f, "scale is not positive and finite")
      .that(dim <= PARLE_ATTENTION_MAX_DIM, PARLE_ESIZE, "dim exceeds PARLE_ATTENTION_MAX_DIM")
      .that(sinks <= PARLE_ATTENTION_MAX_SINKS, PARLE_ESIZE, "sinks exceeds PARLE_ATTENTION_MAX_SINKS")
      .that(heads <= 65535, PARLE_ESIZE, "heads exceeds 65535");
  return c.status == PARLE_OK;
}
bool good(Check &c, const parle_attention_desc *d) {
  c.field(d, "desc is NULL");
  if (c.status || !good_heads(c, d->dtype, d->heads, d->kv_heads, d->dim, d->window, d->sinks, d->scale)) return false;
  c.field(d->n >= 1 && d->n <= 65535, "1 <= n <= 65535")
      .field(d->tokens >= 0 && d->sequences >= 1, "tokens >= 0, sequences >= 1")
      .that(d->tokens <= kMostRows && d->sequences <= kMostRows, PARLE_ESIZE, "tokens or sequences exceeds 2^22")
      .that((long long)d->tokens * d->heads < 1LL << 30, PARLE_ESIZE, "tokens * heads reaches 2^30");
  return c.status == PARLE_OK &&
         good_rows(c, d->n, d->tokens, (long long)d->heads * d->dim, d->ld_q, d->q_stride, "ld_q is less than heads * dim",
                   "q_stride is less than a replica's rows") &&
         good_rows(c, d->n, d->tokens, (long long)d->kv_heads * d->dim, d->ld_kv, d->kv_stride, "ld_kv is less than kv_heads * dim",
                   "kv_stride is less than a replica's rows") &&
         good_rows(c, d->n, d->tokens, (long long)d->heads * d->dim, d->ld_out, d->out_stride, "ld_out is less than heads * dim",
                   "out_stride is less than a replica's rows");
}
// The gradient's workgroups of keys are more than the forward pass', and those of the sinks' queries are added.
bool good_bwd(Check &c, const parle_attention_desc *d) {
  if (!good(c, d)) return false;
  c.that(attention_bwd_fits(*d), PARLE_ESIZE, "the gradient of these tokens, heads and sinks takes more than 2^32 threads of a replica");
  return c.status == PARLE_OK;
}
bool good(Check &c, const parle_cache_desc *d) {
  c.field(d, "desc is NULL");
  if (c.status || !good_heads(c, d->dtype, d->heads, d->kv_heads, d->dim, d->window, d->sinks, d->scale)) return false;
  c.field(d->sequences >= 0 && d->capacity > d->sinks, "sequences >= 0, capacity > sinks")
      .field(d->ld_q >= (int64_t)d->heads * d->dim, "ld_q is less than heads * dim")
      .field(d->ld_kv >= (int64_t)d->kv_heads * d->dim, "ld_kv is less than kv_heads * dim")
      .field(d->ld_out >= (int64_t)d->heads * d->dim, "ld_out is less than heads * dim");
  if (c.status) return false;
  c.that(d->sequences <= 65535, PARLE_ESIZE, "sequences exceeds 65535")
      .that((int64_t)d->capacity <= kMostElems / ((int64_t)d->kv_heads * d->dim * (d->sequences + 1)), PARLE_ESIZE, "a cache exceeds 2^40 elements")
      .that(d->ld_q <= kMostElems / (d->sequences + 1) && d->ld_out <= kMostElems / (d->sequences + 1) && d->ld_kv <= kMostElems / kMostRows, PARLE_ESIZE,
            "rows exceed 2^40 elements");
  return c.status == PARLE_OK;
}
bool good(Check &c, const parle_sample_desc *d) {
  c.field(d, "desc is NULL");
  if (c.status) return false;
  c.field((d->dtype | 1) == 1, "dtype is 0 or 1")
      .field(d->n >= 1 && d->n <= 65535, "1 <= n <= 65535")
      .field(d->rows >= 0 && d->classes >= 1, "rows >= 0, classes >= 1")
      .field(d->ld >= d->classes, "ld is less than classes");
  if (c.status) return false;
  c.that(d->classes <= kMostRows, PARLE_ESIZE, "classes exceeds 2^22")
      .that((long long)d->n * d->rows < kMostRows && d->ld <= kMostElems / ((long long)d->n * d->rows + 1), PARLE_ESIZE,
            "n * rows reaches 2^22 or the logits 2^40 elements");
  return c.status == PARLE_OK;
}

}  // namespace

extern "C" {

int64_t parle_k_embed_scratch_bytes(const parle_embed_desc *desc) {
  Check c{"parle_k_embed_scratch_bytes"};
  return good(c, desc) ? embed_scratch_bytes(*desc) : -1;
}

parle_status parle_k_embed_forward(void *hip_stream, const parle_embed_desc *desc, const void *table, const int32_t *tokens,
                                   void *out) {
  Check c{"parle_k_embed_forward"};
  if (!good(c, desc)) return c.status;
  if (desc->tokens == 0) return PARLE_OK;
  c.given(table, "table is NULL").given(tokens, "tokens is NULL").given(out, "out is NULL");
  if (c.status) return c.status;
  return c.launched(launch_embed_fwd((hipStream_t)hip_stream, *desc, table, tokens, out));
}

parle_status parle_k_embed_backward(void *hip_stream, const parle_embed_desc *desc, const int32_t *tokens, const void *dout,
                                    void *scratch, int64_t scratch_bytes, float *dtable) {
  Check c{"parle_k_embed_backward"};
  if (!good(c, desc)) return c.status;
  if (desc->tokens > 0) c.given(tokens, "tokens is NULL").given(dout, "dout is NULL");
  c.given(dtable, "dtable is NULL").scratch(scratch, scratch_bytes, embed_scratch_bytes(*desc));
  if (c.status) return c.status;
  return c.launched(launch_embed_bwd((hipStream_t)hip_stream, *desc, tokens, dout, scratch, dtable));
}

parle_status parle_k_rmsnorm_forward(void *hip_stream, const parle_norm_desc *desc, const void *x, const void *resid,
                                     const void *w, void *h, void *y, uint8_t *q, uint8_t *scales, float *rstd) {
  Check c{"parle_k_rmsnorm_forward"};
  if (!good(c, desc)) return c.status;
  if (desc->rows == 0) return PARLE_OK;
  c.given(x, "x is NULL").given(w, "w is NULL").maybe(resid).maybe(h).maybe(y).maybe(q).maybe(scales).maybe(rstd);
  c.field(y || q, "one of y and q is wanted").field(!q == !scales, "q and scales come together");
  c.field(!h || h != y, "h and y are one buffer");
  if (c.status) return c.status;
  return c.launched(launch_rmsnorm_fwd((hipStream_t)hip_stream, *desc, x, resid, w, h, y, q, scales, rstd));
}

int64_t parle_k_rmsnorm_scratch_bytes(const parle_norm_desc *desc) {
  Check c{"parle_k_rmsnorm_scratch_bytes"};
  return good(c, desc) ? rmsnorm_scratch_bytes(*desc) : -1;
}

parle_status parle_k_rmsnorm_backward(void *hip_stream, const parle_norm_desc *desc, const void *h, const void *w,
                                      const float *rstd, const void *dout, const void *dresid, void *scratch,
                                      int64_t scratch_bytes, void *dx, float *dw) {
  Check c{"parle_k_rmsnorm_backward"};
  if (!good(c, desc)) return c.status;
  if (desc->rows > 0) c.given(h, "h is NULL").given(w, "w is NULL").given(rstd, "rstd is NULL").given(dout, "dout is NULL").given(dx, "dx is NULL");
  c.given(dw, "dw is NULL").maybe(dresid).scratch(scratch, scratch_bytes, rmsnorm_scratch_bytes(*desc));
  if (c.status) return c.status;
  return c.launched(launch_rmsnorm_bwd((hipStream_t)hip_stream, *desc, h, w, rstd, dout, dresid, (float *)scratch, dx, dw));
}

parle_status parle_k_fp8_quantize(void *hip_stream, const parle_quant_desc *desc, const void *src, uint8_t *q, uint8_t *scales,
                                  uint8_t *qt, uint8_t *scales_t) {
  Check c{"parle_k_fp8_quantize"};
  if (!good(c, desc)) return c.status;
  if (desc->rows == 0) return PARLE_OK;
  c.given(src, "src is NULL").maybe(q).maybe(scales).maybe(qt).maybe(scales_t);
  c.field(q || qt, "one of q and qt is wanted").field(!q == !scales && !qt == !scales_t, "codes and scales come together");
  if (c.status) return c.status;
  return c.launched(launch_fp8_quantize((hipStream_t)hip_stream, *desc, src, q, scales, qt, scales_t));
}

int64_t parle_k_fp8_scratch_bytes(const parle_fp8_desc *desc) {
  Check c{"parle_k_fp8_scratch_bytes"};
  return good(c, desc) ? fp8_scratch_bytes(*desc) : -1;
}

parle_status parle_k_fp8_matmul(void *hip_stream, const parle_fp8_desc *desc, const uint8_t *a, const uint8_t *a_scales,
                                const uint8_t *b, const uint8_t *b_scales, const float *bias, void *scratch,
                                int64_t scratch_bytes, void *out) {
  Check c{"parle_k_fp8_matmul"};
  if (!good(c, desc)) return c.status;
  if (desc->rows == 0) return PARLE_OK;
  if (desc->depth > 0)
    c.given(a, "a is NULL").given(a_scales, "a_scales is NULL").given(b, "b is NULL").given(b_scales, "b_scales is NULL");
  c.given(out, "out is NULL").maybe(bias).scratch(scratch, scratch_bytes, fp8_scratch_bytes(*desc));
  if (c.status) return c.status;
  return c.launched(launch_fp8_matmul((hipStream_t)hip_stream, *desc, a, a_scales, b, b_scales, bias, (float *)scratch, out));
}

int64_t parle_k_logprob_scratch_bytes(const parle_logprob_desc *desc) {
  Check c{"parle_k_logprob_scratch_bytes"};
  return good(c, desc) ? logprob_scratch_bytes(*desc) : -1;
}

parle_status parle_k_logprob_forward(void *hip_stream, const parle_logprob_desc *desc, const void *logits, const int32_t *labels,
                                     void *scratch, int64_t scratch_bytes, float *logp, float *entropy, float *lse,
                                     int32_t *top_ids, float *top_logp) {
  Check c{"parle_k_logprob_forward"};
  if (!good(c, desc)) return c.status;
  if (desc->rows == 0) return PARLE_OK;
  c.given(logits, "logits is NULL").maybe(logp).maybe(entropy).maybe(lse);
  if (logp) c.given(labels, "labels is NULL");
  if (desc->top > 0) c.given(top_ids, "top_ids is NULL").given(top_logp, "top_logp is NULL");
  c.field(desc->top > 0 || (!top_ids && !top_logp), "top_ids and top_logp are NULL where top is 0");
  c.scratch(scratch, scratch_bytes, logprob_scratch_bytes(*desc));
  if (c.status) return c.status;
  return c.launched(launch_logprob_fwd((hipStream_t)hip_stream, *desc, logits, labels, scratch, logp, entropy, lse, top_ids, top_logp));
}

parle_status parle_k_logprob_backward(void *hip_stream, const parle_logprob_desc *desc, const void *logits, const int32_t *labels,
                                      const float *lse, const float *entropy, const float *dlogp, const float *dentropy,
                                      void *dlogits) {
  Check c{"parle_k_logprob_backward"};
  if (!good(c, desc)) return c.status;
  if (desc->rows == 0) return PARLE_OK;
  c.given(logits, "logits is NULL").given(labels, "labels is NULL").given(lse, "lse is NULL").given(dlogp, "dlogp is NULL");
  c.given(dlogits, "dlogits is NULL").maybe(dentropy).maybe(entropy).field(!dentropy || entropy, "dentropy needs entropy");
  if (c.status) return c.status;
  return c.launched(launch_logprob_bwd((hipStream_t)hip_stream, *desc, logits, labels, lse, entropy, dlogp, dentropy, dlogits));
}

parle_status parle_k_rope(void *hip_stream, const parle_rope_desc *desc, const void *x, const int32_t *positions, const float *freqs, void *out) {
  Check c{"parle_k_rope"};
  if (!good(c, desc)) return c.status;
  if (desc->tokens == 0) return PARLE_OK;
  c.given(x, "x is NULL").given(positions, "positions is NULL").given(freqs, "freqs is NULL").given(out, "out is NULL");
  c.field(x != out || (desc->ld == desc->ld_out && (desc->n == 1 || desc->stride == desc->out_stride)), "out is x in another layout");
  if (c.status) return c.status;
  return c.launched(launch_rope((hipStream_t)hip_stream, *desc, x, positions, freqs, out));
}

int64_t parle_k_attention_scratch_bytes(const parle_attention_desc *desc) {
  Check c{"parle_k_attention_scratch_bytes"};
  return good_bwd(c, desc) ? attention_scratch_bytes(*desc) : -1;
}

parle_status parle_k_attention_forward(void *hip_stream, const parle_attention_desc *desc, const void *q, const void *k, const void *v,
                                       const int32_t *offsets, void *out, float *lse) {
  Check c{"parle_k_attention_forward"};
  if (!good(c, desc)) return c.status;
  if (desc->tokens == 0) return PARLE_OK;
  c.given(q, "q is NULL").given(k, "k is NULL").given(v, "v is NULL").given(out, "out is NULL").maybe(offsets).maybe(lse);
  c.field(offsets || desc->sequences == 1, "offsets is NULL with more than one sequence");
  c.field(out != q && out != k && out != v, "out is q, k or v");
  if (c.status) return c.status;
  return c.launched(launch_attention_fwd((hipStream_t)hip_stream, *desc, q, k, v, offsets, out, lse));
}

parle_status parle_k_attention_backward(void *hip_stream, const parle_attention_desc *desc, const void *q, const void *k, const void *v,
                                        const int32_t *offsets, const void *out, const float *lse, const void *dout, void *scratch,
                                        int64_t scratch_bytes, void *dq, void *dk, void *dv) {
  Check c{"parle_k_attention_backward"};
  if (!good_bwd(c, desc)) return c.status;
  if (desc->tokens == 0) return PARLE_OK;
  c.given(q, "q is NULL").given(k, "k is NULL").given(v, "v is NULL").given(out, "out is NULL").given(lse, "lse is NULL").given(dout, "dout is NULL");
  c.given(dq, "dq is NULL").given(dk, "dk is NULL").given(dv, "dv is NULL").maybe(offsets);
  c.field(offsets || desc->sequences == 1, "offsets is NULL with more than one sequence");
  const void *in[] = {q, k, v, out, dout};
  for (const void *p : in) c.field(dq != p && dk != p && dv != p, "a gradient is written over an input");
  c.field(dq != dk && dq != dv && dk != dv, "two gradients are one buffer");
  c.scratch(scratch, scratch_bytes, attention_scratch_bytes(*desc));
  if (c.status) return c.status;
  return c.launched(launch_attention_bwd((hipStream_t)hip_stream, *desc, q, k, v, offsets, out, lse, dout, scratch, dq, dk, dv));
}

parle_status parle_k_attention_store(void *hip_stream, const parle_cache_desc *desc, int32_t tokens, const void *k, const void *v,
                                     const int32_t *offsets, const int32_t *lengths, void *k_cache, void *v_cache) {
  Check c{"parle_k_attention_store"};
  if (!good(c, desc)) return c.status;
  c.field(tokens >= 0, "tokens >= 0").that(tokens <= kMostRows, PARLE_ESIZE, "tokens exceeds 2^22");
  if (c.status || tokens == 0 || desc->sequences == 0) return c.status;
  c.given(k, "k is NULL").given(v, "v is NULL").given(offsets, "offsets is NULL").given(lengths, "lengths is NULL");
  c.given(k_cache, "k_cache is NULL").given(v_cache, "v_cache is NULL").field(k_cache != v_cache, "the caches are one buffer");
  if (c.status) return c.status;
  return c.launched(launch_attention_store((hipStream_t)hip_stream, *desc, tokens, k, v, offsets, lengths, k_cache, v_cache));
}

int64_t parle_k_decode_scratch_bytes(const parle_cache_desc *desc) {
  Check c{"parle_k_decode_scratch_bytes"};
  return good(c, desc) ? decode_scratch_bytes(*desc) : -1;
}

parle_status parle_k_attention_decode(void *hip_stream, const parle_cache_desc *desc, const void *q, const void *k, const void *v,
                                      const int32_t *lengths, void *scratch, int64_t scratch_bytes, void *k_cache, void *v_cache, void *out) {
  Check c{"parle_k_attention_decode"};
  if (!good(c, desc)) return c.status;
  if (desc->sequences == 0) return PARLE_OK;
  c.given(q, "q is NULL").given(lengths, "lengths is NULL").given(k_cache, "k_cache is NULL").given(v_cache, "v_cache is NULL");
  c.given(out, "out is NULL").maybe(k).maybe(v).field(!k == !v, "k and v come together").field(k_cache != v_cache, "the caches are one buffer");
  c.field(out != q && out != k && out != v, "out is q, k or v");
  c.scratch(scratch, scratch_bytes, decode_scratch_bytes(*desc));
  if (c.status) return c.status;
  return c.launched(launch_attention_decode((hipStream_t)hip_stream, *desc, q, k, v, lengths, scratch, k_cache, v_cache, out));
}

int64_t parle_k_sample_scratch_bytes(const parle_sample_desc *desc) {
  Check c{"parle_k_sample_scratch_bytes"};
  return good(c, desc) ? sample_scratch_bytes(*desc) : -1;
}

parle_status parle_k_sample(void *hip_stream, const parle_sample_desc *desc, const void *logits, const float *uniform, const float *temperature,
                            const int32_t *top_k, const float *top_p, const float *min_p, void *scratch, int64_t scratch_bytes, int32_t *tokens,
                            int32_t *kept, float *logp) {
  Check c{"parle_k_sample"};
  if (!good(c, desc)) return c.status;
  if (desc->rows == 0) return PARLE_OK;
  c.given(logits, "logits is NULL").given(uniform, "uniform is NULL").given(tokens, "tokens is NULL");
  c.maybe(temperature).maybe(top_k).maybe(top_p).maybe(min_p).maybe(kept).maybe(logp);
  c.scratch(scratch, scratch_bytes, sample_scratch_bytes(*desc));
  if (c.status) return c.status;
  return c.launched(launch_sample((hipStream_t)hip_stream, *desc, logits, uniform, temperature, top_k, top_p, min_p, scratch, tokens, kept, logp));
}

}  // extern "C"
