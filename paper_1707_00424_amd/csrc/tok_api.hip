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

}  // extern "C"
