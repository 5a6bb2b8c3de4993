// C entries of the operators on rows of logits (see include/hbsjd.h): checks of arguments, then one launch.
#include <cstdarg>
#include <cstdio>

#include "../../include/hbsjd.h"
#include "logit_rows.cuh"

using namespace hbsjd;

namespace {

thread_local char g_detail[256] = "null context";

int refuse(const char* format, ...) {
    va_list ap;
    va_start(ap, format);
    vsnprintf(g_detail, sizeof(g_detail), format, ap);
    va_end(ap);
    return HBSJD_EINVAL;
}

int launched(const char* what, cudaError_t e) {
    if (e == cudaSuccess) return HBSJD_OK;
    cudaGetLastError();  // (a refused launch stays the device's last error else)
    snprintf(g_detail, sizeof(g_detail), "%s: %s", what, cudaGetErrorString(e));
    return e == cudaErrorMemoryAllocation ? HBSJD_ENOMEM : HBSJD_ECUDA;
}

constexpr int64_t MAX_LD = (int64_t)1 << 40;
constexpr int MAX_ROWS = (1 << 27) - 1;  // a launch has up to 16 CTAs a row (128 chunks are for few rows)

int elem(int dtype) { return dtype == HBSJD_DTYPE_BF16 ? 2 : 4; }
bool is_dtype(int d) { return d == HBSJD_DTYPE_FP32 || d == HBSJD_DTYPE_BF16; }
bool is_aligned(const void* p, int bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// What an array of rows may be: null where allowed, aligned to its elements, rows that do not overlap where it is written.
int rows_wrong(const char* what, const char* name, const void* p, int64_t ld, int V, int bytes, bool written) {
    if (!is_aligned(p, bytes)) return refuse("%s: %s is not aligned to its elements", what, name);
    if (ld < (written ? V : 0) || ld > MAX_LD)
        return refuse("%s: row stride %lld of %s is out of range", what, (long long)ld, name);
    return 0;
}

// An array that is written may be one that is read, at the same place; else they may not overlap.  (Arrays of different
// strides are not looked at.)
bool overlaps(const void* out, int64_t ld_out, int bytes_out, const void* in, int64_t ld_in, int bytes_in, int rows, int V) {
    if (!out || !in || ld_out * bytes_out != ld_in * bytes_in) return false;
    if (out == in && bytes_out == bytes_in) return false;
    const int64_t step = ld_out * bytes_out, d = (const char*)out - (const char*)in;
    if (d >= (rows - 1) * step + (int64_t)V * bytes_in || -d >= (rows - 1) * step + (int64_t)V * bytes_out) return false;
    const int64_t m = ((d % step) + step) % step;  // where a row of `out` begins in a row of `in`
    return m < (int64_t)V * bytes_in || m + (int64_t)V * bytes_out > step;
}

int distill_wrong(const char* what, const hbsjd_distill_desc* d, const void* s, const float* loss, const void* grad) {
    if (!d || !s) return refuse("%s: null argument", what);
    if (d->rows < 1 || d->rows > MAX_ROWS || d->V < 1 || d->V > MAX_LOGIT_V)
        return refuse("%s: %d rows of %d logits are out of range", what, d->rows, d->V);
    if (!is_dtype(d->dtype_s)) return refuse("%s: unknown type %d", what, d->dtype_s);
    if (!is_temperature(d->temperature) ||
        !(d->forward >= 0.f) || !(d->reverse >= 0.f) || !std::isfinite(d->forward) || !std::isfinite(d->reverse))
        return refuse("%s: temperature %g or weights %g, %g are out of range", what, d->temperature, d->forward, d->reverse);
    if (!loss && !grad) return refuse("%s: neither loss nor gradient is asked for", what);
    if (const int rc = rows_wrong(what, "logits_s", s, d->ld_s, d->V, elem(d->dtype_s), false)) return rc;
    if (grad) {
        if (const int rc = rows_wrong(what, "grad", grad, d->ld_grad, d->V, elem(d->dtype_s), true)) return rc;
        if (overlaps(grad, d->ld_grad, elem(d->dtype_s), s, d->ld_s, elem(d->dtype_s), d->rows, d->V))
            return refuse("%s: grad overlaps logits_s", what);
    }
    return 0;
}

DistillArgs distill_args(const hbsjd_distill_desc* d, const void* s, const float* weight, float* loss, void* grad) {
    DistillArgs a = {};
    a.s = s;
    a.ld_s = d->ld_s;
    a.ld_t = d->ld_t;
    a.ld_g = d->ld_grad;
    a.weight = weight;
    a.loss = loss;
    a.grad = grad;
    a.V = d->V;
    a.temperature = d->temperature;
    a.forward = d->forward;
    a.reverse = d->reverse;
    return a;
}

}  // namespace

namespace hbsjd {
const char* last_detail() { return g_detail; }
}  // namespace hbsjd

extern "C" {

int hbsjd_adjust_logits(void* cuda_stream, const hbsjd_adjust_desc* d, const void* logits, const void* logits_u,
                        const float* bias, const uint32_t* mask, const int32_t* mask_row, const int32_t* history,
                        const int32_t* history_row, const int32_t* history_len, void* out) {
    const char* what = "hbsjd_adjust_logits";
    if (d && d->rows == 0) return HBSJD_OK;
    if (!d || !logits || !out) return refuse("%s: null argument", what);
    if (d->rows < 1 || d->rows > MAX_ROWS || d->V < 1 || d->V > MAX_LOGIT_V)
        return refuse("%s: %d rows of %d logits are out of range", what, d->rows, d->V);
    if (!is_dtype(d->dtype)) return refuse("%s: unknown type %d", what, d->dtype);
    const int b = elem(d->dtype);
    if (const int rc = rows_wrong(what, "logits", logits, d->ld, d->V, b, false)) return rc;
    if (const int rc = rows_wrong(what, "out", out, d->ld_out, d->V, b, true)) return rc;
    if (overlaps(out, d->ld_out, b, logits, d->ld, b, d->rows, d->V)) return refuse("%s: out overlaps logits", what);
    if (logits_u) {
        if (const int rc = rows_wrong(what, "logits_u", logits_u, d->ld_u, d->V, b, false)) return rc;
        if (overlaps(out, d->ld_out, b, logits_u, d->ld_u, b, d->rows, d->V)) return refuse("%s: out overlaps logits_u", what);
    }
    if (!is_aligned(bias, 4) || !is_aligned(mask, 4) || !is_aligned(history, 4) || !is_aligned(mask_row, 4) ||
        !is_aligned(history_row, 4) || !is_aligned(history_len, 4))
        return refuse("%s: an array of 4-byte elements is not aligned", what);
    if (!std::isfinite(d->cfg_scale) || !std::isfinite(d->frequency) || !std::isfinite(d->presence) ||
        !std::isfinite(d->repetition) || !(d->repetition > 0.f) || !std::isfinite(1.f / d->repetition))
        return refuse("%s: scale %g or penalties %g, %g, %g are out of range", what, d->cfg_scale, d->repetition, d->frequency,
                      d->presence);
    if (mask && (d->masks < 1 || d->ld_mask < (d->V + 31) / 32 || d->ld_mask > MAX_LD))
        return refuse("%s: %d masks of %lld words do not hold %d bits", what, d->masks, (long long)d->ld_mask, d->V);
    if (history && (d->sequences < 1 || d->history_cap < 1 || d->ld_history < d->history_cap || d->ld_history > MAX_LD))
        return refuse("%s: %d histories of %d tokens with stride %lld are out of range", what, d->sequences, d->history_cap,
                      (long long)d->ld_history);
    if (history && !history_row && d->sequences < d->rows)
        return refuse("%s: %d histories for %d rows without history_row", what, d->sequences, d->rows);
    AdjustArgs a = {};
    a.x = logits;
    a.u = logits_u;
    a.out = out;
    a.ld = d->ld;
    a.ld_u = d->ld_u;
    a.ld_out = d->ld_out;
    a.bias = bias;
    a.mask = mask;
    a.mask_row = mask_row;
    a.history = d->repetition == 1.f && d->frequency == 0.f && d->presence == 0.f ? nullptr : history;
    a.history_row = history_row;
    a.history_len = history_len;
    a.ld_mask = d->ld_mask;
    a.ld_history = d->ld_history;
    a.V = d->V;
    a.masks = d->masks;
    a.histories = d->sequences;
    a.history_cap = d->history_cap;
    a.cfg_scale = d->cfg_scale;
    a.repetition = d->repetition;
    a.frequency = d->frequency;
    a.presence = d->presence;
    Stream s((cudaStream_t)cuda_stream);
    return launched(what, launch_adjust(a, d->rows, d->dtype, s));
}

int hbsjd_topk_logits(void* cuda_stream, const hbsjd_topk_desc* d, const void* logits, float* values, int32_t* indices,
                      float* rest) {
    const char* what = "hbsjd_topk_logits";
    if (d && d->rows == 0) return HBSJD_OK;
    if (!d || !logits || !values || !indices) return refuse("%s: null argument", what);
    if (d->rows < 1 || d->rows > MAX_ROWS || d->V < 1 || d->V > MAX_LOGIT_V)
        return refuse("%s: %d rows of %d logits are out of range", what, d->rows, d->V);
    if (!is_dtype(d->dtype)) return refuse("%s: unknown type %d", what, d->dtype);
    if (d->k < 1 || d->k > MAX_LISTED || d->k > d->V) return refuse("%s: k = %d is out of range", what, d->k);
    if (!is_temperature(d->temperature))
        return refuse("%s: temperature %g is out of range", what, d->temperature);
    if (const int rc = rows_wrong(what, "logits", logits, d->ld, d->V, elem(d->dtype), false)) return rc;
    if (!is_aligned(values, 4) || !is_aligned(indices, 4) || !is_aligned(rest, 4))
        return refuse("%s: an array of 4-byte elements is not aligned", what);
    TopkArgs a = {};
    a.x = logits;
    a.ld = d->ld;
    a.values = values;
    a.indices = indices;
    a.rest = rest;
    a.V = d->V;
    a.k = d->k;
    a.temperature = d->temperature;
    Stream s((cudaStream_t)cuda_stream);
    return launched(what, launch_topk(a, d->rows, d->dtype, s));
}

int hbsjd_distill(void* cuda_stream, const hbsjd_distill_desc* d, const void* logits_s, const void* logits_t,
                  const float* weight, float* loss, void* grad) {
    const char* what = "hbsjd_distill";
    if (d && d->rows == 0) return HBSJD_OK;
    if (const int rc = distill_wrong(what, d, logits_s, loss, grad)) return rc;
    if (!logits_t) return refuse("%s: null argument", what);
    if (!is_dtype(d->dtype_t)) return refuse("%s: unknown type %d", what, d->dtype_t);
    if (const int rc = rows_wrong(what, "logits_t", logits_t, d->ld_t, d->V, elem(d->dtype_t), false)) return rc;
    if (overlaps(grad, d->ld_grad, elem(d->dtype_s), logits_t, d->ld_t, elem(d->dtype_t), d->rows, d->V))
        return refuse("%s: grad overlaps logits_t", what);
    if (!is_aligned(weight, 4) || !is_aligned(loss, 4)) return refuse("%s: an array of 4-byte elements is not aligned", what);
    DistillArgs a = distill_args(d, logits_s, weight, loss, grad);
    a.t = logits_t;
    Stream s((cudaStream_t)cuda_stream);
    return launched(what, launch_distill(a, d->rows, d->dtype_s, d->dtype_t, s));
}

int hbsjd_distill_topk(void* cuda_stream, const hbsjd_distill_desc* d, const void* logits_s, const float* values,
                       const int32_t* indices, const float* rest, const float* weight, float* loss, void* grad) {
    const char* what = "hbsjd_distill_topk";
    if (d && d->rows == 0) return HBSJD_OK;
    if (const int rc = distill_wrong(what, d, logits_s, loss, grad)) return rc;
    if (!values || !indices) return refuse("%s: null argument", what);
    if (d->k < 1 || d->k > MAX_LISTED) return refuse("%s: k = %d is out of range", what, d->k);
    if (!rest && d->reverse != 0.f)
        return refuse("%s: KL(student || teacher) is infinite where the teacher has no rest", what);
    if (!is_aligned(weight, 4) || !is_aligned(loss, 4) || !is_aligned(values, 4) || !is_aligned(indices, 4) ||
        !is_aligned(rest, 4))
        return refuse("%s: an array of 4-byte elements is not aligned", what);
    DistillArgs a = distill_args(d, logits_s, weight, loss, grad);
    a.values = values;
    a.indices = indices;
    a.rest = rest;
    a.k = d->k;
    Stream s((cudaStream_t)cuda_stream);
    return launched(what, launch_distill_topk(a, d->rows, d->dtype_s, s));
}

}  // extern "C"
