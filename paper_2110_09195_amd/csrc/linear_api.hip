// C entry points of the projections of real-valued activations: argument checks, dispatch.
#include "linear.h"

using namespace snn;

namespace {

bool desc_ok(const snn_linear_desc *d)
{
    if (!d) return false;
    if (d->groups < 1 || d->groups > 1024 || d->K < 1 || d->K > 256) return false;
    if (d->C_in < 8 || d->C_in > 65536 || d->C_in % 8 || d->C_out < 8 || d->C_out > 65536 || d->C_out % 8) return false;
    return d->dtype == SNN_DTYPE_BF16 || d->dtype == SNN_DTYPE_F16;
}

bool count_ok(int64_t rows) { return rows >= 0 && rows < ((int64_t)1 << 28); }

bool aligned(const void *p, unsigned a) { return ((uintptr_t)p & (a - 1)) == 0; }

// rows of C 16-bit values, `ld` apart
bool rows_ok(const void *p, int64_t ld, int C, int64_t rows)
{
    if (ld < C || ld % 8 || ld > (1 << 20)) return false;
    return rows == 0 || (p && aligned(p, 16));
}

bool weights_ok(const LinearGeom &g, const void *w, size_t bytes) { return w && aligned(w, 256) && bytes >= g.bytes; }

bool adapters_ok(const snn_adapters *a)
{
    return a && a->n >= 1 && a->n <= 65536 && a->rank >= 8 && a->rank <= 128 && a->rank % 8 == 0;
}

bool adapter_weights_ok(const snn_adapters *a) { return a->A && a->B && a->scale && aligned(a->A, 16) && aligned(a->B, 16); }

int rows_call(const snn_linear_desc *desc, bool grad, const void *in, int64_t ld_in, int64_t rows, const int32_t *offsets,
              const void *weights, size_t weights_bytes, void *out, int64_t ld_out, void *stream)
{
    if (!desc_ok(desc) || !count_ok(rows) || (!offsets && desc->groups != 1)) return SNN_ERR_INVALID_ARG;
    if (!rows_ok(in, ld_in, grad ? desc->C_out : desc->C_in, rows) || !rows_ok(out, ld_out, grad ? desc->C_in : desc->C_out, rows))
        return SNN_ERR_INVALID_ARG;
    const LinearGeom g = make_linear_geom(*desc);
    if (!weights_ok(g, weights, weights_bytes)) return SNN_ERR_WORKSPACE;
    if (rows == 0) return SNN_OK;
    return launch_linear_rows(g, grad, in, ld_in, rows, offsets, weights, out, ld_out, nullptr, nullptr, nullptr, (hipStream_t)stream);
}

// the 8-bit form of activations: q rows lie C apart
bool kept_ok(const int8_t *q, const uint8_t *e, int64_t rows) { return rows == 0 || (q && e && aligned(q, 16) && aligned(e, 4)); }

int weight_grad_call(const snn_linear_desc *desc, const RowsIn &x, const void *dy, int64_t lddy, int64_t rows, const int32_t *offsets,
                     const void *weights, size_t weights_bytes, float *dw, float *dalpha, void *workspace, size_t ws_bytes,
                     void *stream)
{
    if (!offsets && desc->groups != 1) return SNN_ERR_INVALID_ARG;
    if (!rows_ok(dy, lddy, desc->C_out, rows) || !dw || !aligned(dw, 16)) return SNN_ERR_INVALID_ARG;
    const LinearGeom g = make_linear_geom(*desc);
    if (!weights_ok(g, weights, weights_bytes)) return SNN_ERR_WORKSPACE;
    if (!workspace || !aligned(workspace, 256) || ws_bytes < linear_weight_grad_workspace_bytes(g, rows, x.e != nullptr)) return SNN_ERR_WORKSPACE;
    return launch_linear_weight_grad(g, x, dy, lddy, rows, offsets, weights, dw, dalpha, workspace, (hipStream_t)stream);
}

int adapters_backward_call(const snn_linear_desc *desc, const snn_adapters *a, const RowsIn &x, const float *low, const void *dy,
                           int64_t lddy, int64_t rows, const int32_t *adapter, const void *weights, size_t weights_bytes, void *dx,
                           int64_t lddx, void *dA, void *dB, void *workspace, size_t ws_bytes, void *stream)
{
    if (!rows_ok(dy, lddy, desc->C_out, rows) || !rows_ok(dx, lddx, desc->C_in, rows) || !adapter_weights_ok(a)) return SNN_ERR_INVALID_ARG;
    if ((rows > 0 && (!adapter || !low || !aligned(low, 16))) || !dA || !dB || !aligned(dA, 16) || !aligned(dB, 16)) return SNN_ERR_INVALID_ARG;
    if (desc->groups != 1) return SNN_ERR_UNSUPPORTED;
    const LinearGeom g = make_linear_geom(*desc);
    if (!weights_ok(g, weights, weights_bytes)) return SNN_ERR_WORKSPACE;
    if (!workspace || !aligned(workspace, 256) || ws_bytes < adapters_workspace_bytes(g, a->n, a->rank, rows, true, x.e != nullptr)) return SNN_ERR_WORKSPACE;
    const Adapters ad = {a->n, a->rank, a->A, a->B, a->scale, adapter};
    return launch_adapters_backward(g, ad, x, low, dy, lddy, rows, weights, dx, lddx, dA, dB, workspace, (hipStream_t)stream);
}

}  // namespace

extern "C" {

size_t snn_linear_weights_bytes(const snn_linear_desc *desc) { return desc_ok(desc) ? make_linear_geom(*desc).bytes : 0; }

int snn_linear_prepare(const snn_linear_desc *desc, const uint16_t *codebook8, const uint16_t *idx, const void *alpha,
                       void *weights, size_t weights_bytes, void *stream)
{
    if (!desc_ok(desc) || !codebook8 || !idx || !alpha || !aligned(alpha, 16)) return SNN_ERR_INVALID_ARG;
    const LinearGeom g = make_linear_geom(*desc);
    if (!weights_ok(g, weights, weights_bytes)) return SNN_ERR_WORKSPACE;
    return launch_linear_prepare(g, codebook8, idx, alpha, weights, (hipStream_t)stream);
}

int snn_linear_forward(const snn_linear_desc *desc, const void *x, int64_t ldx, int64_t rows, const int32_t *offsets,
                       const void *weights, size_t weights_bytes, void *y, int64_t ldy, void *stream)
{
    return rows_call(desc, false, x, ldx, rows, offsets, weights, weights_bytes, y, ldy, stream);
}

int snn_linear_input_grad(const snn_linear_desc *desc, const void *dy, int64_t lddy, int64_t rows, const int32_t *offsets,
                          const void *weights, size_t weights_bytes, void *dx, int64_t lddx, void *stream)
{
    return rows_call(desc, true, dy, lddy, rows, offsets, weights, weights_bytes, dx, lddx, stream);
}

int snn_checkpoint_store(const void *x, int64_t ldx, int64_t rows, int C, int dtype, int8_t *q, uint8_t *e, void *stream)
{
    if (!count_ok(rows) || C < 8 || C > 65536 || C % 8 || (dtype != SNN_DTYPE_BF16 && dtype != SNN_DTYPE_F16)) return SNN_ERR_INVALID_ARG;
    if (!rows_ok(x, ldx, C, rows) || !kept_ok(q, e, rows)) return SNN_ERR_INVALID_ARG;
    if (rows == 0) return SNN_OK;
    return launch_checkpoint_store(x, ldx, rows, C, dtype, q, e, (hipStream_t)stream);
}

int snn_checkpoint_restore(const int8_t *q, const uint8_t *e, int64_t rows, int C, int dtype, void *x, int64_t ldx, void *stream)
{
    if (!count_ok(rows) || C < 8 || C > 65536 || C % 8 || (dtype != SNN_DTYPE_BF16 && dtype != SNN_DTYPE_F16)) return SNN_ERR_INVALID_ARG;
    if (!rows_ok(x, ldx, C, rows) || !kept_ok(q, e, rows)) return SNN_ERR_INVALID_ARG;
    if (rows == 0) return SNN_OK;
    return launch_checkpoint_restore(q, e, rows, C, dtype, x, ldx, (hipStream_t)stream);
}

size_t snn_linear_weight_grad_workspace_bytes(const snn_linear_desc *desc, int64_t rows, int checkpoint)
{
    return desc_ok(desc) && count_ok(rows) ? linear_weight_grad_workspace_bytes(make_linear_geom(*desc), rows, checkpoint != 0) : 0;
}

int snn_linear_weight_grad(const snn_linear_desc *desc, const void *x, int64_t ldx, const void *dy, int64_t lddy, int64_t rows,
                           const int32_t *offsets, const void *weights, size_t weights_bytes, float *dw, float *dalpha,
                           void *workspace, size_t ws_bytes, void *stream)
{
    if (!desc_ok(desc) || !count_ok(rows) || !rows_ok(x, ldx, desc->C_in, rows)) return SNN_ERR_INVALID_ARG;
    return weight_grad_call(desc, {x, nullptr, ldx}, dy, lddy, rows, offsets, weights, weights_bytes, dw, dalpha, workspace, ws_bytes, stream);
}

int snn_linear_weight_grad_checkpoint(const snn_linear_desc *desc, const int8_t *q, const uint8_t *e, const void *dy, int64_t lddy,
                                      int64_t rows, const int32_t *offsets, const void *weights, size_t weights_bytes, float *dw,
                                      float *dalpha, void *workspace, size_t ws_bytes, void *stream)
{
    if (!desc_ok(desc) || !count_ok(rows) || !kept_ok(q, e, rows)) return SNN_ERR_INVALID_ARG;
    // (no rows: nothing is read; the form is told by e)
    static const uint8_t none = 0;
    return weight_grad_call(desc, {q, e ? e : &none, desc->C_in}, dy, lddy, rows, offsets, weights, weights_bytes, dw, dalpha, workspace,
                            ws_bytes, stream);
}

size_t snn_adapters_workspace_bytes(const snn_linear_desc *desc, const snn_adapters *adapters, int64_t rows, int call)
{
    if (!desc_ok(desc) || desc->groups != 1 || !adapters_ok(adapters) || !count_ok(rows)) return 0;
    if (call < SNN_ADAPTERS_FORWARD || call > SNN_ADAPTERS_BACKWARD_CHECKPOINT) return 0;
    return adapters_workspace_bytes(make_linear_geom(*desc), adapters->n, adapters->rank, rows, call != SNN_ADAPTERS_FORWARD,
                                    call == SNN_ADAPTERS_BACKWARD_CHECKPOINT);
}

int snn_adapters_forward(const snn_linear_desc *desc, const snn_adapters *a, const void *x, int64_t ldx, int64_t rows,
                         const int32_t *adapter, const void *weights, size_t weights_bytes, void *y, int64_t ldy, float *low,
                         void *workspace, size_t ws_bytes, void *stream)
{
    if (!desc_ok(desc) || !adapters_ok(a) || !adapter_weights_ok(a) || !count_ok(rows)) return SNN_ERR_INVALID_ARG;
    if (!rows_ok(x, ldx, desc->C_in, rows) || !rows_ok(y, ldy, desc->C_out, rows) || (rows > 0 && !adapter) || !aligned(low, 16))
        return SNN_ERR_INVALID_ARG;
    if (desc->groups != 1) return SNN_ERR_UNSUPPORTED;
    const LinearGeom g = make_linear_geom(*desc);
    if (!weights_ok(g, weights, weights_bytes)) return SNN_ERR_WORKSPACE;
    if (!workspace || !aligned(workspace, 256) || ws_bytes < adapters_workspace_bytes(g, a->n, a->rank, rows, false, false)) return SNN_ERR_WORKSPACE;
    if (rows == 0) return SNN_OK;
    const Adapters ad = {a->n, a->rank, a->A, a->B, a->scale, adapter};
    return launch_adapters_forward(g, ad, x, ldx, rows, weights, y, ldy, low, workspace, (hipStream_t)stream);
}

int snn_adapters_backward(const snn_linear_desc *desc, const snn_adapters *a, const void *x, int64_t ldx, const float *low,
                          const void *dy, int64_t lddy, int64_t rows, const int32_t *adapter, const void *weights,
                          size_t weights_bytes, void *dx, int64_t lddx, void *dA, void *dB, void *workspace, size_t ws_bytes,
                          void *stream)
{
    if (!desc_ok(desc) || !adapters_ok(a) || !count_ok(rows) || !rows_ok(x, ldx, desc->C_in, rows)) return SNN_ERR_INVALID_ARG;
    return adapters_backward_call(desc, a, {x, nullptr, ldx}, low, dy, lddy, rows, adapter, weights, weights_bytes, dx, lddx, dA, dB,
                                  workspace, ws_bytes, stream);
}

int snn_adapters_backward_checkpoint(const snn_linear_desc *desc, const snn_adapters *a, const int8_t *q, const uint8_t *e,
                                     const float *low, const void *dy, int64_t lddy, int64_t rows, const int32_t *adapter,
                                     const void *weights, size_t weights_bytes, void *dx, int64_t lddx, void *dA, void *dB,
                                     void *workspace, size_t ws_bytes, void *stream)
{
    if (!desc_ok(desc) || !adapters_ok(a) || !count_ok(rows) || !kept_ok(q, e, rows)) return SNN_ERR_INVALID_ARG;
    static const uint8_t none = 0;
    return adapters_backward_call(desc, a, {q, e ? e : &none, desc->C_in}, low, dy, lddy, rows, adapter, weights, weights_bytes, dx,
                                  lddx, dA, dB, workspace, ws_bytes, stream);
}

}  // extern "C"
