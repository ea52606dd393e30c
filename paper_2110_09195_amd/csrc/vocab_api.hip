// C entry points of the ends of a network over tokens: argument checks, dispatch.
#include "vocab.h"

using namespace snn;

namespace {

bool desc_ok(const snn_vocab_desc *d)
{
    if (!d || d->V < 1 || d->V > (1 << 24) || d->C < 8 || d->C > 65536 || d->C % 8) return false;
    return d->dtype == SNN_DTYPE_BF16 || d->dtype == SNN_DTYPE_F16;
}

Vocab vocab(const snn_vocab_desc *d) { return {d->V, d->C, d->dtype}; }

bool count_ok(int64_t rows) { return rows >= 0 && rows < ((int64_t)1 << 28); }

bool aligned(const void *p, unsigned a) { return ((uintptr_t)p & (a - 1)) == 0; }

// rows of C 16-bit values, `ld` apart
bool rows_ok(const void *p, int64_t ld, int C, int64_t rows)
{
    if (ld < C || ld % 8 || ld > (1 << 20)) return false;
    return rows == 0 || (p && aligned(p, 16));
}

bool words_ok(const void *p, int64_t rows) { return rows == 0 || (p && aligned(p, 4)); }

bool workspace_ok(const void *ws, size_t bytes, size_t need) { return ws && aligned(ws, 256) && bytes >= need; }

bool temperature_ok(float t) { return t >= 1.0f / 1024 && t <= 1024.0f; }       // (not for NaN)

bool targets_ok(const Targets &t, int64_t rows)
{
    if (t.k < 0 || t.k > 256 || !temperature_ok(t.temperature)) return false;
    return words_ok(t.ids, rows) && (t.k == 0 || words_ok(t.logits, rows));
}

int forward_call(const snn_vocab_desc *desc, const void *x, int64_t ldx, int64_t rows, const void *table, int64_t ldt, const Targets &t, float *loss,
                 float *lse, float *picked, void *workspace, size_t ws_bytes, void *stream)
{
    if (!desc_ok(desc) || !count_ok(rows) || !rows_ok(x, ldx, desc->C, rows) || !rows_ok(table, ldt, desc->C, 1) || !targets_ok(t, rows))
        return SNN_ERR_INVALID_ARG;
    if (!words_ok(loss, rows) || !words_ok(lse, rows) || (t.k && !words_ok(picked, rows))) return SNN_ERR_INVALID_ARG;
    const Vocab v = vocab(desc);
    if (!workspace_ok(workspace, ws_bytes, loss_workspace_bytes(v, rows, t, false))) return SNN_ERR_WORKSPACE;
    if (rows == 0) return SNN_OK;
    return launch_loss_forward(v, {x, ldx}, rows, {table, ldt}, t, loss, lse, picked, workspace, (hipStream_t)stream);
}

int backward_call(const snn_vocab_desc *desc, const void *x, int64_t ldx, int64_t rows, const void *table, int64_t ldt, const Targets &t,
                  const float *lse, const float *dloss, void *dx, int64_t lddx, void *dtable, int accumulate, void *workspace, size_t ws_bytes,
                  void *stream)
{
    if (!desc_ok(desc) || !count_ok(rows) || !rows_ok(x, ldx, desc->C, rows) || !rows_ok(table, ldt, desc->C, 1) || !targets_ok(t, rows))
        return SNN_ERR_INVALID_ARG;
    if (!words_ok(lse, rows) || !words_ok(dloss, rows) || (!dx && !dtable) || !aligned(dtable, 16)) return SNN_ERR_INVALID_ARG;
    if (dx && !rows_ok(dx, lddx, desc->C, rows)) return SNN_ERR_INVALID_ARG;
    const Vocab v = vocab(desc);
    if (!workspace_ok(workspace, ws_bytes, loss_workspace_bytes(v, rows, t, true))) return SNN_ERR_WORKSPACE;
    if (rows == 0 && (!dtable || accumulate)) return SNN_OK;
    return launch_loss_backward(v, {x, ldx}, rows, {table, ldt}, t, lse, dloss, dx, lddx, dtable, accumulate != 0, workspace, (hipStream_t)stream);
}

}  // namespace

extern "C" {

int snn_embedding_forward(const snn_vocab_desc *desc, const void *table, int64_t ldt, const int32_t *ids, int64_t rows, float scale, void *y, int64_t ldy,
                          void *stream)
{
    if (!desc_ok(desc) || !count_ok(rows) || !rows_ok(table, ldt, desc->C, 1) || !words_ok(ids, rows) || !rows_ok(y, ldy, desc->C, rows))
        return SNN_ERR_INVALID_ARG;
    if (rows == 0) return SNN_OK;
    return launch_embedding_forward(vocab(desc), {table, ldt}, ids, rows, scale, y, ldy, (hipStream_t)stream);
}

size_t snn_embedding_grad_workspace_bytes(const snn_vocab_desc *desc, int64_t rows)
{
    if (!desc_ok(desc) || !count_ok(rows)) return 0;
    const size_t n = embedding_grad_workspace_bytes(vocab(desc), rows);
    return n ? n : 256;
}

int snn_embedding_grad(const snn_vocab_desc *desc, const void *dy, int64_t lddy, const int32_t *ids, int64_t rows, float scale, void *dtable,
                       int accumulate, void *workspace, size_t ws_bytes, void *stream)
{
    if (!desc_ok(desc) || !count_ok(rows) || !rows_ok(dy, lddy, desc->C, rows) || !words_ok(ids, rows) || !dtable || !aligned(dtable, 16))
        return SNN_ERR_INVALID_ARG;
    if (!workspace_ok(workspace, ws_bytes, snn_embedding_grad_workspace_bytes(desc, rows))) return SNN_ERR_WORKSPACE;
    return launch_embedding_grad(vocab(desc), {dy, lddy}, ids, rows, scale, dtable, accumulate != 0, workspace, (hipStream_t)stream);
}

size_t snn_loss_workspace_bytes(const snn_vocab_desc *desc, int64_t rows, int k, int call)
{
    if (!desc_ok(desc) || !count_ok(rows) || k < 0 || k > 256 || (call != SNN_LOSS_FORWARD && call != SNN_LOSS_BACKWARD)) return 0;
    return loss_workspace_bytes(vocab(desc), rows, {nullptr, nullptr, k, 1.0f}, call == SNN_LOSS_BACKWARD);
}

int snn_cross_entropy_forward(const snn_vocab_desc *desc, const void *x, int64_t ldx, int64_t rows, const void *table, int64_t ldt,
                              const int32_t *target, float *loss, float *lse, void *workspace, size_t ws_bytes, void *stream)
{
    return forward_call(desc, x, ldx, rows, table, ldt, {target, nullptr, 0, 1.0f}, loss, lse, nullptr, workspace, ws_bytes, stream);
}

int snn_cross_entropy_backward(const snn_vocab_desc *desc, const void *x, int64_t ldx, int64_t rows, const void *table, int64_t ldt,
                               const int32_t *target, const float *lse, const float *dloss, void *dx, int64_t lddx, void *dtable, int accumulate,
                               void *workspace, size_t ws_bytes, void *stream)
{
    return backward_call(desc, x, ldx, rows, table, ldt, {target, nullptr, 0, 1.0f}, lse, dloss, dx, lddx, dtable, accumulate, workspace, ws_bytes, stream);
}

int snn_distill_forward(const snn_vocab_desc *desc, const void *x, int64_t ldx, int64_t rows, const void *table, int64_t ldt, const int32_t *ids,
                        const float *logits, int k, float temperature, float *loss, float *lse, float *picked, void *workspace, size_t ws_bytes,
                        void *stream)
{
    if (k < 1) return SNN_ERR_INVALID_ARG;
    return forward_call(desc, x, ldx, rows, table, ldt, {ids, logits, k, temperature}, loss, lse, picked, workspace, ws_bytes, stream);
}

int snn_distill_backward(const snn_vocab_desc *desc, const void *x, int64_t ldx, int64_t rows, const void *table, int64_t ldt, const int32_t *ids,
                         const float *logits, int k, float temperature, const float *lse, const float *dloss, void *dx, int64_t lddx, void *dtable,
                         int accumulate, void *workspace, size_t ws_bytes, void *stream)
{
    if (k < 1) return SNN_ERR_INVALID_ARG;
    return backward_call(desc, x, ldx, rows, table, ldt, {ids, logits, k, temperature}, lse, dloss, dx, lddx, dtable, accumulate, workspace, ws_bytes,
                         stream);
}

}  // extern "C"
