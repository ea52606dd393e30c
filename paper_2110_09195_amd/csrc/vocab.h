// The ends of a network over tokens: a table of 16-bit rows, a row for each token of a vocabulary; what the calls on it share.
#pragma once

#include "linear.h"

namespace snn {

struct Vocab {
    int V, C, dtype;
};

// Rows of activations or of the table, `ld` elements apart.
struct Rows16 {
    const void *p;
    int64_t ld;
};

int launch_embedding_forward(const Vocab &v, const Rows16 &table, const int32_t *ids, int64_t rows, float scale, void *y, int64_t ldy, hipStream_t s);
size_t embedding_grad_workspace_bytes(const Vocab &v, int64_t rows);
int launch_embedding_grad(const Vocab &v, const Rows16 &dy, const int32_t *ids, int64_t rows, float scale, void *dtable, bool accumulate, void *ws,
                          hipStream_t s);

// What a row is held against: one token (k = 0), or k tokens with a teacher's logits.
struct Targets {
    const int32_t *ids;               // [rows], [rows][k]
    const float *logits;              // [rows][k]
    int k;
    float temperature;
};

size_t loss_workspace_bytes(const Vocab &v, int64_t rows, const Targets &t, bool backward);
int launch_loss_forward(const Vocab &v, const Rows16 &x, int64_t rows, const Rows16 &table, const Targets &t, float *loss, float *lse, float *picked,
                        void *ws, hipStream_t s);
int launch_loss_backward(const Vocab &v, const Rows16 &x, int64_t rows, const Rows16 &table, const Targets &t, const float *lse, const float *dloss,
                         void *dx, int64_t lddx, void *dtable, bool accumulate, void *ws, hipStream_t s);

}  // namespace snn
