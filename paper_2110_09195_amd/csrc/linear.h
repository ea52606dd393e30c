// Projections of real-valued activations by sub-bit weights: geometry, the layout of prepared weights, launchers.
#pragma once

#include "snn_internal.h"

namespace snn {

// The bits of a weight matrix as the matrix instructions' operand is made from them: blocks of 32 output columns n by 64 of the
// contracted axis k, 64 words a block, word of lane l = 32 h + n % 32.  A lane's word holds the signs of k = 64 kb + 16 s + 8 h + j
// (s < 4, j < 8): of the pair (j = 2 r, 2 r + 1), which shares a register of the operand, at bits 15 - (4 s + r) and
// 31 - (4 s + r): shifted left by 4 s + r they are the sign bits of the pair.  Set for -1.
// Two images: F for the outputs (n = output channel, k = input channel), D for the gradient of the inputs (the other way round).
struct LinearGeom {
    int G, C_in, C_out, K, dtype;
    int nb_f, kb_f, nb_d, kb_d;       // blocks of 32 columns and of 64 contracted channels, of either image
    uint32_t words_f, words_d;        // per group
    uint32_t alpha_stride;            // elements per group, whole blocks of 64, zeros behind C_out
    size_t at_d, at_alpha, bytes;     // of the prepared weights (F is at 0)
};

inline LinearGeom make_linear_geom(const snn_linear_desc &d)
{
    LinearGeom g;
    g.G = d.groups; g.C_in = d.C_in; g.C_out = d.C_out; g.K = d.K; g.dtype = d.dtype;
    g.nb_f = (d.C_out + 31) / 32; g.kb_f = (d.C_in + 63) / 64;
    g.nb_d = (d.C_in + 31) / 32;  g.kb_d = (d.C_out + 63) / 64;
    g.words_f = (uint32_t)g.nb_f * g.kb_f * 64;
    g.words_d = (uint32_t)g.nb_d * g.kb_d * 64;
    g.alpha_stride = (uint32_t)g.kb_d * 64;
    g.at_d = align_up((size_t)g.G * g.words_f * 4, 256);
    g.at_alpha = g.at_d + align_up((size_t)g.G * g.words_d * 4, 256);
    g.bytes = g.at_alpha + align_up((size_t)g.G * g.alpha_stride * 2, 256);
    return g;
}

// Rows of one kind of activations: 16-bit values `ld` elements apart, or (e != nullptr) their 8-bit form, `ld` = the channels.
struct RowsIn {
    const void *p;
    const uint8_t *e;
    int64_t ld;
};

struct Adapters {
    int n, rank;
    const void *A, *B;
    const float *scale;
    const int32_t *of_row;
};

int launch_linear_prepare(const LinearGeom &g, const uint16_t *codebook, const uint16_t *idx, const void *alpha, void *weights, hipStream_t s);

// rows through the F image (grad = false: x -> y) or the D image (grad = true: dy -> dx); ad != nullptr: with the adapters' share, from
// `low` (fp32 [rows][rank], scale applied) and `up`, [n][columns of the output][rank]
int launch_linear_rows(const LinearGeom &g, bool grad, const void *in, int64_t ld_in, int64_t rows, const int32_t *offsets,
                       const void *weights, void *out, int64_t ld_out, const Adapters *ad, const void *up, const float *low, hipStream_t s);

// few rows with the adapters' inner products made by the same launch: whether a call is one of these, and it
bool adapters_in_one_launch(const LinearGeom &g, int64_t rows, int rank);
int launch_adapters_in_one(const LinearGeom &g, const Adapters &ad, const void *x, int64_t ldx, int64_t rows, const void *weights, void *y, int64_t ldy,
                           float *low, hipStream_t s);

size_t linear_weight_grad_workspace_bytes(const LinearGeom &g, int64_t rows, bool kept);
int launch_linear_weight_grad(const LinearGeom &g, const RowsIn &x, const void *dy, int64_t lddy, int64_t rows, const int32_t *offsets,
                              const void *weights, float *dw, float *dalpha, void *ws, hipStream_t s);

size_t adapters_workspace_bytes(const LinearGeom &g, int n, int rank, int64_t rows, bool backward, bool kept);
int launch_adapters_forward(const LinearGeom &g, const Adapters &ad, const void *x, int64_t ldx, int64_t rows, const void *weights,
                            void *y, int64_t ldy, float *low, void *ws, hipStream_t s);
int launch_adapters_backward(const LinearGeom &g, const Adapters &ad, const RowsIn &x, const float *low, const void *dy, int64_t lddy,
                             int64_t rows, const void *weights, void *dx, int64_t lddx, void *dA, void *dB, void *ws, hipStream_t s);

int launch_checkpoint_store(const void *x, int64_t ldx, int64_t rows, int C, int dtype, int8_t *q, uint8_t *e, hipStream_t s);
int launch_checkpoint_restore(const int8_t *q, const uint8_t *e, int64_t rows, int C, int dtype, void *x, int64_t ldx, hipStream_t s);

// ---- device helpers ------------------------------------------------------------------------------------------

// rows of group g, whatever the offsets hold: [lo, hi) inside 0 .. rows
__device__ inline void group_rows(const int32_t *offsets, int g, int rows, int &lo, int &hi)
{
    if (!offsets) { lo = 0; hi = rows; return; }
    lo = min(max(offsets[g], 0), rows);
    hi = min(max(offsets[g + 1], lo), rows);
}

// 2^(e - 127); the stored exponents are 1 .. 254
__device__ inline float unit_of(uint32_t e) { return __uint_as_float(e << 23); }

// the value that q of a chunk with unit u stands for
__device__ inline float kept_value(int q, float u) { return q == -128 ? __uint_as_float(0x7fc00000u) : (float)q * u; }

}  // namespace snn
