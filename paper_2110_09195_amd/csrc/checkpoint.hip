// Activations kept in 8 bits: chunks of 32 channels of a row share a power of two.  Both directions move memory and nothing else counts:
// a thread takes 8 channels (16 bytes one side, 8 the other), four neighbouring lanes a chunk.  16384 rows of 8192 channels: 73 - 88 us to
// store, 66 to restore, 407 MB each: 5.1 TB/s and 6.1, a copy's rate (5.05) and, where some is still in the last cache, more.
#include "linear_device.h"

namespace snn {

namespace {

// The unit's biased exponent: that of the largest finite magnitude less 6, not below 2^-126.
__device__ inline uint32_t unit_exponent(float top)
{
    return (uint32_t)max((int)(__float_as_uint(top) >> 23) - 6, 1);
}

template <class T>
__global__ __launch_bounds__(256)
void checkpoint_store_kernel(const T *__restrict__ x, int64_t ldx, Walk w, int C, int8_t *__restrict__ q, uint8_t *__restrict__ e)
{
    using v8 = typename Half<T>::v8;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    int64_t t = id / w.pieces;
    int p = (int)(id - t * w.pieces);
    for (; t < w.rows; t += w.step_rows) {
        const bool in = p * 8 < C;
        u32x4 raw = {0, 0, 0, 0};
        if (in) raw = *(const u32x4 *)(x + t * ldx + p * 8);
        const v8 v = __builtin_bit_cast(v8, raw);
        float f[8], top = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            f[i] = (float)v[i];
            const float m = fabsf(f[i]);
            top = fmaxf(top, m < INFINITY ? m : 0.0f);
        }
        // (lanes of a chunk are in step: pieces is a multiple of 4, and so is the stride)
        top = fmaxf(top, __shfl_xor(top, 1));
        top = fmaxf(top, __shfl_xor(top, 2));
        const uint32_t ue = unit_exponent(top);
        const float inv = unit_of(254 - ue);
        uint32_t out[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int k = fabsf(f[i]) < INFINITY ? (int)fminf(fmaxf(rintf(f[i] * inv), -127.0f), 127.0f) : -128;
            out[i >> 2] |= (uint32_t)(k & 255) << (8 * (i & 3));
        }
        if (in) *(uint2 *)(q + t * C + p * 8) = make_uint2(out[0], out[1]);
        if ((p & 3) == 0) e[t * (w.pieces >> 2) + (p >> 2)] = (uint8_t)ue;
        p += w.step_pieces;
        if (p >= w.pieces) {
            p -= w.pieces;
            ++t;
        }
    }
}

template <class T>
__global__ __launch_bounds__(256)
void checkpoint_restore_kernel(const int8_t *__restrict__ q, const uint8_t *__restrict__ e, Walk w, int C, T *__restrict__ x, int64_t ldx)
{
    restore_rows(q, e, w, C, x, ldx, blockIdx.x);
}

}  // namespace

int launch_checkpoint_store(const void *x, int64_t ldx, int64_t rows, int C, int dtype, int8_t *q, uint8_t *e, hipStream_t s)
{
    Walk w;
    const unsigned grid = walk_of(rows, C, w);
    if (dtype == SNN_DTYPE_BF16)
        checkpoint_store_kernel<__bf16><<<grid, 256, 0, s>>>((const __bf16 *)x, ldx, w, C, q, e);
    else
        checkpoint_store_kernel<_Float16><<<grid, 256, 0, s>>>((const _Float16 *)x, ldx, w, C, q, e);
    return check_launch();
}

int launch_checkpoint_restore(const int8_t *q, const uint8_t *e, int64_t rows, int C, int dtype, void *x, int64_t ldx, hipStream_t s)
{
    Walk w;
    const unsigned grid = walk_of(rows, C, w);
    if (dtype == SNN_DTYPE_BF16)
        checkpoint_restore_kernel<__bf16><<<grid, 256, 0, s>>>(q, e, w, C, (__bf16 *)x, ldx);
    else
        checkpoint_restore_kernel<_Float16><<<grid, 256, 0, s>>>(q, e, w, C, (_Float16 *)x, ldx);
    return check_launch();
}

}  // namespace snn
