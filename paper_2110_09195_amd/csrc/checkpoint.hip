// Activations kept in 8 bits: chunks of 32 channels of a row share a power of two.
#include "linear.h"

namespace snn {

namespace {

constexpr int CHUNK = 32;

// The unit's biased exponent: that of the largest finite magnitude less 6, not below 2^-126.
__device__ inline uint32_t unit_exponent(float top)
{
    return (uint32_t)max((int)(__float_as_uint(top) >> 23) - 6, 1);
}

template <class T>
__global__ __launch_bounds__(256)
void checkpoint_store_kernel(const T *__restrict__ x, int64_t ldx, int64_t rows, int C, int8_t *__restrict__ q, uint8_t *__restrict__ e)
{
    const int chunks = (C + CHUNK - 1) / CHUNK;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= rows * chunks) return;
    const int64_t t = i / chunks;
    const int c0 = (int)(i % chunks) * CHUNK, c1 = min(c0 + CHUNK, C);
    float top = 0.0f;
    for (int c = c0; c < c1; ++c) {
        const float v = fabsf((float)x[t * ldx + c]);
        if (v < INFINITY) top = fmaxf(top, v);
    }
    const uint32_t ue = unit_exponent(top);
    const float inv = unit_of(254 - ue);
    for (int c = c0; c < c1; ++c) {
        const float v = (float)x[t * ldx + c];
        q[t * C + c] = fabsf(v) < INFINITY ? (int8_t)fminf(fmaxf(rintf(v * inv), -127.0f), 127.0f) : (int8_t)-128;
    }
    e[i] = (uint8_t)ue;
}

template <class T>
__global__ __launch_bounds__(256)
void checkpoint_restore_kernel(const int8_t *__restrict__ q, const uint8_t *__restrict__ e, int64_t rows, int C, T *__restrict__ x, int64_t ldx)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= rows * C) return;
    const int64_t t = i / C;
    const int c = (int)(i % C);
    x[t * ldx + c] = (T)kept_value(q[i], unit_of(e[t * ((C + CHUNK - 1) / CHUNK) + c / CHUNK]));
}

}  // namespace

int launch_checkpoint_store(const void *x, int64_t ldx, int64_t rows, int C, int dtype, int8_t *q, uint8_t *e, hipStream_t s)
{
    const unsigned blocks = (unsigned)((rows * ((C + CHUNK - 1) / CHUNK) + 255) / 256);
    if (dtype == SNN_DTYPE_BF16)
        checkpoint_store_kernel<__bf16><<<blocks, 256, 0, s>>>((const __bf16 *)x, ldx, rows, C, q, e);
    else
        checkpoint_store_kernel<_Float16><<<blocks, 256, 0, s>>>((const _Float16 *)x, ldx, rows, C, q, e);
    return check_launch();
}

int launch_checkpoint_restore(const int8_t *q, const uint8_t *e, int64_t rows, int C, int dtype, void *x, int64_t ldx, hipStream_t s)
{
    const unsigned blocks = (unsigned)((rows * C + 255) / 256);
    if (dtype == SNN_DTYPE_BF16)
        checkpoint_restore_kernel<__bf16><<<blocks, 256, 0, s>>>(q, e, rows, C, (__bf16 *)x, ldx);
    else
        checkpoint_restore_kernel<_Float16><<<blocks, 256, 0, s>>>(q, e, rows, C, (_Float16 *)x, ldx);
    return check_launch();
}

}  // namespace snn
