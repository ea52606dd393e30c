// Gradients of the weights of projections, from activations or from their 8-bit form.
#include "linear.h"

namespace snn {

namespace {

template <class T>
__device__ inline float row_value(const RowsIn &x, int C, int64_t t, int c)
{
    if (!x.e) return (float)((const T *)x.p)[t * x.ld + c];
    return kept_value(((const int8_t *)x.p)[t * x.ld + c], unit_of(x.e[t * ((C + 31) / 32) + c / 32]));
}

// One thread an element of G; a block one row of it, whose sum with the weights is the scale's gradient.
template <class T>
__global__ __launch_bounds__(256)
void linear_weight_grad_kernel(LinearGeom g, RowsIn x, const T *__restrict__ dy, int64_t lddy, int rows, const int32_t *__restrict__ offsets,
                               const uint32_t *__restrict__ image, const T *__restrict__ alpha, float *__restrict__ dw,
                               float *__restrict__ dalpha)
{
    __shared__ float part[256];
    const int o = blockIdx.x, grp = blockIdx.y, tid = threadIdx.x;
    int lo, hi;
    group_rows(offsets, grp, rows, lo, hi);
    image += (size_t)grp * g.words_f;
    const float a = (float)alpha[(size_t)grp * g.alpha_stride + o];
    float sum = 0.0f;
    for (int i = tid; i < g.C_in; i += 256) {
        float acc = 0.0f;
        for (int t = lo; t < hi; ++t) acc += (float)dy[t * lddy + o] * row_value<T>(x, g.C_in, t, i);
        dw[((size_t)grp * g.C_out + o) * g.C_in + i] = acc * a;
        sum += weight_negative(image, g.kb_f, o, i) ? -acc : acc;
    }
    part[tid] = sum;
    __syncthreads();
    for (int n = 128; n; n >>= 1) {
        if (tid < n) part[tid] += part[tid + n];
        __syncthreads();
    }
    if (tid == 0 && dalpha) dalpha[(size_t)grp * g.C_out + o] = part[0];
}

}  // namespace

size_t linear_weight_grad_workspace_bytes(const LinearGeom &, int64_t) { return 256; }

int launch_linear_weight_grad(const LinearGeom &g, const RowsIn &x, const void *dy, int64_t lddy, int64_t rows, const int32_t *offsets,
                              const void *weights, float *dw, float *dalpha, void *, hipStream_t s)
{
    const char *w = (const char *)weights;
    const dim3 grid(g.C_out, g.G);
    if (g.dtype == SNN_DTYPE_BF16)
        linear_weight_grad_kernel<__bf16><<<grid, 256, 0, s>>>(g, x, (const __bf16 *)dy, lddy, (int)rows, offsets, (const uint32_t *)w,
                                                               (const __bf16 *)(w + g.at_alpha), dw, dalpha);
    else
        linear_weight_grad_kernel<_Float16><<<grid, 256, 0, s>>>(g, x, (const _Float16 *)dy, lddy, (int)rows, offsets, (const uint32_t *)w,
                                                                 (const _Float16 *)(w + g.at_alpha), dw, dalpha);
    return check_launch();
}

}  // namespace snn
