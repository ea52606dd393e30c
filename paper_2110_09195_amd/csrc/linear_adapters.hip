// Low-rank adapters beside a shared projection: their inner products and gradients.
#include "linear.h"

namespace snn {

namespace {

template <class T>
__device__ inline float row_value(const RowsIn &x, int C, int64_t t, int c)
{
    if (!x.e) return (float)((const T *)x.p)[t * x.ld + c];
    return kept_value(((const int8_t *)x.p)[t * x.ld + c], unit_of(x.e[t * ((C + 31) / 32) + c / 32]));
}

// low[t][r] = A[a][r] . x[t], and scaled[t][r] = scale[a] times it;  BACK: scaled[t][r] = scale[a] B[a][:, r] . dy[t]
template <class T, bool BACK>
__global__ __launch_bounds__(128)
void adapters_low_kernel(int C, Adapters ad, const T *__restrict__ x, int64_t ldx, float *__restrict__ low, float *__restrict__ scaled)
{
    const int t = blockIdx.x, r = threadIdx.x;
    if (r >= ad.rank) return;
    const int a = ad.of_row[t];
    float acc = 0.0f, c = 0.0f;
    if (a >= 0 && a < ad.n) {
        c = ad.scale[a];
        for (int k = 0; k < C; ++k)
            acc += (float)x[t * ldx + k] * (BACK ? (float)((const T *)ad.B)[((size_t)a * C + k) * ad.rank + r]
                                                 : (float)((const T *)ad.A)[((size_t)a * ad.rank + r) * C + k]);
    }
    if (low) low[(size_t)t * ad.rank + r] = acc;
    scaled[(size_t)t * ad.rank + r] = acc * c;
}

// dA[a][r][i] = sum of dlow[t][r] x[t][i];  IS_B: dB[a][o][r] = scale[a] * sum of low[t][r] dy[t][o]
template <class T, bool IS_B>
__global__ __launch_bounds__(256)
void adapters_grad_kernel(int C, Adapters ad, RowsIn x, const float *__restrict__ low, int rows, T *__restrict__ out)
{
    const int c = blockIdx.x * 256 + threadIdx.x, r = blockIdx.y, a = blockIdx.z;
    if (c >= C) return;
    float acc = 0.0f;
    for (int t = 0; t < rows; ++t)
        if (ad.of_row[t] == a) acc += low[(size_t)t * ad.rank + r] * row_value<T>(x, C, t, c);
    if (IS_B) out[((size_t)a * C + c) * ad.rank + r] = (T)(acc * ad.scale[a]);
    else out[((size_t)a * ad.rank + r) * C + c] = (T)acc;
}

template <class T>
int backward(const LinearGeom &g, const Adapters &ad, const RowsIn &x, const float *low, const void *dy, int64_t lddy, int64_t rows,
             const void *weights, void *dx, int64_t lddx, void *dA, void *dB, float *dlow, hipStream_t s)
{
    if (rows) {
        adapters_low_kernel<T, true><<<(unsigned)rows, 128, 0, s>>>(g.C_out, ad, (const T *)dy, lddy, nullptr, dlow);
        const int rc = launch_linear_rows(g, true, dy, lddy, rows, nullptr, weights, dx, lddx, &ad, dlow, s);
        if (rc != SNN_OK) return rc;
    }
    adapters_grad_kernel<T, false><<<dim3((g.C_in + 255) / 256, ad.rank, ad.n), 256, 0, s>>>(g.C_in, ad, x, dlow, (int)rows, (T *)dA);
    adapters_grad_kernel<T, true><<<dim3((g.C_out + 255) / 256, ad.rank, ad.n), 256, 0, s>>>(g.C_out, ad, RowsIn{dy, nullptr, lddy}, low, (int)rows, (T *)dB);
    return check_launch();
}

}  // namespace

size_t adapters_workspace_bytes(const LinearGeom &, int rank, int64_t rows) { return align_up((size_t)rows * rank * 4 + 256, 256); }

int launch_adapters_forward(const LinearGeom &g, const Adapters &ad, const void *x, int64_t ldx, int64_t rows, const void *weights,
                            void *y, int64_t ldy, float *low, void *ws, hipStream_t s)
{
    float *scaled = (float *)ws;
    if (g.dtype == SNN_DTYPE_BF16)
        adapters_low_kernel<__bf16, false><<<(unsigned)rows, 128, 0, s>>>(g.C_in, ad, (const __bf16 *)x, ldx, low, scaled);
    else
        adapters_low_kernel<_Float16, false><<<(unsigned)rows, 128, 0, s>>>(g.C_in, ad, (const _Float16 *)x, ldx, low, scaled);
    return launch_linear_rows(g, false, x, ldx, rows, nullptr, weights, y, ldy, &ad, scaled, s);
}

int launch_adapters_backward(const LinearGeom &g, const Adapters &ad, const RowsIn &x, const float *low, const void *dy, int64_t lddy,
                             int64_t rows, const void *weights, void *dx, int64_t lddx, void *dA, void *dB, void *ws, hipStream_t s)
{
    return g.dtype == SNN_DTYPE_BF16
               ? backward<__bf16>(g, ad, x, low, dy, lddy, rows, weights, dx, lddx, dA, dB, (float *)ws, s)
               : backward<_Float16>(g, ad, x, low, dy, lddy, rows, weights, dx, lddx, dA, dB, (float *)ws, s);
}

}  // namespace snn
