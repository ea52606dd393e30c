// Low-rank adapters beside a shared projection: their inner products and gradients.
#include "linear_device.h"

namespace snn {

namespace {

template <class T>
__device__ inline float row_value(const RowsIn &x, int C, int64_t t, int c)
{
    if (!x.e) return (float)((const T *)x.p)[t * x.ld + c];
    return kept_value(((const int8_t *)x.p)[t * x.ld + c], unit_of(x.e[t * (4 * exponent_words(C)) + c / 32]));
}

// low[t][r] = down[a][r] . x[t] and scaled[t][r] = scale[a] times it, a = the row's adapter; down [n][rank][C].
// Few rows: a wave an inner product, so that the adapters' matrices, of which nearly every row has its own, are read by many CUs.
template <class T>
__global__ __launch_bounds__(256)
void low_few_kernel(int C, Adapters ad, const T *__restrict__ down, const T *__restrict__ x, int64_t ldx, float *__restrict__ low,
                    float *__restrict__ scaled)
{
    using v8 = typename Half<T>::v8;
    const int t = blockIdx.x, lane = threadIdx.x & 63, r = blockIdx.y * 4 + (threadIdx.x >> 6);
    const int a = ad.of_row[t];                                // (rank is a multiple of 4: every wave has an r)
    float acc = 0.0f, c = 0.0f;
    if (a >= 0 && a < ad.n) {
        c = ad.scale[a];
        const T *xr = x + t * ldx, *dr = down + ((int64_t)a * ad.rank + r) * C;
#pragma unroll 4
        for (int k = lane * 8; k < C; k += 512) {
            const v8 u = *(const v8 *)(xr + k), v = *(const v8 *)(dr + k);
#pragma unroll
            for (int i = 0; i < 8; ++i) acc = fmaf((float)u[i], (float)v[i], acc);
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) acc += __shfl_xor(acc, d);
    }
    if (lane == 0) {
        if (low) low[(int64_t)t * ad.rank + r] = acc;
        scaled[(int64_t)t * ad.rank + r] = acc * c;
    }
}

// Many rows: 32 rows by 32 of the rank on the matrix cores, for each adapter of the 32 rows in turn; the eight waves take the channels
// in turn and are joined in LDS.
template <class T>
__global__ __launch_bounds__(512)
void low_tile_kernel(int C, Adapters ad, const T *__restrict__ down, const T *__restrict__ x, int64_t ldx, int rows,
                     float *__restrict__ low, float *__restrict__ scaled)
{
    using H = Half<T>;
    using v8 = typename H::v8;
    constexpr int WAVES = 8;
    __shared__ float part[WAVES][32][33];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = lane >> 5, ln = lane & 31;
    const int t0 = blockIdx.x * 32, r0 = blockIdx.y * 32;
    const int t = t0 + ln;
    const int id = t < rows ? ad.of_row[t] : -1;
    const bool some = id >= 0 && id < ad.n;
    uint64_t left = __ballot(some);
    const int rr = tid >> 4, rc = r0 + (tid & 15) * 2;         // what this thread joins and writes
    const int rid = __shfl(id, rr & 31);
    const bool rsome = rid >= 0 && rid < ad.n;
    float v0 = 0.0f, v1 = 0.0f;
    const T *xr = x + (int64_t)min(t, rows - 1) * ldx + 8 * h;
    while (left) {
        const int a = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
        left &= ~__ballot(id == a);
        const T *dr = down + ((int64_t)a * ad.rank + min(r0 + ln, ad.rank - 1)) * C + 8 * h;
        f32x16 acc = {};
#pragma unroll 4
        for (int k = wave * 16; k < C; k += WAVES * 16) {
            u32x4 u = {0, 0, 0, 0}, v = {0, 0, 0, 0};
            if (k + 8 * h < C) {
                u = *(const u32x4 *)(dr + k);
                if (id == a) v = *(const u32x4 *)(xr + k);
            }
            acc = H::mfma(__builtin_bit_cast(v8, u), __builtin_bit_cast(v8, v), acc);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) part[wave][ln][8 * (i >> 2) + 4 * h + (i & 3)] = acc[i];
        __syncthreads();
        if (rid == a) {
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                v0 += part[w][rr][(tid & 15) * 2];
                v1 += part[w][rr][(tid & 15) * 2 + 1];
            }
        }
        __syncthreads();
    }
    if (t0 + rr >= rows || rc >= ad.rank) return;
    const float c = rsome ? ad.scale[rid] : 0.0f;
    const int64_t at = (int64_t)(t0 + rr) * ad.rank + rc;
    if (low) *(float2 *)(low + at) = make_float2(v0, v1);
    *(float2 *)(scaled + at) = rsome ? make_float2(v0 * c, v1 * c) : make_float2(0.0f, 0.0f);
}

// [n][R][C] -> [n][C][R], 16-bit values
__global__ __launch_bounds__(256)
void transpose_kernel(const uint16_t *__restrict__ in, uint16_t *__restrict__ out, int R, int C)
{
    __shared__ uint16_t s[64][66];
    const int tid = threadIdx.x, c0 = blockIdx.x * 64, r0 = blockIdx.y * 64;
    const size_t base = (size_t)blockIdx.z * R * C;
    for (int i = tid; i < 64 * 64; i += 256) {
        const int r = r0 + i / 64, c = c0 + i % 64;
        if (r < R && c < C) s[i / 64][i % 64] = in[base + (size_t)r * C + c];
    }
    __syncthreads();
    for (int i = tid; i < 64 * 64; i += 256) {
        const int c = c0 + i / 64, r = r0 + i % 64;
        if (r < R && c < C) out[base + (size_t)c * R + r] = s[i % 64][i / 64];
    }
}

template <class T>
int launch_low(int C, const Adapters &ad, const void *down, const void *x, int64_t ldx, int64_t rows, float *low, float *scaled, hipStream_t s)
{
    if (rows <= 64)
        low_few_kernel<T><<<dim3((unsigned)rows, ad.rank / 4), 256, 0, s>>>(C, ad, (const T *)down, (const T *)x, ldx, low, scaled);
    else
        low_tile_kernel<T><<<dim3((unsigned)((rows + 31) / 32), (ad.rank + 31) / 32), 512, 0, s>>>(C, ad, (const T *)down, (const T *)x, ldx,
                                                                                                 (int)rows, low, scaled);
    return check_launch();
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

// the workspace: scaled inner products, A and B with their last two axes exchanged
struct Scratch {
    float *scaled;
    void *At, *Bt;
    size_t bytes;
};

Scratch scratch(const LinearGeom &g, int n, int rank, int64_t rows, void *ws)
{
    const size_t a = align_up((size_t)rows * rank * 4, 256), b = align_up((size_t)n * rank * g.C_in * 2, 256);
    char *w = (char *)ws;
    return {(float *)w, w + a, w + a + b, a + b + align_up((size_t)n * rank * g.C_out * 2, 256)};
}

template <class T>
int forward(const LinearGeom &g, const Adapters &ad, const void *x, int64_t ldx, int64_t rows, const void *weights, void *y, int64_t ldy,
            float *low, const Scratch &w, hipStream_t s)
{
    const int rc = launch_low<T>(g.C_in, ad, ad.A, x, ldx, rows, low, w.scaled, s);
    if (rc != SNN_OK) return rc;
    return launch_linear_rows(g, false, x, ldx, rows, nullptr, weights, y, ldy, &ad, ad.B, w.scaled, s);
}

template <class T>
int backward(const LinearGeom &g, const Adapters &ad, const RowsIn &x, const float *low, const void *dy, int64_t lddy, int64_t rows,
             const void *weights, void *dx, int64_t lddx, void *dA, void *dB, const Scratch &w, hipStream_t s)
{
    if (rows) {
        transpose_kernel<<<dim3((g.C_in + 63) / 64, (ad.rank + 63) / 64, ad.n), 256, 0, s>>>((const uint16_t *)ad.A, (uint16_t *)w.At, ad.rank, g.C_in);
        transpose_kernel<<<dim3((ad.rank + 63) / 64, (g.C_out + 63) / 64, ad.n), 256, 0, s>>>((const uint16_t *)ad.B, (uint16_t *)w.Bt, g.C_out, ad.rank);
        int rc = launch_low<T>(g.C_out, ad, w.Bt, dy, lddy, rows, nullptr, w.scaled, s);
        if (rc != SNN_OK) return rc;
        rc = launch_linear_rows(g, true, dy, lddy, rows, nullptr, weights, dx, lddx, &ad, w.At, w.scaled, s);
        if (rc != SNN_OK) return rc;
    }
    adapters_grad_kernel<T, false><<<dim3((g.C_in + 255) / 256, ad.rank, ad.n), 256, 0, s>>>(g.C_in, ad, x, w.scaled, (int)rows, (T *)dA);
    adapters_grad_kernel<T, true><<<dim3((g.C_out + 255) / 256, ad.rank, ad.n), 256, 0, s>>>(g.C_out, ad, RowsIn{dy, nullptr, lddy}, low, (int)rows, (T *)dB);
    return check_launch();
}

}  // namespace

size_t adapters_workspace_bytes(const LinearGeom &g, int n, int rank, int64_t rows) { return scratch(g, n, rank, rows, nullptr).bytes; }

int launch_adapters_forward(const LinearGeom &g, const Adapters &ad, const void *x, int64_t ldx, int64_t rows, const void *weights,
                            void *y, int64_t ldy, float *low, void *ws, hipStream_t s)
{
    const Scratch w = scratch(g, ad.n, ad.rank, rows, ws);
    return g.dtype == SNN_DTYPE_BF16 ? forward<__bf16>(g, ad, x, ldx, rows, weights, y, ldy, low, w, s)
                                     : forward<_Float16>(g, ad, x, ldx, rows, weights, y, ldy, low, w, s);
}

int launch_adapters_backward(const LinearGeom &g, const Adapters &ad, const RowsIn &x, const float *low, const void *dy, int64_t lddy,
                             int64_t rows, const void *weights, void *dx, int64_t lddx, void *dA, void *dB, void *ws, hipStream_t s)
{
    const Scratch w = scratch(g, ad.n, ad.rank, rows, ws);
    return g.dtype == SNN_DTYPE_BF16 ? backward<__bf16>(g, ad, x, low, dy, lddy, rows, weights, dx, lddx, dA, dB, w, s)
                                     : backward<_Float16>(g, ad, x, low, dy, lddy, rows, weights, dx, lddx, dA, dB, w, s);
}

}  // namespace snn
