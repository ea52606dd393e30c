// Rows through sub-bit weights: outputs and the gradient of the inputs (see linear.h for the bits' layout).
#include "linear.h"

namespace snn {

namespace {

// The member bits of a block of 64 output channels by 64 vectors (512 input channels), turned into the words of both images.
constexpr int PREP_O = 64, PREP_V = 64, PREP_THREADS = 256;

__global__ __launch_bounds__(PREP_THREADS)
void linear_prepare_kernel(LinearGeom g, const uint16_t *__restrict__ codebook, const uint16_t *__restrict__ idx,
                           const uint16_t *__restrict__ alpha, uint32_t *__restrict__ image_f, uint32_t *__restrict__ image_d,
                           uint16_t *__restrict__ alpha_out)
{
    __shared__ uint8_t code[PREP_O][PREP_V + 4];       // inverted: bit 7 - j set where element j is -1
    __shared__ uint8_t member[256];
    const int tid = threadIdx.x, grp = blockIdx.z;
    const int ob = blockIdx.y, o0 = ob * PREP_O, v0 = blockIdx.x * PREP_V;
    const int V = g.C_in / 8;
    codebook += (size_t)grp * g.K;
    idx += (size_t)grp * g.C_out * V;
    if (tid < g.K) member[tid] = (uint8_t)~codebook[tid];
    __syncthreads();
    for (int i = tid; i < PREP_O * PREP_V; i += PREP_THREADS) {
        const int o = i / PREP_V, v = i % PREP_V;
        uint8_t c = 0;
        if (o0 + o < g.C_out && v0 + v < V) c = member[min((int)idx[(size_t)(o0 + o) * V + v0 + v], g.K - 1)];
        code[o][v] = c;
    }
    __syncthreads();
    // F: 2 blocks of 32 outputs x 8 blocks of 64 inputs
    image_f += (size_t)grp * g.words_f;
    for (int i = tid; i < 2 * 8 * 64; i += PREP_THREADS) {
        const int l = i & 63, kbl = (i >> 6) & 7, nbl = i >> 9, h = l >> 5;
        const int nb = 2 * ob + nbl, kb = v0 / 8 + kbl;
        if (nb >= g.nb_f || kb >= g.kb_f) continue;
        uint32_t w = 0;
        for (int s = 0; s < 4; ++s) {
            const uint32_t c = code[nbl * 32 + (l & 31)][kbl * 8 + 2 * s + h];
            for (int r = 0; r < 4; ++r)
                w |= ((c >> (7 - 2 * r)) & 1u) << (15 - 4 * s - r) | ((c >> (6 - 2 * r)) & 1u) << (31 - 4 * s - r);
        }
        image_f[((size_t)nb * g.kb_f + kb) * 64 + l] = w;
    }
    // D: 16 blocks of 32 inputs x this block of 64 outputs
    image_d += (size_t)grp * g.words_d;
    for (int i = tid; i < 16 * 64; i += PREP_THREADS) {
        const int l = i & 63, nbl = i >> 6, h = l >> 5;
        const int nb = v0 / 4 + nbl;
        if (nb >= g.nb_d) continue;
        const int v = nbl * 4 + ((l & 31) >> 3), bit = 7 - (l & 7);
        uint32_t w = 0;
        for (int s = 0; s < 4; ++s)
            for (int r = 0; r < 4; ++r) {
                const int o = 16 * s + 8 * h + 2 * r;
                w |= (((uint32_t)code[o][v] >> bit) & 1u) << (15 - 4 * s - r) | (((uint32_t)code[o + 1][v] >> bit) & 1u) << (31 - 4 * s - r);
            }
        image_d[((size_t)nb * g.kb_d + ob) * 64 + l] = w;
    }
    if (blockIdx.x == 0 && tid < PREP_O)
        alpha_out[(size_t)grp * g.alpha_stride + o0 + tid] = o0 + tid < g.C_out ? alpha[(size_t)grp * g.C_out + o0 + tid] : (uint16_t)0;
}

// One thread an output: the definition.
template <class T, bool GRAD>
__global__ __launch_bounds__(256)
void linear_rows_kernel(LinearGeom g, const T *__restrict__ in, int64_t ld_in, int rows, const int32_t *__restrict__ offsets,
                        const uint32_t *__restrict__ image, const T *__restrict__ alpha, T *__restrict__ out, int64_t ld_out,
                        Adapters ad, const float *__restrict__ low)
{
    const int N = GRAD ? g.C_in : g.C_out, K = GRAD ? g.C_out : g.C_in, kbs = GRAD ? g.kb_d : g.kb_f;
    const int n = blockIdx.x * 256 + threadIdx.x, t = blockIdx.y + blockIdx.z * 32768;
    if (n >= N || t >= rows) return;
    int grp = -1;
    for (int i = 0; i < g.G && grp < 0; ++i) {
        int lo, hi;
        group_rows(offsets, i, rows, lo, hi);
        if (t >= lo && t < hi) grp = i;
    }
    if (grp < 0) return;
    image += (size_t)grp * (GRAD ? g.words_d : g.words_f);
    alpha += (size_t)grp * g.alpha_stride;
    const T *x = in + t * ld_in;
    float acc = 0.0f;
    for (int k = 0; k < K; ++k) {
        const float v = GRAD ? (float)x[k] * (float)alpha[k] : (float)x[k];
        acc += weight_negative(image, kbs, n, k) ? -v : v;
    }
    if (!GRAD) acc *= (float)alpha[n];
    if (ad.of_row) {
        const int a = ad.of_row[t];
        if (a >= 0 && a < ad.n)
            for (int r = 0; r < ad.rank; ++r) {
                const float w = GRAD ? (float)((const T *)ad.A)[((size_t)a * ad.rank + r) * g.C_in + n]
                                     : (float)((const T *)ad.B)[((size_t)a * g.C_out + n) * ad.rank + r];
                acc += low[(size_t)t * ad.rank + r] * w;
            }
    }
    out[t * ld_out + n] = (T)acc;
}

}  // namespace

int launch_linear_prepare(const LinearGeom &g, const uint16_t *codebook, const uint16_t *idx, const void *alpha, void *weights, hipStream_t s)
{
    const dim3 grid((g.C_in / 8 + PREP_V - 1) / PREP_V, (g.C_out + PREP_O - 1) / PREP_O, g.G);
    char *w = (char *)weights;
    linear_prepare_kernel<<<grid, PREP_THREADS, 0, s>>>(g, codebook, idx, (const uint16_t *)alpha, (uint32_t *)w,
                                                        (uint32_t *)(w + g.at_d), (uint16_t *)(w + g.at_alpha));
    return check_launch();
}

template <class T>
static int rows_simple(const LinearGeom &g, bool grad, const void *in, int64_t ld_in, int64_t rows, const int32_t *offsets,
                       const char *w, void *out, int64_t ld_out, const Adapters &ad, const float *low, hipStream_t s)
{
    const int N = grad ? g.C_in : g.C_out;
    const dim3 grid((N + 255) / 256, rows < 32768 ? rows : 32768, (rows + 32767) / 32768);
    if (grad)
        linear_rows_kernel<T, true><<<grid, 256, 0, s>>>(g, (const T *)in, ld_in, (int)rows, offsets, (const uint32_t *)(w + g.at_d),
                                                         (const T *)(w + g.at_alpha), (T *)out, ld_out, ad, low);
    else
        linear_rows_kernel<T, false><<<grid, 256, 0, s>>>(g, (const T *)in, ld_in, (int)rows, offsets, (const uint32_t *)w,
                                                          (const T *)(w + g.at_alpha), (T *)out, ld_out, ad, low);
    return check_launch();
}

int launch_linear_rows(const LinearGeom &g, bool grad, const void *in, int64_t ld_in, int64_t rows, const int32_t *offsets,
                       const void *weights, void *out, int64_t ld_out, const Adapters *ad, const float *low, hipStream_t s)
{
    const Adapters a = ad ? *ad : Adapters{};
    return g.dtype == SNN_DTYPE_BF16 ? rows_simple<__bf16>(g, grad, in, ld_in, rows, offsets, (const char *)weights, out, ld_out, a, low, s)
                                     : rows_simple<_Float16>(g, grad, in, ld_in, rows, offsets, (const char *)weights, out, ld_out, a, low, s);
}

}  // namespace snn
