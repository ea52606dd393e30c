// Low-rank adapters beside a shared projection: their inner products and gradients.
#include "linear_device.h"

namespace snn {

namespace {

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

// Gradients of an adapter: D[c][r] = sum over its rows of x[t][c] low[t][r], for A (x the inputs, low = dlow) and B (x = dy, low as the
// forward call left it, times scale).  A workgroup takes one adapter and CH channels and the whole rank.
//   - Rows come in chunks of 32.  Lanes look 64 chunks over at once for the adapter's rows, and the waves take the chunks that
//     have some in turn, each with its own double buffer in LDS, filled without registers; no wave waits for another until the sums are joined.
//   - Rows of other adapters inside a chunk are not loaded (zeros in LDS, and zeros for their inner products).
//   - The inner products are held in two values of the activations' type.
struct AdapterGradArgs {
    RowsIn x;
    const float *low;
    int C;
    void *out;
    bool is_b;                        // out [C][rank] times scale, else [rank][C]
};

template <int CH, int RB, int W>
struct AdapterGrad {
    static constexpr int WAVES = W, X_BYTES = 32 * CH * 2, STAGE = X_BYTES + 32 * RB * 32 * 4 + 256;
    static constexpr int JOIN = WAVES * 32 * 33 * 4;
    static constexpr size_t LDS = (size_t)WAVES * 2 * STAGE > JOIN ? (size_t)WAVES * 2 * STAGE : JOIN;
};

template <class T, bool KEPT, int CH, int RB, int WAVES>
__device__ inline void adapters_grad_tile(const Adapters &ad, const AdapterGradArgs &g, int a, int c0, int r0, int rows, char *lds)
{
    using H = Half<T>;
    using v8 = typename H::v8;
    using S = AdapterGrad<CH, RB, WAVES>;
    constexpr int CB = CH / 32;
    constexpr int PX = KEPT ? CH / 16 : CH / 8, XL = 32 * PX / 64;     // pieces of a row, loads of a lane for a chunk
    constexpr int LL = RB * 4;                                         // loads of a lane for the inner products of a chunk
    constexpr int LOADS = XL + LL + (KEPT ? 1 : 0);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, ln = lane & 31;
    const int x_size = KEPT ? 1 : 2, ew = 4 * exponent_words(g.C);
    // rows of 64 channels are half of the banks wide: what keeps rows 0 .. 3 apart is their second bit
    const auto turn = [](int r) { return CH >= 128 ? (r & 3) << 1 : (r & 2); };
    char *mine = lds + wave * 2 * S::STAGE;
    const uint32_t mine0 = lds_address(mine);

    uint32_t xo[XL];
    int xrow[XL];
#pragma unroll
    for (int i = 0; i < XL; ++i) {
        const int r = (i * 64 + lane) / PX, c = lane % PX;
        xrow[i] = r;
        xo[i] = (uint32_t)r * (uint32_t)(g.x.ld * x_size) + (KEPT ? c * 16 : ((((c >> 1) ^ turn(r)) << 1) | (c & 1)) * 16);
    }
    auto issue = [&](int chunk, uint32_t own, int slot) {
        const int64_t t = (int64_t)chunk * 32;
        const int left = min(rows - (int)t, 32);
        const uint32_t at = __builtin_amdgcn_readfirstlane(mine0 + slot * S::STAGE);
        const s32x4 rx = resource((const char *)g.x.p + (t * g.x.ld + c0) * x_size, (uint32_t)(((left - 1) * g.x.ld + g.C - c0) * x_size));
        const s32x4 rl = resource(g.low + t * ad.rank + r0, (uint32_t)(left * ad.rank - r0) * 4);
#pragma unroll
        for (int i = 0; i < XL; ++i) load_lds16(at + i * 1024, (own >> xrow[i]) & 1 ? xo[i] : NOWHERE, rx);
        // inner products: rows of RB * 32 in LDS
#pragma unroll
        for (int i = 0; i < LL; ++i) {
            const int r = (i * 64 + lane) / (RB * 8), c = lane % (RB * 8) * 4;
            load_lds16(at + S::X_BYTES + i * 1024, ((own >> r) & 1) && r0 + c < ad.rank ? (uint32_t)(r * ad.rank + c) * 4 : NOWHERE, rl);
        }
        if constexpr (KEPT) {
            constexpr int EW = CH >= 128 ? CH / 128 : 1;
            const s32x4 re = resource(g.x.e + t * ew + c0 / 128 * 4, (uint32_t)((left - 1) * ew + ew - c0 / 128 * 4));
            load_lds4(at + S::X_BYTES + 32 * RB * 32 * 4, lane < 32 * EW ? (uint32_t)(lane / EW) * ew + lane % EW * 4 : NOWHERE, re);
        }
    };

    f32x16 acc[CB][RB] = {};
    const int q = lane >> 4, rr = (lane & 15) >> 2;
    uint32_t xa[CB];
#pragma unroll
    for (int i = 0; i < CB; ++i) xa[i] = (8 * h + rr) * (CH * 2) + (((2 * i + (q & 1)) ^ turn(rr)) * 32) + (lane & 3) * 8;

    auto compute = [&](uint32_t own, int slot) {
        char *at = mine + slot * S::STAGE;
        if constexpr (KEPT) {
            // a lane's own pieces, widened in place: all of them are read before the first is written
            u32x4 raw[XL];
            float u[XL];
#pragma unroll
            for (int i = 0; i < XL; ++i) {
                constexpr int EB = CH >= 128 ? CH / 32 : 4;
                raw[i] = *(const u32x4 *)(at + (i * 64 + lane) * 16);
                u[i] = unit_of(*(const uint8_t *)(at + S::X_BYTES + 32 * RB * 32 * 4 + xrow[i] * EB + ((c0 & 127) >> 5) + (lane % PX >> 1)));
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
            for (int i = 0; i < XL; ++i) {
                v8 v[2];
                widen16<T>(raw[i], (own >> xrow[i]) & 1 ? u[i] : 0.0f, v);
                char *to = at + xrow[i] * (CH * 2) + ((lane % PX) ^ turn(xrow[i])) * 32;
                *(v8 *)to = v[0];
                *(v8 *)(to + 16) = v[1];
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            v8 x[CB];
#pragma unroll
            for (int i = 0; i < CB; ++i) x[i] = read_turned<T>(at + xa[i] + s * 16 * (CH * 2), 4 * (CH * 2));
#pragma unroll
            for (int j = 0; j < RB; ++j) {
                float z[8];
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    z[k] = *(const float *)(at + S::X_BYTES + ((16 * s + 8 * h + k) * (RB * 32) + j * 32 + ln) * 4);
                v8 hi, lo;
                split8<T>(z, hi, lo);
#pragma unroll
                for (int i = 0; i < CB; ++i) {
                    acc[i][j] = H::mfma(x[i], hi, acc[i][j]);
                    acc[i][j] = H::mfma(x[i], lo, acc[i][j]);
                }
            }
        }
    };

    const int chunks = (rows + 31) / 32;
    for (int base = 0; base < chunks; base += 64) {
        uint32_t match = 0;
        const int t = (base + lane) * 32;
        if (base + lane < chunks)
            for (int i = 0; i < 32 && t + i < rows; ++i) match |= (ad.of_row[t + i] == a ? 1u : 0u) << i;
        uint64_t some = __ballot(match != 0);
        // every WAVES-th of the chunks that have rows of this adapter, from the wave's own on
        int skip = wave;
        auto next = [&](int &chunk, uint32_t &own) {
            while (some && skip) {
                some &= some - 1;
                --skip;
            }
            if (!some) return false;
            const int l = __builtin_ctzll(some);
            some &= some - 1;
            skip = WAVES - 1;
            chunk = base + l;
            own = (uint32_t)__builtin_amdgcn_readlane((int)match, l);
            return true;
        };
        int chunk, slot = 0;
        uint32_t own, own2;
        // (the look-over's loads are done: what is waited for below are the chunk's)
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        bool more = next(chunk, own);
        if (more) issue(chunk, own, 0);
        while (more) {
            const bool more2 = next(chunk, own2);
            if (more2) {
                issue(chunk, own2, slot ^ 1);
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");
            } else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            compute(own, slot);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            own = own2;
            slot ^= 1;
            more = more2;
        }
    }

    // the waves' sums, 32 x 32 at a time, in their order
    const float scale = g.is_b ? ad.scale[a] : 1.0f;
    float(*part)[32][33] = (float(*)[32][33])lds;
#pragma unroll
    for (int i = 0; i < CB; ++i)
#pragma unroll
        for (int j = 0; j < RB; ++j) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 16; ++k) part[wave][ln][8 * (k >> 2) + 4 * h + (k & 3)] = acc[i][j][k];     // [r][c]
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 16 / WAVES; ++k) {
                const int m = k * 64 * WAVES + tid, r = g.is_b ? m & 31 : m >> 5, c = g.is_b ? m >> 5 : m & 31;
                float v = 0.0f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) v += part[w][r][c];
                const int cc = c0 + i * 32 + c, rank = r0 + j * 32 + r;
                if (cc < g.C && rank < ad.rank) {
                    const int64_t at = g.is_b ? ((int64_t)a * g.C + cc) * ad.rank + rank : ((int64_t)a * ad.rank + rank) * g.C + cc;
                    // (an adapter without rows has a gradient of zero, whatever its scale)
                    ((T *)g.out)[at] = (T)(v == 0.0f ? 0.0f : v * scale);
                }
            }
        }
}

template <class T, bool KEPT, int CH, int RB, int WAVES>
__global__ __launch_bounds__(64 * WAVES)
void adapters_grad_kernel(Adapters ad, AdapterGradArgs A, AdapterGradArgs B, int rows, int tiles_a, int tiles)
{
    extern __shared__ __align__(16) char lds[];
    const int a = blockIdx.x / tiles, tile = blockIdx.x % tiles, r0 = blockIdx.y * RB * 32;
    if (tile < tiles_a) adapters_grad_tile<T, KEPT, CH, RB, WAVES>(ad, A, a, tile * CH, r0, rows, lds);
    else adapters_grad_tile<T, false, CH, RB, WAVES>(ad, B, a, (tile - tiles_a) * CH, r0, rows, lds);
}

template <class T, bool KEPT, int CH, int RB, int WAVES>
int launch_adapters_grad(const Adapters &ad, const AdapterGradArgs &A, const AdapterGradArgs &B, int64_t rows, hipStream_t s)
{
    constexpr size_t LDS = AdapterGrad<CH, RB, WAVES>::LDS;
    static_assert(LDS <= 160 * 1024, "LDS");
    static LdsGrant grant;
    const auto kernel = adapters_grad_kernel<T, KEPT, CH, RB, WAVES>;
    const int rc = grant_dynamic_lds((const void *)kernel, LDS, grant);
    if (rc != SNN_OK) return rc;
    const int tiles_a = (A.C + CH - 1) / CH, tiles = tiles_a + (B.C + CH - 1) / CH;
    kernel<<<dim3((unsigned)tiles * ad.n, (ad.rank + RB * 32 - 1) / (RB * 32)), 64 * WAVES, LDS, s>>>(ad, A, B, (int)rows, tiles_a, tiles);
    return check_launch();
}

template <class T, bool KEPT>
int launch_adapters_grad(const Adapters &ad, const AdapterGradArgs &A, const AdapterGradArgs &B, int64_t rows, hipStream_t s)
{
    if (ad.rank <= 32) return launch_adapters_grad<T, KEPT, 64, 1, 8>(ad, A, B, rows, s);
    return launch_adapters_grad<T, KEPT, 64, 2, 4>(ad, A, B, rows, s);
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
    const AdapterGradArgs A = {x, w.scaled, g.C_in, dA, false}, B = {{dy, nullptr, lddy}, low, g.C_out, dB, true};
    return x.e ? launch_adapters_grad<T, true>(ad, A, B, rows, s) : launch_adapters_grad<T, false>(ad, A, B, rows, s);
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
