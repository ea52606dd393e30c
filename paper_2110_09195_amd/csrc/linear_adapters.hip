// Low-rank adapters beside a shared projection: their inner products and gradients.
#include "linear_device.h"

namespace snn {

namespace {

// low[t][r] = down[a][r] . x[t] and scaled[t][r] = scale[a] times it, a = the row's adapter; down [n][rank][C].
// Few rows: a wave takes NR inner products of a row, so that the adapters' matrices, of which nearly every row has its own, are read by many CUs.
// Bound by latency: 48 rows of rank 16, 4096 channels (6 MB) 3.4 us.
template <class T, int NR>
__global__ __launch_bounds__(256)
void low_few_kernel(int C, Adapters ad, const T *__restrict__ down, const T *__restrict__ x, int64_t ldx, float *__restrict__ low,
                    float *__restrict__ scaled)
{
    using v8 = typename Half<T>::v8;
    const int t = blockIdx.x, lane = threadIdx.x & 63, r = (blockIdx.y * 4 + (threadIdx.x >> 6)) * NR;
    if (r >= ad.rank) return;                                  // (rank is a multiple of NR)
    const int a = ad.of_row[t];
    float acc[NR] = {}, c = 0.0f;
    if (a >= 0 && a < ad.n) {
        c = ad.scale[a];
        const T *xr = x + t * ldx, *dr = down + ((int64_t)a * ad.rank + r) * C;
#pragma unroll(NR == 1 ? 4 : 2)
        for (int k = lane * 8; k < C; k += 512) {
            const v8 u = *(const v8 *)(xr + k);
#pragma unroll
            for (int j = 0; j < NR; ++j) {
                const v8 v = *(const v8 *)(dr + (int64_t)j * C + k);
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[j] = fmaf((float)u[i], (float)v[i], acc[j]);
            }
        }
#pragma unroll
        for (int d = 32; d; d >>= 1)
#pragma unroll
            for (int j = 0; j < NR; ++j) acc[j] += __shfl_xor(acc[j], d);
    }
    if (lane == 0) {
        const int64_t at = (int64_t)t * ad.rank + r;
#pragma unroll
        for (int j = 0; j < NR; ++j) {
            if (low) low[at + j] = acc[j];
            scaled[scaled_at(t, r + j, ad.rank)] = acc[j] * c;
        }
    }
}

// Many rows: 32 rows by 32 RB of the rank on the matrix cores, for each adapter of the 32 rows in turn.  The waves take the channels in
// turn (blocks of 64), rows and matrix both by way of LDS, a wave's own part of it, STAGES in flight without registers; then
// their sums are joined there.  A wave's blocks are consecutive ones: with the waves' blocks in turn every workgroup reads the same columns of all its
// rows at once, and rows a power of two apart lie in the same few channels of memory (8192 rows of rank 64, 4096 channels 33 us; 29 so).
// Bound by the rows' way from memory, of which a workgroup has 96 KB in flight: 64 MB, 13 us at a copy's rate, in 24 - 29.
template <class T, int RB, int STAGES>
__global__ __launch_bounds__(256)
void low_tile_kernel(int C, Adapters ad, const T *__restrict__ down, const T *__restrict__ x, int64_t ldx, int rows,
                     float *__restrict__ low, float *__restrict__ scaled)
{
    using H = Half<T>;
    using v8 = typename H::v8;
    constexpr int WAVES = 4, STAGE = 4096 * (1 + RB), LOADS = 4 * (1 + RB), PITCH = 32 * RB + 1;
    extern __shared__ __align__(16) char lds[];
    float *part = (float *)lds;                                // [WAVES][32][PITCH], when the loads are done
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, ln = lane & 31;
    const int t0 = blockIdx.x * 32, r0 = blockIdx.y * 32 * RB, here = min(rows - t0, 32), ranks = min(ad.rank - r0, 32 * RB);
    const int t = t0 + ln;
    const int id = t < rows ? ad.of_row[t] : -1;
    uint64_t left = __ballot(id >= 0 && id < ad.n);
    const int rr = tid >> 3, rc = (tid & 7) * 4 * RB, rid = __shfl(id, rr);      // what this thread joins and writes: 4 RB sums of a row
    float sum[4 * RB] = {};

    // a load: 8 rows of 128 bytes, 16-byte pieces xor-ed by half the row's number
    const int lr = lane >> 3, lp = (lane & 7) ^ (lr >> 1);
    char *mine = lds + wave * STAGES * STAGE;
    const uint32_t mine0 = __builtin_amdgcn_readfirstlane(lds_address(mine));
    const s32x4 rx = resource(x + (int64_t)t0 * ldx, (uint32_t)(here - 1) * (uint32_t)ldx * 2 + C * 2);
    uint32_t xo[4], piece[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) piece[s] = ln * 128 + (((2 * s + h) ^ ((ln >> 1) & 7)) << 4);
    const int blocks = (C + 63) / 64, each = (blocks + WAVES - 1) / WAVES, first = wave * each, last = min(first + each, blocks);
    while (left) {
        const int a = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
        const uint64_t own = __ballot(id == a);
        left &= ~own;
#pragma unroll
        for (int i = 0; i < 4; ++i) {                          // (rows 8 i + lr: their half's number ends in 4 i + lr / 2)
            const int r = 8 * i + lr;
            xo[i] = (own >> r) & 1 ? (uint32_t)r * (uint32_t)ldx * 2 + ((lp ^ ((4 * i) & 7)) << 4) : NOWHERE;
        }
        const s32x4 rd = resource(down + ((int64_t)a * ad.rank + r0) * C, (uint32_t)ranks * C * 2);
        auto issue = [&](int k, int slot) {
            const uint32_t at = __builtin_amdgcn_readfirstlane(mine0 + slot * STAGE);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = lp ^ ((4 * i) & 7);
                load_lds16(at + i * 1024, k * 64 + c * 8 < C ? xo[i] + k * 128 : NOWHERE, rx);
            }
#pragma unroll
            for (int i = 0; i < 4 * RB; ++i) {
                const int c = lp ^ ((4 * i) & 7), r = 8 * i + lr;
                load_lds16(at + 4096 + i * 1024, k * 64 + c * 8 < C && r < ranks ? (uint32_t)r * C * 2 + (c << 4) + k * 128 : NOWHERE, rd);
            }
        };
        f32x16 acc[RB] = {};
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s) issue(first + s, s);
        int slot = 0;
        for (int k = first; k < last; ++k) {
            issue(k + STAGES - 1, slot == 0 ? STAGES - 1 : slot - 1);
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS * (STAGES - 1)) : "memory");
            const char *at = mine + slot * STAGE;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const v8 v = *(const v8 *)(at + piece[s]);
#pragma unroll
                for (int i = 0; i < RB; ++i) acc[i] = H::mfma(*(const v8 *)(at + 4096 + i * 4096 + piece[s]), v, acc[i]);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            slot = slot == STAGES - 1 ? 0 : slot + 1;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
#pragma unroll
        for (int j = 0; j < RB; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) part[(wave * 32 + ln) * PITCH + j * 32 + 8 * (i >> 2) + 4 * h + (i & 3)] = acc[j][i];
        __syncthreads();
        if (rid == a) {
#pragma unroll
            for (int w = 0; w < WAVES; ++w)
#pragma unroll
                for (int i = 0; i < 4 * RB; ++i) sum[i] += part[(w * 32 + rr) * PITCH + rc + i];
        }
        __syncthreads();
    }
    if (rr >= here) return;
    const bool some = rid >= 0 && rid < ad.n;
    const float c = some ? ad.scale[rid] : 0.0f;
    const int64_t at = (int64_t)(t0 + rr) * ad.rank + r0 + rc;
#pragma unroll
    for (int i = 0; i < 4 * RB; i += 4) {
        if (rc + i >= ranks) break;
        const f32x4 v = {sum[i], sum[i + 1], sum[i + 2], sum[i + 3]};
        if (low) *(f32x4 *)(low + at + i) = v;
        const f32x4 z = some ? v * c : v;
        *(f32x4 *)(scaled + scaled_at(t0 + rr, r0 + rc + i, ad.rank)) = z;
    }
}

// What the backward call needs laid out otherwise, in one launch: A and B with their last two axes exchanged (tiles of 64 x 64), and the inputs
// from their 8-bit form.  Bound by memory, and in small calls by the launch.
struct KeptRows {
    const int8_t *q;
    const uint8_t *e;
    Walk walk;
    int C;
    void *x;                          // [rows][C]
};

struct Exchange {
    const uint16_t *in;
    uint16_t *out;
    int R, C, tiles_r, tiles_c;       // [n][R][C] -> [n][C][R]
};

__device__ inline void exchange_tile(const Exchange &e, int id, uint16_t (*s)[72])
{
    const int tid = threadIdx.x, per = e.tiles_r * e.tiles_c, n = id / per, r0 = id % per / e.tiles_c * 64, c0 = id % e.tiles_c * 64;
    const size_t base = (size_t)n * e.R * e.C;
#pragma unroll
    for (int i = 0; i < 2; ++i) {                              // (R and C are multiples of 8)
        const int k = i * 256 + tid, r = k >> 3, c = (k & 7) * 8;
        if (r0 + r < e.R && c0 + c < e.C) *(u32x4 *)&s[r][c] = *(const u32x4 *)(e.in + base + (size_t)(r0 + r) * e.C + c0 + c);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int k = i * 256 + tid, c = k >> 3, r = (k & 7) * 8;
        if (r0 + r >= e.R || c0 + c >= e.C) continue;
        u32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = s[r + 2 * j][c] | (uint32_t)s[r + 2 * j + 1][c] << 16;
        *(u32x4 *)(e.out + base + (size_t)(c0 + c) * e.R + r0 + r) = v;
    }
}

template <class T>
__global__ __launch_bounds__(256)
void adapters_lay_out_kernel(Exchange A, Exchange B, int tiles_a, int tiles_ab, KeptRows kept)
{
    __shared__ __align__(16) uint16_t s[64][72];
    const int id = blockIdx.x;
    if (id < tiles_a) exchange_tile(A, id, s);
    else if (id < tiles_ab) exchange_tile(B, id - tiles_a, s);
    else restore_rows(kept.q, kept.e, kept.walk, kept.C, (T *)kept.x, kept.C, id - tiles_ab);
}

// Up to so many products (rows x rank x channels) a wave takes four inner products of a row, and the matrices come from L2 again for every row: 512 rows,
// rank 16, 4096 channels 5.4 us against 13.3 by tiles; 1000 rows, rank 32, 2048 channels (62 M) 9.3 against 9.5; 1000 rows, rank 64, 4096 channels 29 against 22.
constexpr int64_t LOW_FEW_PRODUCTS = (int64_t)64 << 20;

template <class T, int RB, int STAGES>
int launch_low_tile(int C, const Adapters &ad, const T *down, const T *x, int64_t ldx, int64_t rows, float *low, float *scaled, hipStream_t s)
{
    constexpr size_t LDS = (size_t)4 * STAGES * 4096 * (1 + RB);
    static_assert(LDS >= 4 * 32 * (32 * RB + 1) * sizeof(float) && LDS <= 160 * 1024, "LDS");
    static LdsGrant grant;
    const auto kernel = low_tile_kernel<T, RB, STAGES>;
    const int rc = grant_dynamic_lds((const void *)kernel, LDS, grant);
    if (rc != SNN_OK) return rc;
    kernel<<<dim3((unsigned)((rows + 31) / 32), (ad.rank + 32 * RB - 1) / (32 * RB)), 256, LDS, s>>>(C, ad, down, x, ldx, (int)rows, low, scaled);
    return check_launch();
}

template <class T>
int launch_low(int C, const Adapters &ad, const void *down, const void *x, int64_t ldx, int64_t rows, float *low, float *scaled, hipStream_t s)
{
    if (rows <= 64) {
        low_few_kernel<T, 1><<<dim3((unsigned)rows, ad.rank / 4), 256, 0, s>>>(C, ad, (const T *)down, (const T *)x, ldx, low, scaled);
        return check_launch();
    }
    if (rows * ad.rank * C <= LOW_FEW_PRODUCTS) {
        low_few_kernel<T, 4><<<dim3((unsigned)rows, (ad.rank + 15) / 16), 256, 0, s>>>(C, ad, (const T *)down, (const T *)x, ldx, low, scaled);
        return check_launch();
    }
    if (ad.rank <= 32) return launch_low_tile<T, 1, 4>(C, ad, (const T *)down, (const T *)x, ldx, rows, low, scaled, s);
    return launch_low_tile<T, 2, 3>(C, ad, (const T *)down, (const T *)x, ldx, rows, low, scaled, s);
}

// Gradients of an adapter: the sum over its rows of x[t][c] low[t][r], for A (x the inputs, low = dlow) and B (x = dy, low as the forward
// call left it, times scale).  A workgroup takes one adapter, 256 channels and 32 RB of the rank, a
// wave 32 of the rank by as many channels as that leaves it.
//   - Rows come in chunks of 32.  Lanes look 64 chunks over at once for the adapter's rows, and the chunks that have some are gone through, the loads
//     of two of them in flight, without registers.  Rows of other adapters inside a chunk are not loaded: zeros in LDS.
//   - Bound by memory: 8192 rows of rank 64, 4096 -> 4096 (134 MB) 56 - 64 us (less where the inputs are still in the last cache) and 7 for the join; 27 at a copy's
//     rate.
//   - Both operands have the contracted axis across memory.  Rows are turned by the reads of their fragments; inner products are read as they
//     are (fp32, one of the rank a lane) and cut into values of the activations' type by the waves: three of bf16 (with two, that
//     is 16 bits, and cut once in memory, the call above took 44 - 47).  128-byte pieces of rows 8 .. 15 of sixteen are exchanged two by two, so
//     that both halves of a wave read different banks.
struct AdapterGradArgs {
    const void *x;
    int64_t ld;
    const float *low;                 // the inner products, by row [rows][rank] or (blocked) as scaled_at says
    bool blocked;
    int C;
    void *out;                        // A: [n][rank][C]; B: [n][C][rank], times scale
};

template <int RB>
struct AdapterGrad {
    static constexpr int CH = 256, WAVES = 4, STAGES = 3;
    static constexpr int X_BYTES = 32 * CH * 2, STAGE = X_BYTES + 32 * RB * 128;
    static constexpr size_t LDS = STAGES * STAGE;
    static_assert(LDS <= 80 * 1024, "two workgroups a CU");
};

template <class T, bool IS_B, int RB>
__device__ inline void adapters_grad_tile(const Adapters &ad, const AdapterGradArgs &g, int a, int c0, int r0, int rows, int chunk0, int chunks, float *part_out,
                                          uint32_t *flag, char *lds)
{
    using H = Half<T>;
    using v8 = typename H::v8;
    using S = AdapterGrad<RB>;
    constexpr int CH = S::CH, STAGES = S::STAGES, THREADS = 64 * S::WAVES, CB = CH / 32 * RB / S::WAVES;
    constexpr int PX = CH / 8, XL = 32 * PX / THREADS;                      // 16-byte pieces of a row, loads of a thread for a chunk
    constexpr int PL = RB;                                                  // loads for the inner products: 32 rows of 8 RB pieces
    constexpr int LOADS = XL + PL;
    static_assert(XL * THREADS == 32 * PX && THREADS == 32 * 8, "whole loads");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, ln = lane & 31;
    const int wr = wave % RB, wc = wave / RB;                               // 32 of the rank and CB blocks of channels a wave
    const uint32_t lds0 = lds_address(lds);

    uint32_t xo[XL], po[PL];
    int xr[XL], pr[PL];
#pragma unroll
    for (int i = 0; i < XL; ++i) {
        const int r = (i * THREADS + tid) / PX, c = tid % PX;
        xr[i] = r;
        xo[i] = (uint32_t)r * (uint32_t)(g.ld * 2) + ((((c >> 1) ^ ((r & 3) << 1)) << 1) | (c & 1)) * 16;
    }
#pragma unroll
    for (int i = 0; i < PL; ++i) {
        int piece = (i * THREADS + tid) / 8;                                // of 128 bytes: row piece / RB, 32 of the rank
        piece ^= (piece / RB >> 3) & 1;
        const int t = piece / RB, r = r0 + piece % RB * 32 + tid % 8 * 4;
        pr[i] = t;
        po[i] = r < ad.rank ? (uint32_t)(g.blocked ? r * 32 + t * 4 : t * ad.rank + r) * 4 : NOWHERE;
    }
    // (a chunk that is none: zeros)
    auto issue = [&](int chunk, uint32_t own, int slot) {
        const int64_t t = (int64_t)chunk * 32;
        const int left = min(rows - (int)t, 32);
        const uint32_t at = __builtin_amdgcn_readfirstlane(lds0 + slot * S::STAGE);
        const s32x4 rx = resource((const T *)g.x + t * g.ld + c0, (uint32_t)((left - 1) * (int)g.ld + g.C - c0) * 2);
        const s32x4 rp = resource(g.low + t * ad.rank, (uint32_t)((g.blocked ? 32 : left) * ad.rank) * 4);
#pragma unroll
        for (int i = 0; i < XL; ++i) load_lds16(at + i * THREADS * 16 + wave * 1024, (own >> xr[i]) & 1 ? xo[i] : NOWHERE, rx);
#pragma unroll
        for (int i = 0; i < PL; ++i) load_lds16(at + S::X_BYTES + i * THREADS * 16 + wave * 1024, (own >> pr[i]) & 1 ? po[i] : NOWHERE, rp);
    };

    f32x16 acc[CB] = {};
    float scale = Pieces<T>::SCALED ? power_of_two(126) : 1.0f;               // SCALED: a power of two that the wave's inner products and sums are times
    const int q = lane >> 4, rr = (lane & 15) >> 2;
    uint32_t xa[CB];                                           // this lane's place in a tile of rows
#pragma unroll
    for (int i = 0; i < CB; ++i) xa[i] = (8 * h + rr) * (CH * 2) + (((2 * (wc * CB + i) + (q & 1)) ^ (rr << 1)) * 32) + (lane & 3) * 8;

    const __amdgpu_buffer_rsrc_t r_ids = buffer(ad.of_row, (uint32_t)rows * 4);
    bool any = false;
    for (int base = chunk0; base < chunks; base += 64) {
        uint32_t match = 0;
        const int t = (base + lane) * 32;
        u32x4 ids[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) ids[i] = __builtin_amdgcn_raw_buffer_load_b128(r_ids, (uint32_t)(t + 4 * i) * 4, 0, 0);
#pragma unroll
        for (int i = 0; i < 32; ++i) match |= ((int)ids[i >> 2][i & 3] == a ? 1u : 0u) << i;
        if (t + 32 > rows) match &= t < rows ? (1u << (rows - t)) - 1 : 0u;
        if (base + lane >= chunks) match = 0;
        uint64_t some = __ballot(match != 0);                  // (the same in every wave)
        any |= some != 0;
        uint32_t own0 = 0, own1 = 0, own2 = 0;                 // this chunk's rows of the adapter, the next one's, and of the one after
        int chunk = base;
        auto next = [&]() {
            if (!some) return 0u;
            const int l = __builtin_ctzll(some);
            some &= some - 1;
            chunk = base + l;
            return (uint32_t)__builtin_amdgcn_readlane((int)match, l);
        };
        // (the look-over's loads are done, and the last chunks' fragments read: what is waited for below are loads of chunks)
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        own0 = next();
        issue(chunk, own0, 0);
        own1 = next();
        issue(chunk, own1, 1);
        int slot = 0;
        while (own0) {
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS) : "memory");
            own2 = next();
            issue(chunk, own2, slot == 0 ? STAGES - 1 : slot - 1);
            // While the products of 16 rows run, the next sixteen's inner products are cut, in their shadow.
            const char *at = lds + slot * S::STAGE;
            float v[2][8];
            v8 x[2][CB];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[s][e] = *(const float *)(at + S::X_BYTES + (((16 * s + 8 * h + e) * RB + wr) ^ h) * 128 + ln * 4);
#pragma unroll
                for (int i = 0; i < CB; ++i) x[s][i] = read_turned<T>(at + xa[i] + s * 16 * (CH * 2), 4 * (CH * 2));
            }
            if constexpr (Pieces<T>::SCALED) {
                float top = 0.0f;
#pragma unroll
                for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(v[e >> 3][e & 7]));
                if (__any(top * scale >= 32768.0f)) {
                    // larger ones than the scale is for: it goes down, and the sums so far with it
                    top = wave_top(top);
                    if (top == INFINITY) {                                   // (the others decide)
                        top = 0.0f;
#pragma unroll
                        for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(v[e >> 3][e & 7]) < INFINITY ? fabsf(v[e >> 3][e & 7]) : 0.0f);
                        top = wave_top(top);
                    }
                    const float next = fminf(power_of_two(piece_exponent(top)), scale);
                    const int down = (__float_as_int(next) - __float_as_int(scale)) >> 23;
#pragma unroll
                    for (int i = 0; i < CB; ++i)
#pragma unroll
                        for (int k = 0; k < 16; ++k) acc[i][k] = ldexpf(acc[i][k], down);
                    scale = next;
                }
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const Pieces<T> z = split8<T>(v[s], scale);
#pragma unroll
                for (int k = 0; k < Pieces<T>::N; ++k)
#pragma unroll
                    for (int i = 0; i < CB; ++i) acc[i] = IS_B ? H::mfma(x[s][i], z.of[k], acc[i]) : H::mfma(z.of[k], x[s][i], acc[i]);
            }
            own0 = own1;
            own1 = own2;
            slot = slot == STAGES - 1 ? 0 : slot + 1;
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (part_out) {
        if (tid == 0 && flag) *flag = any;
        if (!any) return;
    }
    // The lane's column is what is contiguous in the result: the channel of A, the rank of B.  Stores that lie outside are sent past the end.
    // (an adapter without rows has a gradient of zero, whatever its scale)
    const float factor = !any ? 0.0f : IS_B ? ad.scale[a] : 1.0f;
    const float up = power_of_two(127 - (int)(__float_as_uint(scale) >> 23));
    const uint32_t size = part_out ? 4 : 2, whole = (uint32_t)g.C * ad.rank;
    const __amdgpu_buffer_rsrc_t to = part_out ? buffer(part_out, whole * 4) : buffer((T *)g.out + (int64_t)a * whole, whole * 2);
#pragma unroll
    for (int i = 0; i < CB; ++i)
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const int row = 8 * m + 4 * h, c = c0 + (wc * CB + i) * 32 + (IS_B ? row : ln), r = r0 + wr * 32 + (IS_B ? ln : row);
            // (C and rank are multiples of 8: the four rows exist together)
            const uint32_t step = (uint32_t)(IS_B ? ad.rank : g.C) * size;
            const uint32_t at = c < g.C && r < ad.rank ? (IS_B ? (uint32_t)c * ad.rank + r : (uint32_t)r * g.C + c) * size : NOWHERE;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float v = Pieces<T>::SCALED ? acc[i][4 * m + k] * up : acc[i][4 * m + k];
                if (part_out) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), to, at + k * step, 0, 0);
                else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, (T)(v * factor)), to, at + k * step, 0, 0);
            }
        }
}

template <class T, int RB>
__global__ __launch_bounds__(256, 2)
void adapters_grad_kernel(Adapters ad, AdapterGradArgs A, AdapterGradArgs B, int rows, int tiles_a, int tiles, float *part, uint32_t *flags)
{
    extern __shared__ __align__(16) char lds[];
    const int a = blockIdx.x / tiles, tile = blockIdx.x % tiles, r0 = blockIdx.y * RB * 32;
    // part z of the rows, in whole chunks
    const int all = (rows + 31) / 32, each = (all + (int)gridDim.z - 1) / (int)gridDim.z, chunk0 = blockIdx.z * each, chunks = min(all, chunk0 + each);
    const int at = blockIdx.z * ad.n + a;
    if (part) part += (int64_t)at * ad.rank * (A.C + B.C);
    uint32_t *flag = part && tile == 0 && r0 == 0 ? flags + at : nullptr;
    if (tile < tiles_a) adapters_grad_tile<T, false, RB>(ad, A, a, tile * 256, r0, rows, chunk0, chunks, part, flag, lds);
    else adapters_grad_tile<T, true, RB>(ad, B, a, (tile - tiles_a) * 256, r0, rows, chunk0, chunks, part ? part + (int64_t)ad.rank * A.C : nullptr, flag, lds);
}

// The parts of the rows in their order, those that had some of the adapter's.
template <class T>
__global__ __launch_bounds__(256)
void adapters_join_kernel(Adapters ad, AdapterGradArgs A, AdapterGradArgs B, const float *__restrict__ part, const uint32_t *__restrict__ flags, int parts)
{
    const int64_t per = (int64_t)ad.rank * (A.C + B.C), in_a = (int64_t)ad.rank * A.C;
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    const int a = blockIdx.y;
    if (i >= per) return;
    f32x4 v = {0, 0, 0, 0};
    bool any = false;
    for (int s = 0; s < parts; ++s)
        if (flags[s * ad.n + a]) {
            v += *(const f32x4 *)(part + ((int64_t)s * ad.n + a) * per + i);
            any = true;
        }
    const bool is_b = i >= in_a;
    const float scale = !any ? 0.0f : is_b ? ad.scale[a] : 1.0f;
    typename Half<T>::v4 out;
#pragma unroll
    for (int k = 0; k < 4; ++k) out[k] = (T)(v[k] * scale);
    T *to = is_b ? (T *)B.out + (int64_t)a * ad.rank * B.C + (i - in_a) : (T *)A.out + (int64_t)a * in_a + i;
    *(typename Half<T>::v4 *)to = out;
}

template <class T, int RB>
int launch_adapters_grad(const Adapters &ad, const AdapterGradArgs &A, const AdapterGradArgs &B, int64_t rows, int parts, float *part, uint32_t *flags,
                         hipStream_t s)
{
    constexpr int CH = AdapterGrad<RB>::CH;
    constexpr size_t LDS = AdapterGrad<RB>::LDS;
    static LdsGrant grant;
    const auto kernel = adapters_grad_kernel<T, RB>;
    int rc = grant_dynamic_lds((const void *)kernel, LDS, grant);
    if (rc != SNN_OK) return rc;
    const int tiles_a = (A.C + CH - 1) / CH, tiles = tiles_a + (B.C + CH - 1) / CH;
    kernel<<<dim3((unsigned)tiles * ad.n, (ad.rank + RB * 32 - 1) / (RB * 32), parts), 256, LDS, s>>>(ad, A, B, (int)rows, tiles_a, tiles, parts > 1 ? part : nullptr, flags);
    rc = check_launch();
    if (rc != SNN_OK || parts == 1) return rc;
    adapters_join_kernel<T><<<dim3((unsigned)(((int64_t)ad.rank * (A.C + B.C) / 4 + 255) / 256), ad.n), 256, 0, s>>>(ad, A, B, part, flags, parts);
    return check_launch();
}

// Parts of the rows, joined by another launch: an adapter can have nearly all of them, and then its tiles alone would occupy a
// fraction of the CUs (the call of 8192 rows of one adapter of rank 64, 4096 -> 4096, 452 us whole, 344, 290, 270 and 269 in 2, 4, 8 and 16 parts).  Parts of
// at least 384 rows, while the workgroups (most of which find no rows of theirs, and end) stay few; of 96, and 75 an adapter, where
// there are not even as many of them as CUs (the call of 1274 rows of two adapters of rank 32, 1440 -> 608: two parts 39.9 us, eight 31.2; one
// of 400 rows of eight adapters, 2048 -> 2048, 34.3 whole and 37.1 in two).
int grad_parts(const LinearGeom &g, int n, int64_t rows)
{
    const int64_t tiles = (g.C_in + 255) / 256 + (g.C_out + 255) / 256;
    for (int parts = 1;; parts *= 2) {
        const int64_t of = rows / (2 * parts), workgroups = n * tiles * 2 * parts;
        const bool more = tiles * parts < 256 && ((of >= 384 && workgroups <= 4096) || (of >= 96 && of / n >= 75 && workgroups <= 256));
        if (parts == 16 || !more) return parts;
    }
}

// The backward call's workspace: scaled inner products; A and B with their last two axes exchanged; inputs in 8 bits as the values that they
// stand for.  (The forward call's: scaled inner products.)
struct Scratch {
    float *scaled;
    char *At, *Bt, *kept;
    float *part;                      // sums of parts of the rows, and which parts have some of an adapter's
    uint32_t *flags;
    int parts;
    size_t bytes;
};

size_t scaled_bytes(int64_t rows, int rank) { return align_up((size_t)((rows + 31) / 32) * 32 * rank * 4, 256); }

Scratch scratch(const LinearGeom &g, int n, int rank, int64_t rows, bool kept, void *ws)
{
    const int parts = grad_parts(g, n, rows);
    const size_t z = scaled_bytes(rows, rank), a = align_up((size_t)n * rank * g.C_in * 2, 256), b = align_up((size_t)n * rank * g.C_out * 2, 256);
    const size_t sums = parts > 1 ? align_up((size_t)parts * n * rank * (g.C_in + g.C_out) * 4, 256) : 0, flags = align_up((size_t)parts * n * 4, 256);
    const size_t x = kept ? align_up((size_t)rows * g.C_in * 2, 256) : 0;
    char *w = (char *)ws, *e = w + z + a + b;
    return {(float *)w, w + z, w + z + a, e + sums + flags, (float *)e, (uint32_t *)(e + sums), parts, z + a + b + sums + flags + x};
}

template <class T>
int forward(const LinearGeom &g, const Adapters &ad, const void *x, int64_t ldx, int64_t rows, const void *weights, void *y, int64_t ldy,
            float *low, float *scaled, hipStream_t s)
{
    if (adapters_in_one_launch(g, rows, ad.rank)) return launch_adapters_in_one(g, ad, x, ldx, rows, weights, y, ldy, low, s);
    const int rc = launch_low<T>(g.C_in, ad, ad.A, x, ldx, rows, low, scaled, s);
    if (rc != SNN_OK) return rc;
    return launch_linear_rows(g, false, x, ldx, rows, nullptr, weights, y, ldy, &ad, ad.B, scaled, s);
}

template <class T>
int backward(const LinearGeom &g, const Adapters &ad, const RowsIn &x, const float *low, const void *dy, int64_t lddy, int64_t rows,
             const void *weights, void *dx, int64_t lddx, void *dA, void *dB, const Scratch &w, hipStream_t s)
{
    if (rows) {
        const int rt = (ad.rank + 63) / 64, ct = (g.C_in + 63) / 64, ot = (g.C_out + 63) / 64;
        const Exchange A = {(const uint16_t *)ad.A, (uint16_t *)w.At, ad.rank, g.C_in, rt, ct};
        const Exchange B = {(const uint16_t *)ad.B, (uint16_t *)w.Bt, g.C_out, ad.rank, ot, rt};
        const int tiles_a = ad.n * rt * ct, tiles_ab = tiles_a + ad.n * rt * ot;
        // (the inputs as 16-bit values once, not bytes widened by every tile: see launch_linear_weight_grad)
        KeptRows kept = {};
        unsigned kept_blocks = 0;
        if (x.e) {
            kept = {(const int8_t *)x.p, x.e, {}, g.C_in, w.kept};
            kept_blocks = walk_of(rows, g.C_in, kept.walk);
        }
        adapters_lay_out_kernel<T><<<(unsigned)tiles_ab + kept_blocks, 256, 0, s>>>(A, B, tiles_a, tiles_ab, kept);
        int rc = check_launch();
        if (rc != SNN_OK) return rc;
        rc = launch_low<T>(g.C_out, ad, w.Bt, dy, lddy, rows, nullptr, w.scaled, s);
        if (rc != SNN_OK) return rc;
        rc = launch_linear_rows(g, true, dy, lddy, rows, nullptr, weights, dx, lddx, &ad, w.At, w.scaled, s);
        if (rc != SNN_OK) return rc;
    }
    AdapterGradArgs A = {x.p, x.ld, w.scaled, true, g.C_in, dA};
    const AdapterGradArgs B = {dy, lddy, low, false, g.C_out, dB};
    if (x.e) {
        A.x = w.kept;
        A.ld = g.C_in;
    }
    return ad.rank <= 32 ? launch_adapters_grad<T, 1>(ad, A, B, rows, w.parts, w.part, w.flags, s)
                         : launch_adapters_grad<T, 2>(ad, A, B, rows, w.parts, w.part, w.flags, s);
}

}  // namespace

size_t adapters_workspace_bytes(const LinearGeom &g, int n, int rank, int64_t rows, bool backward, bool kept)
{
    return backward ? scratch(g, n, rank, rows, kept, nullptr).bytes : scaled_bytes(rows, rank) + 256;
}

int launch_adapters_forward(const LinearGeom &g, const Adapters &ad, const void *x, int64_t ldx, int64_t rows, const void *weights,
                            void *y, int64_t ldy, float *low, void *ws, hipStream_t s)
{
    return g.dtype == SNN_DTYPE_BF16 ? forward<__bf16>(g, ad, x, ldx, rows, weights, y, ldy, low, (float *)ws, s)
                                     : forward<_Float16>(g, ad, x, ldx, rows, weights, y, ldy, low, (float *)ws, s);
}

int launch_adapters_backward(const LinearGeom &g, const Adapters &ad, const RowsIn &x, const float *low, const void *dy, int64_t lddy,
                             int64_t rows, const void *weights, void *dx, int64_t lddx, void *dA, void *dB, void *ws, hipStream_t s)
{
    const Scratch w = scratch(g, ad.n, ad.rank, rows, x.e != nullptr, ws);
    return g.dtype == SNN_DTYPE_BF16 ? backward<__bf16>(g, ad, x, low, dy, lddy, rows, weights, dx, lddx, dA, dB, w, s)
                                     : backward<_Float16>(g, ad, x, low, dy, lddy, rows, weights, dx, lddx, dA, dB, w, s);
}

}  // namespace snn
