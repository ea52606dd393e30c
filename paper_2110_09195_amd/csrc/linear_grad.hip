// Gradients of the weights of projections, from activations or from their 8-bit form: G = dy^T x over the rows of a group.
#include "linear_device.h"

namespace snn {

namespace {

struct GradArgs {
    RowsIn x;
    const void *dy;
    int64_t lddy;
    int rows, groups;
    const int32_t *offsets;
    const uint32_t *image;            // F, of group 0
    uint32_t words;
    int nbs, kbs;
    const void *alpha;
    uint32_t alpha_stride;
    int C_in, C_out;
    int ti, to, splits;               // tiles of inputs and outputs of a group, parts of its rows
    float *dw;                        // splits = 1: the result
    float *part;                      // else [split][group][C_out][C_in], not yet scaled
    float *alpha_part;                // [split][tile of inputs][group][C_out], or nullptr
};

// A tile of BI inputs x BO outputs of a group's gradient, D[i][o] on the matrix cores, over 32 rows at a time.
//   - Both operands have the contracted axis (rows) across memory.  Their tiles go to LDS as they lie, without registers, STAGES in
//     flight, and are turned by the reads that fetch fragments.  32-byte pieces of a row are xor-ed with the row's low two bits, so that the four rows
//     that such a read touches lie in different banks.
//   - KEPT: inputs come as bytes; the thread that loaded 16 of them widens them for everyone, a step ahead of their use: once an element
//     instead of once a fragment.
template <class T, bool KEPT, int BI, int BO, int WI, int WO, int STAGES>
__global__ __launch_bounds__(64 * (BI / WI) * (BO / WO))
void linear_weight_grad_kernel(GradArgs p)
{
    using H = Half<T>;
    using v8 = typename H::v8;
    constexpr int WAVES_I = BI / WI, WAVES = WAVES_I * (BO / WO), THREADS = 64 * WAVES;
    constexpr int IB = WI / 32, OB = WO / 32;
    constexpr int PX = KEPT ? BI / 16 : BI / 8, PD = BO / 8;   // 16-byte pieces of a row
    constexpr int XL = 32 * PX / THREADS, DL = 32 * PD / THREADS;
    static_assert(XL * THREADS == 32 * PX && DL * THREADS == 32 * PD, "whole loads");
    constexpr int X_BYTES = 32 * PX * 16, D_BYTES = 32 * PD * 16, E_BYTES = KEPT ? WAVES * 256 : 0;
    constexpr int STAGE = X_BYTES + D_BYTES + E_BYTES;
    constexpr int WIDE = 32 * BI * 2;                          // KEPT: the widened tile, two of them behind the stages
    constexpr int LOADS = XL + DL + (KEPT ? 1 : 0);
    extern __shared__ __align__(16) char lds[];

    // XCDs (workgroups in turn) take a share of every group's tiles
    const int per_group = p.ti * p.to * p.splits, share = (per_group + 7) / 8;
    const int turn = blockIdx.x >> 3, grp = turn / share, id = (blockIdx.x & 7) * share + turn % share;
    if (id >= per_group) return;
    const int split = id / (p.ti * p.to), tile = id % (p.ti * p.to);
    const int it = tile % p.ti, i0 = it * BI, o0 = tile / p.ti * BO;
    int lo, hi;
    group_rows(p.offsets, grp, p.rows, lo, hi);
    if (p.splits > 1) {
        const int run = ((hi - lo + p.splits - 1) / p.splits + 31) & ~31;
        lo = (int)min((int64_t)hi, lo + (int64_t)split * run);
        hi = min(hi, lo + run);
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
    const int steps = (hi - lo + 31) / 32;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = wave % WAVES_I, wo = wave / WAVES_I;
    const uint32_t lds0 = lds_address(lds);
    const int x_size = KEPT ? 1 : 2, ew = 4 * exponent_words(p.C_in);
    uint32_t xo[XL], dof[DL], eo = NOWHERE;
#pragma unroll
    for (int i = 0; i < XL; ++i) {
        const int r = (i * THREADS + tid) / PX, c = tid % PX;
        xo[i] = (uint32_t)r * (uint32_t)(p.x.ld * x_size) + (KEPT ? c * 16 : ((((c >> 1) ^ ((r & 3) << 1)) << 1) | (c & 1)) * 16);
    }
#pragma unroll
    for (int i = 0; i < DL; ++i) {
        const int r = (i * THREADS + tid) / PD, c = tid % PD;
        dof[i] = (uint32_t)r * (uint32_t)(p.lddy * 2) + ((((c >> 1) ^ ((r & 3) << 1)) << 1) | (c & 1)) * 16;
    }
    if constexpr (KEPT) {
        constexpr int EW = BI / 128;                           // words of a row's exponents in this tile
        if (lane < 32 * EW) eo = (uint32_t)(lane / EW) * ew + (lane % EW) * 4;
    }
    auto issue = [&](int step, int slot) {
        const int t = lo + step * 32, left = min(hi - t, 32);
        const uint32_t at = __builtin_amdgcn_readfirstlane(lds0 + slot * STAGE);
        const int64_t t64 = left > 0 ? t : 0;
        const s32x4 rx = resource((const char *)p.x.p + (t64 * p.x.ld + i0) * x_size, left > 0 ? (uint32_t)(((left - 1) * p.x.ld + p.C_in - i0) * x_size) : 0);
        const s32x4 rd = resource((const char *)p.dy + (t64 * p.lddy + o0) * 2, left > 0 ? (uint32_t)(((left - 1) * p.lddy + p.C_out - o0) * 2) : 0);
#pragma unroll
        for (int i = 0; i < XL; ++i) load_lds16(at + i * THREADS * 16 + wave * 1024, xo[i], rx);
#pragma unroll
        for (int i = 0; i < DL; ++i) load_lds16(at + X_BYTES + i * THREADS * 16 + wave * 1024, dof[i], rd);
        if constexpr (KEPT) {
            const s32x4 re = resource(p.x.e + t64 * ew + i0 / 32, left > 0 ? (uint32_t)((left - 1) * ew + ew - i0 / 32) : 0);
            load_lds4(at + X_BYTES + D_BYTES + wave * 256, eo, re);
        }
    };
    // the thread's own pieces of a stage, widened
    auto widen = [&](int slot, int wide) {
        if constexpr (KEPT) {
            const char *at = lds + slot * STAGE;
#pragma unroll
            for (int i = 0; i < XL; ++i) {
                const int r = (i * THREADS + tid) / PX, c = tid % PX;
                const u32x4 raw = *(const u32x4 *)(at + (i * THREADS + tid) * 16);
                const uint32_t e = *(const uint8_t *)(at + X_BYTES + D_BYTES + wave * 256 + r * (BI / 32) + (c >> 1));
                v8 v[2];
                widen16<T>(raw, unit_of(e), v);
                char *to = lds + STAGES * STAGE + wide * WIDE + r * (BI * 2) + (c ^ ((r & 3) << 1)) * 32;
                *(v8 *)to = v[0];
                *(v8 *)(to + 16) = v[1];
            }
        }
    };

    f32x16 acc[IB][OB] = {};
    const int q = lane >> 4, rr = (lane & 15) >> 2, h = lane >> 5, ln = lane & 31;
    uint32_t xa[IB], da[OB];                                   // this lane's place in fragment 0 of a tile
#pragma unroll
    for (int i = 0; i < IB; ++i) xa[i] = (8 * h + rr) * (BI * 2) + (((2 * (wi * IB + i) + (q & 1)) ^ (rr << 1)) * 32) + (lane & 3) * 8;
#pragma unroll
    for (int i = 0; i < OB; ++i) da[i] = (8 * h + rr) * (BO * 2) + (((2 * (wo * OB + i) + (q & 1)) ^ (rr << 1)) * 32) + (lane & 3) * 8;

    for (int s = 0; s < STAGES - 1; ++s) issue(s, s);
    if constexpr (KEPT) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS * (STAGES - 2)) : "memory");
        widen(0, 0);
    }
    int slot = 0;
    for (int k = 0; k < steps; ++k) {
        // This step's tiles have landed (KEPT: and the next one's bytes, for the thread that loaded them), and everyone is done with
        // what is written next.
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS * (KEPT ? STAGES - 3 : STAGES - 2)) : "memory");
        issue(k + STAGES - 1, slot == 0 ? STAGES - 1 : slot - 1);
        const char *xt = KEPT ? lds + STAGES * STAGE + (k & 1) * WIDE : lds + slot * STAGE, *dt = lds + slot * STAGE + X_BYTES;
        slot = slot == STAGES - 1 ? 0 : slot + 1;
        widen(slot, (k + 1) & 1);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            v8 x[IB], d[OB];
#pragma unroll
            for (int i = 0; i < IB; ++i) x[i] = read_turned<T>(xt + xa[i] + s * 16 * (BI * 2), 4 * (BI * 2));
#pragma unroll
            for (int i = 0; i < OB; ++i) d[i] = read_turned<T>(dt + da[i] + s * 16 * (BO * 2), 4 * (BO * 2));
#pragma unroll
            for (int i = 0; i < IB; ++i)
#pragma unroll
                for (int j = 0; j < OB; ++j) acc[i][j] = H::mfma(x[i], d[j], acc[i][j]);
        }
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");

    // Lane: output ln of a block of 32, inputs 8 g + 4 h + i of register 4 g + i.
    const T *alpha = (const T *)p.alpha + (size_t)grp * p.alpha_stride;
    if (p.alpha_part) {
        float *sums = (float *)lds;                            // [WAVES_I][BO]
        const uint32_t *image = p.image + (size_t)grp * p.words;
#pragma unroll
        for (int j = 0; j < OB; ++j) {
            const int nb = o0 / 32 + wo * OB + j;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < IB; ++i) {
                const int ib = i0 + wi * WI + i * 32, kb = ib >> 6;
                uint32_t word[2] = {0, 0};
                if (nb < p.nbs && kb < p.kbs) {
                    const uint32_t *w = image + ((size_t)nb * p.kbs + kb) * 64 + ln;
                    word[0] = w[0];
                    word[1] = w[32];
                }
                // input 8 g + 4 h + k of the block: step (ib / 32 % 2) 2 + g / 2 of the half g % 2, element 4 h + k
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const uint32_t w = word[g & 1] << (4 * (((ib >> 5) & 1) * 2 + (g >> 1)) + 2 * h);
                    const uint32_t sign[4] = {w << 16, w, w << 17, w << 1};
                    if (ib + 8 * g < p.C_in) {
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            sum += __uint_as_float(__float_as_uint(acc[i][j][4 * g + k]) ^ (sign[k] & 0x80000000u));
                    }
                }
            }
            sum += __shfl_xor(sum, 32);
            if (h == 0) sums[wi * BO + (wo * OB + j) * 32 + ln] = sum;
        }
        __syncthreads();
        for (int o = tid; o < BO; o += THREADS) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < WAVES_I; ++i) sum += sums[i * BO + o];
            if (o0 + o < p.C_out) p.alpha_part[(((size_t)split * p.ti + it) * p.groups + grp) * p.C_out + o0 + o] = sum;
        }
        __syncthreads();
    }
    float *out = p.splits > 1 ? p.part + (size_t)split * p.groups * p.C_out * p.C_in : p.dw;
    out += (size_t)grp * p.C_out * p.C_in;
    constexpr int PITCH = WI * 4 + 16;
    char *mine = lds + wave * 32 * PITCH;
#pragma unroll
    for (int j = 0; j < OB; ++j) {
        const int o = o0 + (wo * OB + j) * 32;
        const float a = p.splits > 1 ? 1.0f : (float)alpha[min(o + ln, p.C_out - 1)];
#pragma unroll
        for (int i = 0; i < IB; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4 v;
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = acc[i][j][4 * g + k] * a;
                *(f32x4 *)(mine + ln * PITCH + (i * 32 + 8 * g + 4 * h) * 4) = v;
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        constexpr int PIECES = WI / 4;
#pragma unroll
        for (int i = 0; i < PIECES / 2; ++i) {
            const int n = i * 64 + lane, r = n / PIECES, c = i0 + wi * WI + n % PIECES * 4;
            const f32x4 v = *(const f32x4 *)(mine + r * PITCH + n % PIECES * 16);
            if (o + r < p.C_out && c < p.C_in) *(f32x4 *)(out + (size_t)(o + r) * p.C_in + c) = v;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

// The parts of a sum in their order: workgroups of `dw` first (splits > 1), then those of dalpha.
template <class T>
__global__ __launch_bounds__(256)
void linear_grad_join_kernel(GradArgs p, float *__restrict__ dw, float *__restrict__ dalpha, unsigned dw_blocks)
{
    const int64_t n = (int64_t)p.groups * p.C_out * p.C_in;
    if (blockIdx.x < dw_blocks) {
        for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n; i += (int64_t)dw_blocks * 1024) {
            f32x4 v = *(const f32x4 *)(p.part + i);
            for (int s = 1; s < p.splits; ++s) v += *(const f32x4 *)(p.part + s * n + i);
            const int64_t row = i / p.C_in;
            const int grp = (int)(row / p.C_out);
            *(f32x4 *)(dw + i) = v * (float)((const T *)p.alpha)[(size_t)grp * p.alpha_stride + (row - (int64_t)grp * p.C_out)];
        }
        return;
    }
    const int i = (int)(blockIdx.x - dw_blocks) * 256 + threadIdx.x, m = p.groups * p.C_out;
    if (i >= m) return;
    float sum = 0.0f;
    for (int s = 0; s < p.splits * p.ti; ++s) sum += p.alpha_part[(size_t)s * m + i];
    dalpha[i] = sum;
}

// Tiles and parts of a call.  Tiles of 256 x 256 where they fill the chip; else of 128 x 128, and where these do not either and
// groups are long, their rows in up to eight parts, which a second launch joins.
struct GradPlan {
    bool large;
    int ti, to, splits;
    size_t alpha_floats, part_floats;
};

GradPlan grad_plan(const LinearGeom &g, int64_t rows)
{
    GradPlan p;
    const int64_t large = (int64_t)g.G * ((g.C_in + 255) / 256) * ((g.C_out + 255) / 256);
    p.large = large >= 200;
    const int B = p.large ? 256 : 128;
    p.ti = (g.C_in + B - 1) / B;
    p.to = (g.C_out + B - 1) / B;
    const int64_t tiles = (int64_t)g.G * p.ti * p.to, each = rows / g.G;
    p.splits = 1;
    while (p.splits < 8 && tiles * p.splits < 384 && each / (2 * p.splits) >= 256) p.splits *= 2;
    p.alpha_floats = (size_t)p.splits * p.ti * g.G * g.C_out;
    p.part_floats = p.splits > 1 ? (size_t)p.splits * g.G * g.C_out * g.C_in : 0;
    return p;
}

template <class T, bool KEPT, int B, int WI, int WO>
int launch_grad(const GradArgs &p, hipStream_t s)
{
    constexpr int WAVES = (B / WI) * (B / WO), STAGES = 4;
    constexpr size_t TILES = KEPT ? STAGES * (32 * B + 32 * B * 2 + WAVES * 256) + 2 * 32 * B * 2 : STAGES * (32 * B * 2 * 2);
    constexpr size_t OUT = (size_t)WAVES * 32 * (WI * 4 + 16), LDS = TILES > OUT ? TILES : OUT;
    static_assert(LDS <= 160 * 1024, "LDS");
    static LdsGrant grant;
    const auto kernel = linear_weight_grad_kernel<T, KEPT, B, B, WI, WO, STAGES>;
    const int rc = grant_dynamic_lds((const void *)kernel, LDS, grant);
    if (rc != SNN_OK) return rc;
    const int64_t grid = (int64_t)((p.ti * p.to * p.splits + 7) / 8) * 8 * p.groups;
    if (grid >= ((int64_t)1 << 31)) return SNN_ERR_UNSUPPORTED;
    kernel<<<dim3((unsigned)grid), 64 * WAVES, LDS, s>>>(p);
    return check_launch();
}

template <class T>
int launch_typed(const GradArgs &p, bool large, float *dalpha, hipStream_t s)
{
    int rc;
    if (large) rc = p.x.e ? launch_grad<T, true, 256, 128, 64>(p, s) : launch_grad<T, false, 256, 128, 64>(p, s);
    else rc = p.x.e ? launch_grad<T, true, 128, 64, 64>(p, s) : launch_grad<T, false, 128, 64, 64>(p, s);
    if (rc != SNN_OK || (p.splits == 1 && !dalpha)) return rc;
    const int64_t pieces = (int64_t)p.groups * p.C_out * p.C_in / 4, blocks = (pieces + 255) / 256;
    const unsigned dw_blocks = p.splits > 1 ? (unsigned)(blocks < 4096 ? blocks : 4096) : 0;
    const unsigned alpha_blocks = dalpha ? (unsigned)((p.groups * p.C_out + 255) / 256) : 0;
    linear_grad_join_kernel<T><<<dw_blocks + alpha_blocks, 256, 0, s>>>(p, p.dw, dalpha, dw_blocks);
    return check_launch();
}

}  // namespace

size_t linear_weight_grad_workspace_bytes(const LinearGeom &g, int64_t rows)
{
    const GradPlan p = grad_plan(g, rows);
    return align_up(p.alpha_floats * 4, 256) + p.part_floats * 4;
}

int launch_linear_weight_grad(const LinearGeom &g, const RowsIn &x, const void *dy, int64_t lddy, int64_t rows, const int32_t *offsets,
                              const void *weights, float *dw, float *dalpha, void *ws, hipStream_t s)
{
    const GradPlan plan = grad_plan(g, rows);
    const char *w = (const char *)weights;
    GradArgs p = {};
    p.x = x; p.dy = dy; p.lddy = lddy; p.rows = (int)rows; p.groups = g.G; p.offsets = offsets;
    p.image = (const uint32_t *)w; p.words = g.words_f; p.nbs = g.nb_f; p.kbs = g.kb_f;
    p.alpha = w + g.at_alpha; p.alpha_stride = g.alpha_stride;
    p.C_in = g.C_in; p.C_out = g.C_out;
    p.ti = plan.ti; p.to = plan.to; p.splits = plan.splits;
    p.dw = dw;
    p.alpha_part = dalpha ? (float *)ws : nullptr;
    p.part = (float *)((char *)ws + align_up(plan.alpha_floats * 4, 256));
    return g.dtype == SNN_DTYPE_BF16 ? launch_typed<__bf16>(p, plan.large, dalpha, s) : launch_typed<_Float16>(p, plan.large, dalpha, s);
}

}  // namespace snn
