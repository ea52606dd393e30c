// Gradients of the weights of projections: G = dy^T x over the rows of a group.
#include "linear_device.h"

#include <climits>

namespace snn {

namespace {

struct GradArgs {
    const void *x, *dy;
    int64_t ldx, lddy;
    int rows, groups;
    const int32_t *offsets;
    const uint32_t *image;            // F, of group 0
    uint32_t words;
    int kbs;
    const void *alpha;
    uint32_t alpha_stride;
    int C_in, C_out;
    int ti, to, splits;               // tiles of inputs and outputs of a group, parts of its rows
    int share, xcds_i, share_i;       // an XCD's tiles of all parts: a block, share_i along the inputs, of xcds_i XCDs side by side there; or (share_i = 0) a row
    float *dw;                        // splits = 1: the result
    float *part;                      // else [split][group][C_out][C_in], not yet scaled
    float *alpha_part;                // [split][tile of inputs][group][C_out], or nullptr
};

// A tile of BI inputs x BO outputs of a group's gradient, D[i][o] on the matrix cores, over 32 rows at a time.  Both operands have the contracted
// axis (rows) across memory.  Their tiles go to LDS as they lie, without registers, STAGES in flight, and are turned by the reads that fetch
// fragments.  32-byte pieces of a row are xor-ed with the row's low two bits, so that the four rows that such a read touches lie in
// different banks.  alpha's gradient comes from the same sums, with the signs of the tile's own bits.
// Bound: the matrix pipes at the clock that the chip's power leaves them (16384 rows 4096 -> 4096 400 - 426 us by card, 1.29 -
// 1.37 PFLOP/s), and for each tile the 256 KB that it writes, with nothing else on the CU (8 groups of as many rows, 512 MB of results: 500 - 546 us).  Tiles of 128 x 256
// two on a CU, which do not hide it either, take 585; groups in another order on each XCD 554, and 8192 rows 2048 -> 2048 107 for 91.
template <class T, int BI, int BO, int WI, int WO, int STAGES>
__global__ __launch_bounds__(64 * (BI / WI) * (BO / WO))
void linear_weight_grad_kernel(GradArgs p)
{
    using H = Half<T>;
    using v8 = typename H::v8;
    constexpr int WAVES_I = BI / WI, WAVES = WAVES_I * (BO / WO), THREADS = 64 * WAVES;
    constexpr int IB = WI / 32, OB = WO / 32;
    constexpr int PX = BI / 8, PD = BO / 8;                    // 16-byte pieces of a row
    constexpr int XL = 32 * PX / THREADS, DL = 32 * PD / THREADS;
    static_assert(XL * THREADS == 32 * PX && DL * THREADS == 32 * PD, "whole loads");
    constexpr int X_BYTES = 32 * PX * 16, STAGE = X_BYTES + 32 * PD * 16, LOADS = XL + DL;
    extern __shared__ __align__(16) char lds[];

    // XCDs (workgroups in turn) take a share of every group's tiles
    const int turn = blockIdx.x >> 3, xcd = blockIdx.x & 7, grp = turn / p.share, id = turn % p.share;
    int split, it, ot;
    if (p.share_i) {
        const int block = p.share / p.splits, tile = id % block;
        split = id / block;
        it = xcd % p.xcds_i * p.share_i + tile % p.share_i;
        ot = xcd / p.xcds_i * (block / p.share_i) + tile / p.share_i;
    } else {
        const int all = xcd * p.share + id, tile = all % (p.ti * p.to);
        split = all / (p.ti * p.to);
        it = tile % p.ti;
        ot = tile / p.ti;
    }
    if (split >= p.splits || it >= p.ti || ot >= p.to) return;
    const int i0 = it * BI, o0 = ot * BO;
    int lo, hi;
    group_rows(p.offsets, grp, p.rows, lo, hi);
    const bool some = hi > lo;
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
    uint32_t xo[XL], dof[DL];
#pragma unroll
    for (int i = 0; i < XL; ++i) {
        const int r = (i * THREADS + tid) / PX, c = tid % PX;
        xo[i] = (uint32_t)r * (uint32_t)(p.ldx * 2) + ((((c >> 1) ^ ((r & 3) << 1)) << 1) | (c & 1)) * 16;
    }
#pragma unroll
    for (int i = 0; i < DL; ++i) {
        const int r = (i * THREADS + tid) / PD, c = tid % PD;
        dof[i] = (uint32_t)r * (uint32_t)(p.lddy * 2) + ((((c >> 1) ^ ((r & 3) << 1)) << 1) | (c & 1)) * 16;
    }
    // Half of a step's loads: inputs, gradients of outputs.  Steps are issued in order; resources end with the group's last row (a
    // row's end is past by a tile's columns that do not exist: what they hold is not used).
    const int x_row = (int)p.ldx * 2, d_row = (int)p.lddy * 2;
    const char *x_at = (const char *)p.x + ((int64_t)lo * p.ldx + i0) * 2, *d_at = (const char *)p.dy + ((int64_t)lo * p.lddy + o0) * 2;
    const int x_gap = x_row - (p.C_in - i0) * 2, d_gap = d_row - (p.C_out - o0) * 2;
    int x_left = hi - lo, d_left = hi - lo;
    auto issue = [&](int slot, int part) {
        const uint32_t at = __builtin_amdgcn_readfirstlane(lds0 + slot * STAGE);
        if (part == 0) {
            const s32x4 rx = resource(x_at, (uint32_t)max(min(max(x_left, 0), 32) * x_row - x_gap, 0));
#pragma unroll
            for (int i = 0; i < XL; ++i) load_lds16(at + i * THREADS * 16 + wave * 1024, xo[i], rx);
            x_at += 32 * x_row;
            x_left -= 32;
        } else {
            const s32x4 rd = resource(d_at, (uint32_t)max(min(max(d_left, 0), 32) * d_row - d_gap, 0));
#pragma unroll
            for (int i = 0; i < DL; ++i) load_lds16(at + X_BYTES + i * THREADS * 16 + wave * 1024, dof[i], rd);
            d_at += 32 * d_row;
            d_left -= 32;
        }
    };

    f32x16 acc[IB][OB] = {};
    const int q = lane >> 4, rr = (lane & 15) >> 2, h = lane >> 5, ln = lane & 31;
    uint32_t xa[IB], da[OB];                                   // this lane's place in fragment 0 of a tile
#pragma unroll
    for (int i = 0; i < IB; ++i) xa[i] = (8 * h + rr) * (BI * 2) + (((2 * (wi * IB + i) + (q & 1)) ^ (rr << 1)) * 32) + (lane & 3) * 8;
#pragma unroll
    for (int i = 0; i < OB; ++i) da[i] = (8 * h + rr) * (BO * 2) + (((2 * (wo * OB + i) + (q & 1)) ^ (rr << 1)) * 32) + (lane & 3) * 8;

    // While the products of 16 rows run, the fragments of the next 16 are read, in the shadow of the matrix instructions.
    v8 x[2][IB], d[2][OB];
    auto read = [&](const char *at, int s, int to) {
#pragma unroll
        for (int i = 0; i < IB; ++i) x[to][i] = read_turned<T>(at + xa[i] + s * 16 * (BI * 2), 4 * (BI * 2));
#pragma unroll
        for (int i = 0; i < OB; ++i) d[to][i] = read_turned<T>(at + X_BYTES + da[i] + s * 16 * (BO * 2), 4 * (BO * 2));
    };
    auto multiply = [&](int from) {
#pragma unroll
        for (int i = 0; i < IB; ++i)
#pragma unroll
            for (int j = 0; j < OB; ++j) acc[i][j] = H::mfma(x[from][i], d[from][j], acc[i][j]);
#pragma unroll
        for (int i = 0; i < IB * OB; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                // a matrix instruction
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);                // LDS reads
            __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);                // VALU
        }
    };
    for (int s = 0; s < STAGES - 1; ++s)
        for (int q = 0; q < 2; ++q) issue(s, q);
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(LOADS * (STAGES - 2)) : "memory");
    read(lds, 0, 0);
    int slot = 0;
    for (int k = 0; k < steps; ++k) {
        // the next step's tiles have landed, and everyone is done with what is loaded next
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS * (STAGES - 3)) : "memory");
        const char *at = lds + slot * STAGE;
        const int free = slot == 0 ? STAGES - 1 : slot - 1;
        slot = slot == STAGES - 1 ? 0 : slot + 1;
        issue(free, 0);
        read(at, 1, 1);
        multiply(0);
        issue(free, 1);
        read(lds + slot * STAGE, 0, 0);
        multiply(1);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");

    // Lane: output ln of a block of 32, inputs 8 g + 4 h + i of register 4 g + i.
    const T *alpha = (const T *)p.alpha + (size_t)grp * p.alpha_stride;
    if (p.alpha_part) {
        float *sums = (float *)lds;                            // [WAVES_I][BO]
        // (blocks past the image's end give zeros; no channel of theirs counts)
        const __amdgpu_buffer_rsrc_t image = buffer(p.image + (size_t)grp * p.words, p.words * 4);
        uint32_t word[OB][IB][2];
#pragma unroll
        for (int j = 0; j < OB; ++j)
#pragma unroll
            for (int i = 0; i < IB; ++i)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t block = (uint32_t)(o0 / 32 + wo * OB + j) * p.kbs + ((i0 + wi * WI + i * 32) >> 6);
                    word[j][i][k] = __builtin_amdgcn_raw_buffer_load_b32(image, (block * 64 + k * 32 + ln) * 4, 0, 0);
                }
#pragma unroll
        for (int j = 0; j < OB; ++j) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < IB; ++i) {
                const int ib = i0 + wi * WI + i * 32;
                // input 8 g + 4 h + k of the block: step (ib / 32 % 2) 2 + g / 2 of the half g % 2, element 4 h + k
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const uint32_t w = word[j][i][g & 1] << (4 * (((ib >> 5) & 1) * 2 + (g >> 1)) + 2 * h);
                    const uint32_t sign[4] = {w << 16, w, w << 17, w << 1};
                    const bool in = ib + 8 * g < p.C_in;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        sum += in ? __uint_as_float(__float_as_uint(acc[i][j][4 * g + k]) ^ (sign[k] & 0x80000000u)) : 0.0f;
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
        // (a group without rows has a gradient of zero, whatever its scales)
        const float a = p.splits > 1 ? 1.0f : some ? (float)alpha[min(o + ln, p.C_out - 1)] : 0.0f;
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
            if (o + r < p.C_out && c < p.C_in) {
                // (not read again here: 2 - 4 % faster past the caches; parts are)
                f32x4 *const to = (f32x4 *)(out + (size_t)(o + r) * p.C_in + c);
                if (p.splits > 1) *to = v;
                else __builtin_nontemporal_store(v, to);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

// The parts of a sum in their order: workgroups of `dw` first, a row (or some of it) each (splits > 1), then those of dalpha.
template <class T, int SPLITS>
__global__ __launch_bounds__(256)
void linear_grad_join_kernel(GradArgs p, float *__restrict__ dw, float *__restrict__ dalpha, unsigned dw_blocks)
{
    const int rows = p.groups * p.C_out;
    if (blockIdx.x < dw_blocks) {
        const int row = blockIdx.x, grp = row / p.C_out;
        int lo, hi;
        group_rows(p.offsets, grp, p.rows, lo, hi);
        const float a = hi > lo ? (float)((const T *)p.alpha)[(size_t)grp * p.alpha_stride + (row - grp * p.C_out)] : 0.0f;
        const int64_t n = (int64_t)rows * p.C_in;
        for (int i = threadIdx.x * 4; i < p.C_in; i += 1024) {
            const float *from = p.part + (int64_t)row * p.C_in + i;
            f32x4 v[SPLITS];
#pragma unroll
            for (int s = 0; s < SPLITS; ++s) v[s] = *(const f32x4 *)(from + s * n);
#pragma unroll
            for (int s = 1; s < SPLITS; ++s) v[0] += v[s];
            *(f32x4 *)(dw + (int64_t)row * p.C_in + i) = v[0] * a;
        }
        return;
    }
    const int i = (int)(blockIdx.x - dw_blocks) * 256 + threadIdx.x;
    if (i >= rows) return;
    const int parts = p.splits * p.ti;
    float sum = 0.0f;
    for (int s = 0; s < parts; s += 8) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = s + k < parts ? p.alpha_part[(size_t)(s + k) * rows + i] : 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += v[k];
    }
    dalpha[i] = sum;
}

// Tiles and parts of a call.  Tiles of 256 x 256 where they fill the chip (16384 rows, 8 groups 4096 -> 4096: 550 us against 751 in 128 x 128;
// 8 groups of 3000 rows 512 -> 2904, 192 tiles: 31 against 30; 5 groups of 2999 rows 776 -> 1304, 120 tiles: 32 against 25); else of
// 128 x 128, and where these do not either and groups are long, their rows in up to eight parts, which a second launch joins
// (4096 rows 1024 -> 1024, 64 tiles: 44 us whole, 30, 26 and 32 in 2, 4 and 8 parts; 385 tiles: 25 whole, 35 in 2).
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
    while (!p.large && p.splits < 8 && tiles * p.splits < 256 && each / (2 * p.splits) >= 256) p.splits *= 2;
    p.alpha_floats = (size_t)p.splits * p.ti * g.G * g.C_out;
    p.part_floats = p.splits > 1 ? (size_t)p.splits * g.G * g.C_out * g.C_in : 0;
    return p;
}

template <class T, int B, int WI, int WO>
int launch_grad(const GradArgs &p, hipStream_t s)
{
    constexpr int WAVES = (B / WI) * (B / WO), STAGES = 4;
    constexpr size_t TILES = STAGES * (32 * B * 2 * 2), OUT = (size_t)WAVES * 32 * (WI * 4 + 16), LDS = TILES > OUT ? TILES : OUT;
    static_assert(LDS <= 160 * 1024, "LDS");
    static LdsGrant grant;
    const auto kernel = linear_weight_grad_kernel<T, B, B, WI, WO, STAGES>;
    const int rc = grant_dynamic_lds((const void *)kernel, LDS, grant);
    if (rc != SNN_OK) return rc;
    const int64_t grid = (int64_t)p.share * 8 * p.groups;
    if (grid >= ((int64_t)1 << 31)) return SNN_ERR_UNSUPPORTED;
    kernel<<<dim3((unsigned)grid), 64 * WAVES, LDS, s>>>(p);
    return check_launch();
}

template <class T>
int launch_typed(const GradArgs &p, bool large, float *dalpha, hipStream_t s)
{
    const int rc = large ? launch_grad<T, 256, 128, 64>(p, s) : launch_grad<T, 128, 64, 64>(p, s);
    if (rc != SNN_OK || (p.splits == 1 && !dalpha)) return rc;
    const unsigned dw_blocks = p.splits > 1 ? (unsigned)(p.groups * p.C_out) : 0;
    const unsigned alpha_blocks = dalpha ? (unsigned)((p.groups * p.C_out + 255) / 256) : 0;
    switch (p.splits) {
    case 8: linear_grad_join_kernel<T, 8><<<dw_blocks + alpha_blocks, 256, 0, s>>>(p, p.dw, dalpha, dw_blocks); break;
    case 4: linear_grad_join_kernel<T, 4><<<dw_blocks + alpha_blocks, 256, 0, s>>>(p, p.dw, dalpha, dw_blocks); break;
    default: linear_grad_join_kernel<T, 2><<<dw_blocks + alpha_blocks, 256, 0, s>>>(p, p.dw, dalpha, dw_blocks); break;
    }
    return check_launch();
}

}  // namespace

size_t linear_weight_grad_workspace_bytes(const LinearGeom &g, int64_t rows, bool kept)
{
    const GradPlan p = grad_plan(g, rows);
    return align_up(p.alpha_floats * 4, 256) + align_up(p.part_floats * 4, 256) + (kept ? align_up((size_t)rows * g.C_in * 2, 256) : 0);
}

// Inputs in 8 bits are first written to the workspace as the values that they stand for.  A product that widens bytes itself is slower: every
// tile of outputs widens its inputs again (150 VALU instructions for 16 matrix instructions of a wave, as many cycles as these take), 16384 rows
// 4096 -> 4096 545 us against 420 and 35 for writing them.
int launch_linear_weight_grad(const LinearGeom &g, const RowsIn &x, const void *dy, int64_t lddy, int64_t rows, const int32_t *offsets,
                              const void *weights, float *dw, float *dalpha, void *ws, hipStream_t s)
{
    const GradPlan plan = grad_plan(g, rows);
    const char *w = (const char *)weights;
    char *const at = (char *)ws + align_up(plan.alpha_floats * 4, 256);
    GradArgs p = {};
    p.x = x.p; p.ldx = x.ld;
    if (x.e && rows) {
        p.x = at + align_up(plan.part_floats * 4, 256);
        p.ldx = g.C_in;
        const int rc = launch_checkpoint_restore((const int8_t *)x.p, x.e, rows, g.C_in, g.dtype, (void *)p.x, p.ldx, s);
        if (rc != SNN_OK) return rc;
    }
    p.dy = dy; p.lddy = lddy; p.rows = (int)rows; p.groups = g.G; p.offsets = offsets;
    p.image = (const uint32_t *)w; p.words = g.words_f; p.kbs = g.kb_f;
    p.alpha = w + g.at_alpha; p.alpha_stride = g.alpha_stride;
    p.C_in = g.C_in; p.C_out = g.C_out;
    p.ti = plan.ti; p.to = plan.to; p.splits = plan.splits;
    // An XCD's tiles form a block, the squarest that leaves none with more than its share, for each reads the inputs and gradients of its tiles: 16384
    // rows 4096 -> 4096, 16 x 16 tiles in 8 x 4 instead of 16 x 2, 8 groups 546 us against 561, one 426 against 430.  (Where no block is as even as a
    // row of tiles it is slower: 2 groups of 12000 rows 600 -> 800, 5 x 7 tiles, 39 against 35; with few rows the results' writing counts: 512 rows
    // 4096 -> 4096 33.9 against 32.9.)
    p.share = (p.ti * p.to * p.splits + 7) / 8;
    int edge = INT_MAX;
    for (int a = rows / g.G >= 1024 ? 8 : 0; a; a >>= 1) {
        const int si = (p.ti + a - 1) / a, so = (p.to + 8 / a - 1) / (8 / a);
        if (si * so * p.splits == p.share && si + so < edge) {
            p.xcds_i = a;
            p.share_i = si;
            edge = si + so;
        }
    }
    p.dw = dw;
    p.alpha_part = dalpha ? (float *)ws : nullptr;
    p.part = (float *)at;
    return g.dtype == SNN_DTYPE_BF16 ? launch_typed<__bf16>(p, plan.large, dalpha, s) : launch_typed<_Float16>(p, plan.large, dalpha, s);
}

}  // namespace snn
