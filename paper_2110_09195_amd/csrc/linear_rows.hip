// Rows through sub-bit weights: outputs and the gradient of the inputs (see linear.h for the bits' layout).
#include "linear_device.h"

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

// ---- many rows ---------------------------------------------------------------------------------------------------

// The signs of step s of a lane's word, on the pairs `one` (ones, or the scales of the eight channels): the operand's registers.
template <class T>
__device__ inline typename Half<T>::v8 signed_operand(uint32_t word, int s, u32x4 one)
{
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = ((word << (4 * s + i)) & 0x80008000u) ^ one[i];
    return __builtin_bit_cast(typename Half<T>::v8, r);
}

// The tile that a workgroup computes: rows [t0, t1) of a group, and a block of columns.  Row tiles lie inside groups; which they
// are is known on the device only, so the grid has as many workgroups as there could be and the rest end at once.  Tiles go to the
// XCDs (workgroups in turn) in runs, columns first, so that an XCD's L2 holds the rows that its workgroups share.
struct RowTile {
    int group, t0, t1, col;
};

template <int BT>
__device__ inline bool find_tile(const int32_t *offsets, int groups, int rows, int col_tiles, RowTile &tile)
{
    const int lane = threadIdx.x & 63;
    int total = 0;
    if (!offsets) total = (rows + BT - 1) / BT;
    else
        for (int g0 = 0; g0 < groups; g0 += 64) {
            int lo = 0, hi = 0;
            if (g0 + lane < groups) group_rows(offsets, g0 + lane, rows, lo, hi);
            int n = (hi - lo + BT - 1) / BT;
#pragma unroll
            for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d);
            total += n;
        }
    const int64_t tiles = (int64_t)total * col_tiles;
    const int64_t share = (tiles + 7) / 8, at = blockIdx.x / 8;
    const int64_t id = (int64_t)(blockIdx.x % 8) * share + at;
    if (at >= share || id >= tiles) return false;
    int m = (int)(id / col_tiles);
    tile.col = (int)(id - (int64_t)m * col_tiles);
    if (!offsets) {
        tile.group = 0;
        tile.t0 = m * BT;
        tile.t1 = min(tile.t0 + BT, rows);
        return true;
    }
    for (int g0 = 0; g0 < groups; g0 += 64) {
        int lo = 0, hi = 0;
        if (g0 + lane < groups) group_rows(offsets, g0 + lane, rows, lo, hi);
        const int n = (hi - lo + BT - 1) / BT;
        int upto = n;                                          // tiles of this group and those before it
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int v = __shfl_up(upto, d);
            if (lane >= d) upto += v;
        }
        const uint64_t past = __ballot(upto > m);
        if (past) {
            const int l = __builtin_ctzll(past);
            m -= __builtin_amdgcn_readlane(upto - n, l);
            tile.group = g0 + l;
            tile.t0 = __builtin_amdgcn_readlane(lo, l) + m * BT;
            tile.t1 = min(tile.t0 + BT, __builtin_amdgcn_readlane(hi, l));
            return true;
        }
        m -= __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// The adapters' share as the rows kernels add it: up [n][N][rank] and the scaled inner products, fp32 [rows][rank].
struct AdapterShare {
    const void *up;
    const float *low;
    const int32_t *of_row;
    int n, rank;
};

struct RowsArgs {
    const void *in;
    int64_t ld_in;
    int rows, groups;
    const int32_t *offsets;
    const uint32_t *image;           // of group 0
    uint32_t words;                  // of an image
    int kbs;                         // blocks of 64 contracted channels
    const void *alpha;
    uint32_t alpha_stride;
    void *out;
    int64_t ld_out;
    int N, K, col_tiles;
    AdapterShare ad;
};

// out tile = rows x signs on the matrix cores (D[n][t]: n from the bits, t the rows).
//   - Rows go to LDS 64 channels at a time (128 bytes a row, 16-byte pieces xor-ed by the row so that a fragment's reads meet no bank
//     twice), with the 64-channel blocks of the bits; STAGES of these in flight, loaded without registers.
//   - Bits become operand registers by a shift and a masked xor (two VALU instructions for 128 weights): the weights cost LDS a
//     sixteenth of what the rows cost, and HBM as well.
//   - GRAD: the contracted axis is the output channels, and alpha, on that axis, is what the signs are put on: exact, and free.
template <class T, bool GRAD, bool ADAPT, int BT, int BN, int WT, int WN, int STAGES>
__global__ __launch_bounds__(64 * (BT / WT) * (BN / WN))
void linear_rows_kernel(RowsArgs p)
{
    using H = Half<T>;
    using v8 = typename H::v8;
    constexpr int WAVES = (BT / WT) * (BN / WN), THREADS = 64 * WAVES;
    constexpr int TB = WT / 32, NB = WN / 32;
    constexpr int X_BYTES = BT * 128, BIT_BYTES = BN * 8, ALPHA_BYTES = GRAD ? 256 * WAVES : 0;
    constexpr int STAGE = X_BYTES + BIT_BYTES + ALPHA_BYTES;
    constexpr int XL = BT * 8 / THREADS;                       // 16-byte loads of a thread for the rows of a stage
    constexpr int BL = BN / 32 / WAVES;                        // and the wave's blocks of bits
    static_assert(XL * THREADS == BT * 8 && BL * WAVES * 32 == BN, "whole loads");
    constexpr int LOADS = XL + BL + (GRAD ? 1 : 0);
    extern __shared__ __align__(16) char lds[];

    RowTile tile;
    if (!find_tile<BT>(p.offsets, p.groups, p.rows, p.col_tiles, tile)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wt = wave % (BT / WT), wn = wave / (BT / WT);
    const int n0 = tile.col * BN, rows = tile.t1 - tile.t0;
    const int row_bytes = (int)p.ld_in * 2;

    const s32x4 rx = resource((const char *)p.in + (int64_t)tile.t0 * p.ld_in * 2, (uint32_t)(rows - 1) * row_bytes + p.K * 2);
    const s32x4 rb = resource(p.image + (size_t)tile.group * p.words, p.words * 4);
    const T *alpha = (const T *)p.alpha + (size_t)tile.group * p.alpha_stride;
    const s32x4 ra = resource(alpha, p.alpha_stride * 2);

    // where this thread's pieces come from
    uint32_t xo[XL];
    const int xr = tid >> 3, xc = (tid & 7) ^ (xr & 7);        // (THREADS / 8 rows further on the row's low three bits are the same)
#pragma unroll
    for (int i = 0; i < XL; ++i) {
        const int r = xr + i * (THREADS / 8);
        xo[i] = r < rows ? (uint32_t)r * row_bytes + xc * 16 : NOWHERE;
    }
    const uint32_t lds0 = lds_address(lds);
    auto issue = [&](int kb, int slot) {
        const uint32_t at = __builtin_amdgcn_readfirstlane(lds0 + slot * STAGE);
        const bool in = kb * 64 + xc * 8 < p.K;                // (past the last channel: zeros, whatever the row holds there)
#pragma unroll
        for (int i = 0; i < XL; ++i)
            load_lds16(at + i * THREADS * 16 + wave * 1024, in ? xo[i] + (uint32_t)kb * 128 : NOWHERE, rx);
#pragma unroll
        for (int i = 0; i < BL; ++i) {
            const int nb = n0 / 32 + wave * BL + i;
            load_lds4(at + X_BYTES + (wave * BL + i) * 256, kb < p.kbs ? (uint32_t)((nb * p.kbs + kb) * 64 + lane) * 4 : NOWHERE, rb);
        }
        if constexpr (GRAD) load_lds4(at + X_BYTES + BIT_BYTES + wave * 256, kb < p.kbs ? (uint32_t)kb * 128 + lane * 4 : NOWHERE, ra);
    };

    f32x16 acc[NB][TB] = {};
    for (int s = 0; s < STAGES - 1; ++s) issue(s, s);
    const int h = lane >> 5, ln = lane & 31;
    uint32_t piece[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) piece[s] = (uint32_t)(wt * WT + ln) * 128 + (((2 * s + h) ^ (ln & 7)) << 4);

    int slot = 0;
    for (int kb = 0; kb < p.kbs; ++kb) {
        // this stage has landed (the ones behind it may be in flight), and everyone is done with the slot that is loaded next
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS * (STAGES - 2)) : "memory");
        issue(kb + STAGES - 1, slot == 0 ? STAGES - 1 : slot - 1);
        const char *at = lds + slot * STAGE;
        uint32_t word[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) word[i] = *(const uint32_t *)(at + X_BYTES + ((wn * NB + i) * 64 + lane) * 4);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            u32x4 one = {H::ONES, H::ONES, H::ONES, H::ONES};
            if constexpr (GRAD) one = *(const u32x4 *)(at + X_BYTES + BIT_BYTES + wave * 256 + (2 * s + h) * 16);
            v8 x[TB], w[NB];
#pragma unroll
            for (int i = 0; i < TB; ++i) x[i] = *(const v8 *)(at + piece[s] + i * 4096);
#pragma unroll
            for (int i = 0; i < NB; ++i) w[i] = signed_operand<T>(word[i], s, one);
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int j = 0; j < TB; ++j) acc[i][j] = H::mfma(w[i], x[j], acc[i][j]);
        }
        slot = slot == STAGES - 1 ? 0 : slot + 1;
    }
    // nothing of this workgroup writes to LDS any more, and every wave is done reading
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");

    // Lane: row ln of a block of 32, columns 8 g + 4 h + i of register 4 g + i.  Through LDS (a wave's own 32 rows) to whole lines.
    constexpr int PITCH = WN * 2 + 16;
    char *mine = lds + wave * 32 * PITCH;
    const int nw = n0 + wn * WN;
#pragma unroll
    for (int j = 0; j < TB; ++j) {
        const int tj = tile.t0 + wt * WT + j * 32;
        if constexpr (!GRAD) {
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int n = min(nw + i * 32 + g * 8, p.N - 8) + 4 * h;
                    const typename H::v4 a = *(const typename H::v4 *)(alpha + n);
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[i][j][4 * g + k] *= (float)a[k];
                }
        }
        if constexpr (ADAPT) {
            // For each adapter of these 32 rows in turn: its product with the rows' inner products, added where the row is its own.
            const int t = tj + ln;
            const int id = t < tile.t1 ? p.ad.of_row[t] : -1;
            uint64_t left = __ballot(id >= 0 && id < p.ad.n);
            while (left) {
                const int a = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
                const bool own = id == a;
                left &= ~__ballot(own);
                f32x16 d[NB] = {};
                for (int r0 = 0; r0 < p.ad.rank; r0 += 16) {
                    const int r = r0 + 8 * h;
                    const bool in = r < p.ad.rank;
                    float z[8] = {};
                    if (in && own) {
                        *(f32x4 *)z = *(const f32x4 *)(p.ad.low + (int64_t)t * p.ad.rank + r);
                        *(f32x4 *)(z + 4) = *(const f32x4 *)(p.ad.low + (int64_t)t * p.ad.rank + r + 4);
                    }
                    v8 hi, lo;
                    split8<T>(z, hi, lo);
#pragma unroll
                    for (int i = 0; i < NB; ++i) {
                        const int n = min(nw + i * 32 + ln, p.N - 1);
                        v8 u = {};
                        if (in) u = *(const v8 *)((const T *)p.ad.up + ((int64_t)a * p.N + n) * p.ad.rank + r);
                        d[i] = H::mfma(u, hi, d[i]);
                        d[i] = H::mfma(u, lo, d[i]);
                    }
                }
#pragma unroll
                for (int i = 0; i < NB; ++i)
#pragma unroll
                    for (int k = 0; k < 16; ++k) acc[i][j][k] += own ? d[i][k] : 0.0f;
            }
        }
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                typename H::v4 v;
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = (T)acc[i][j][4 * g + k];
                *(typename H::v4 *)(mine + ln * PITCH + (i * 32 + g * 8 + 4 * h) * 2) = v;
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        constexpr int PIECES = WN / 8;                         // of a row
#pragma unroll
        for (int i = 0; i < PIECES / 2; ++i) {
            const int q = i * 64 + lane, r = q / PIECES, c = q % PIECES;
            const u32x4 v = *(const u32x4 *)(mine + r * PITCH + c * 16);
            if (tj + r < tile.t1 && nw + c * 8 < p.N) *(u32x4 *)((T *)p.out + (int64_t)(tj + r) * p.ld_out + nw + c * 8) = v;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

// ---- few rows ----------------------------------------------------------------------------------------------------
// 32 rows by 32 columns a workgroup: its eight waves take the contracted channels in turn (blocks of 64), straight from memory (the
// weights are read once, one bit each, and the rows stay in L2), and their sums are joined in LDS in the order of the waves.
template <class T, bool GRAD, bool ADAPT>
__global__ __launch_bounds__(512)
void linear_few_kernel(RowsArgs p)
{
    using H = Half<T>;
    using v8 = typename H::v8;
    constexpr int WAVES = 8;
    __shared__ float part[WAVES][32][33];
    RowTile tile;
    if (!find_tile<32>(p.offsets, p.groups, p.rows, p.col_tiles, tile)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane >> 5, ln = lane & 31;
    const bool in_rows = tile.t0 + ln < tile.t1;
    const T *x = (const T *)p.in + (int64_t)(tile.t0 + (in_rows ? ln : 0)) * p.ld_in + 8 * h;
    const uint32_t *bits = p.image + (size_t)tile.group * p.words + (size_t)tile.col * p.kbs * 64 + lane;
    const T *alpha = (const T *)p.alpha + (size_t)tile.group * p.alpha_stride;

    f32x16 acc = {};
#pragma unroll 2
    for (int kb = wave; kb < p.kbs; kb += WAVES) {
        const uint32_t word = bits[kb * 64];
        u32x4 xs[4], one[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int k = kb * 64 + 16 * s;
            xs[s] = u32x4{0, 0, 0, 0};
            if (in_rows && k + 8 * h < p.K) xs[s] = *(const u32x4 *)(x + k);
            one[s] = u32x4{H::ONES, H::ONES, H::ONES, H::ONES};
            if constexpr (GRAD) one[s] = *(const u32x4 *)(alpha + k + 8 * h);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s)
            acc = H::mfma(signed_operand<T>(word, s, one[s]), __builtin_bit_cast(v8, xs[s]), acc);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) part[wave][ln][8 * (r >> 2) + 4 * h + (r & 3)] = acc[r];
    __syncthreads();

    const int r = tid >> 4, c = (tid & 15) * 2, t = tile.t0 + r, n = tile.col * 32 + c;
    if (t >= tile.t1 || n >= p.N) return;
    float v0 = 0.0f, v1 = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        v0 += part[w][r][c];
        v1 += part[w][r][c + 1];
    }
    if constexpr (!GRAD) {
        v0 *= (float)alpha[n];
        v1 *= (float)alpha[n + 1];
    }
    if constexpr (ADAPT) {
        const int a = p.ad.of_row[t];
        if (a >= 0 && a < p.ad.n) {
            const T *u = (const T *)p.ad.up + ((int64_t)a * p.N + n) * p.ad.rank;
            const float *z = p.ad.low + (int64_t)t * p.ad.rank;
            for (int q = 0; q < p.ad.rank; q += 8) {
                const v8 u0 = *(const v8 *)(u + q), u1 = *(const v8 *)(u + p.ad.rank + q);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v0 = fmaf(z[q + i], (float)u0[i], v0);
                    v1 = fmaf(z[q + i], (float)u1[i], v1);
                }
            }
        }
    }
    const typename H::v2 out = {(T)v0, (T)v1};
    *(typename H::v2 *)((T *)p.out + (int64_t)t * p.ld_out + n) = out;
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

namespace {

// workgroups for tiles of BT rows: as many as there can be, in whole turns of the XCDs
int64_t tile_grid(int64_t rows, int groups, int BT, int col_tiles)
{
    const int64_t used = rows < groups ? rows : groups;
    return ((rows + used * (BT - 1)) / BT * col_tiles + 7) / 8 * 8;
}

template <class T, bool GRAD, bool ADAPT, int BT, int BN, int WT, int WN, int STAGES>
int launch_tiles(RowsArgs p, hipStream_t s)
{
    constexpr int WAVES = (BT / WT) * (BN / WN);
    constexpr size_t LDS = (size_t)STAGES * (BT * 128 + BN * 8 + (GRAD ? 256 * WAVES : 0));
    static_assert(LDS >= (size_t)WAVES * 32 * (WN * 2 + 16) && LDS <= 160 * 1024, "LDS");
    static LdsGrant grant;
    const auto kernel = linear_rows_kernel<T, GRAD, ADAPT, BT, BN, WT, WN, STAGES>;
    const int rc = grant_dynamic_lds((const void *)kernel, LDS, grant);
    if (rc != SNN_OK) return rc;
    p.col_tiles = (p.N + BN - 1) / BN;
    const int64_t grid = tile_grid(p.rows, p.groups, BT, p.col_tiles);
    if (grid >= ((int64_t)1 << 31)) return SNN_ERR_UNSUPPORTED;
    kernel<<<dim3((unsigned)grid), 64 * WAVES, LDS, s>>>(p);
    return check_launch();
}

template <class T, bool GRAD, bool ADAPT>
int launch_rows(RowsArgs p, hipStream_t s)
{
    const int64_t per_group = (p.rows + p.groups - 1) / p.groups;
    if (per_group <= 64) {
        p.col_tiles = (p.N + 31) / 32;
        const int64_t grid = tile_grid(p.rows, p.groups, 32, p.col_tiles);
        linear_few_kernel<T, GRAD, ADAPT><<<dim3((unsigned)grid), 512, 0, s>>>(p);
        return check_launch();
    }
    const int64_t large = (int64_t)((p.rows + 255) / 256) * ((p.N + 255) / 256);
    if (per_group >= 256 && large >= 200) return launch_tiles<T, GRAD, ADAPT, 256, 256, 128, 64, 4>(p, s);
    return launch_tiles<T, GRAD, ADAPT, 128, 128, 64, 64, 4>(p, s);
}

template <class T>
int launch_typed(const RowsArgs &p, bool grad, hipStream_t s)
{
    if (p.ad.up) return grad ? launch_rows<T, true, true>(p, s) : launch_rows<T, false, true>(p, s);
    return grad ? launch_rows<T, true, false>(p, s) : launch_rows<T, false, false>(p, s);
}

}  // namespace

int launch_linear_rows(const LinearGeom &g, bool grad, const void *in, int64_t ld_in, int64_t rows, const int32_t *offsets,
                       const void *weights, void *out, int64_t ld_out, const Adapters *ad, const void *up, const float *low, hipStream_t s)
{
    const char *w = (const char *)weights;
    RowsArgs p = {};
    p.in = in; p.ld_in = ld_in; p.rows = (int)rows; p.groups = offsets ? g.G : 1; p.offsets = offsets;
    p.image = (const uint32_t *)(grad ? w + g.at_d : w);
    p.words = grad ? g.words_d : g.words_f;
    p.kbs = grad ? g.kb_d : g.kb_f;
    p.alpha = w + g.at_alpha; p.alpha_stride = g.alpha_stride;
    p.out = out; p.ld_out = ld_out;
    p.N = grad ? g.C_in : g.C_out;
    p.K = grad ? g.C_out : g.C_in;
    if (ad) p.ad = {up, low, ad->of_row, ad->n, ad->rank};
    return g.dtype == SNN_DTYPE_BF16 ? launch_typed<__bf16>(p, grad, s) : launch_typed<_Float16>(p, grad, s);
}

}  // namespace snn
