// Rows through sub-bit weights: outputs and the gradient of the inputs (see linear.h for the bits' layout).
#include "linear_device.h"

#include <type_traits>

#include <math.h>

namespace snn {

namespace {

// ---- the images of the weights ---------------------------------------------------------------------------------
// A block of 64 output channels by 64 vectors (512 input channels).  A member's byte is kept with the bits of its odd elements (1, 3, 5, 7 from the top) in the
// high nibble and those of its even ones in the low one, set for -1: in that order four bytes make a word by their nibbles alone (linear.h).
// F takes the bytes as they are; for D, 8 x 8 bits (the members of 8 outputs) are turned by three exchanges of bits.
// Bound by memory and the members' look-up: 8 matrices of 4096 x 4096 (34 MB of indices in, 34 MB of images out) 18.3 us, 3.7 TB/s.
constexpr int PREP_O = 64, PREP_V = 64, PREP_THREADS = 256;

// The word of four bytes B0 .. B3, given with B0 at the top: low nibbles to the low half, high ones to the high half.
__device__ inline uint32_t word_of_nibbles(uint32_t b)
{
    uint32_t even = b & 0x0f0f0f0fu, odd = (b >> 4) & 0x0f0f0f0fu;
    even = (even | even >> 4) & 0x00ff00ffu;
    odd = (odd | odd >> 4) & 0x00ff00ffu;
    even = (even | even >> 8) & 0xffffu;
    odd = (odd | odd >> 8) & 0xffffu;
    return even | odd << 16;
}

// Bit c of byte r <-> bit r of byte c, of the eight bytes lo (0 .. 3), hi (4 .. 7): 2 x 2 bits, then 2 x 2 such blocks, then those.
__device__ inline void turn_8x8(uint32_t &lo, uint32_t &hi)
{
    uint32_t t = (lo ^ lo >> 7) & 0x00aa00aau;
    lo ^= t ^ t << 7;
    t = (hi ^ hi >> 7) & 0x00aa00aau;
    hi ^= t ^ t << 7;
    t = (lo ^ lo >> 14) & 0x0000ccccu;
    lo ^= t ^ t << 14;
    t = (hi ^ hi >> 14) & 0x0000ccccu;
    hi ^= t ^ t << 14;
    t = (lo ^ hi << 4) & 0xf0f0f0f0u;
    lo ^= t;
    hi ^= t >> 4;
}

__global__ __launch_bounds__(PREP_THREADS)
void linear_prepare_kernel(LinearGeom g, const uint16_t *__restrict__ codebook, const uint16_t *__restrict__ idx,
                           const uint16_t *__restrict__ alpha, uint32_t *__restrict__ image_f, uint32_t *__restrict__ image_d,
                           uint16_t *__restrict__ alpha_out)
{
    __shared__ __align__(16) uint8_t by_o[PREP_O][PREP_V + 8], by_v[PREP_V][PREP_O + 8];
    __shared__ uint8_t member[256];
    const int tid = threadIdx.x, grp = blockIdx.z;
    const int ob = blockIdx.y, o0 = ob * PREP_O, v0 = blockIdx.x * PREP_V;
    const int V = g.C_in / 8;
    codebook += (size_t)grp * g.K;
    idx += (size_t)grp * g.C_out * V;
    int k[PREP_O * PREP_V / PREP_THREADS];                     // this thread's indices: all loads before the first use
#pragma unroll
    for (int i = 0; i < PREP_O * PREP_V / PREP_THREADS; ++i) {
        const int n = i * PREP_THREADS + tid, o = o0 + n / PREP_V, v = v0 + n % PREP_V;
        k[i] = o < g.C_out && v < V ? idx[(size_t)o * V + v] : -1;
    }
    if (tid < g.K) {
        const uint32_t c = ~(uint32_t)codebook[tid];           // element j at bit 7 - j, set for -1
        uint32_t m = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) m |= ((c >> (7 - 2 * r)) & 1u) << (3 - r) | ((c >> (6 - 2 * r)) & 1u) << (7 - r);
        member[tid] = (uint8_t)m;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PREP_O * PREP_V / PREP_THREADS; ++i) {
        const int n = i * PREP_THREADS + tid, o = n / PREP_V, v = n % PREP_V;
        const uint8_t c = k[i] < 0 ? (uint8_t)0 : member[min(k[i], g.K - 1)];
        by_o[o][v] = c;
        by_v[v][o] = c;
    }
    __syncthreads();
    if (tid < 128) {
        // F, half h of the words of an output: bytes 2 s + h of its eight of a block of 64 inputs
        const int h = tid >> 6, o = tid & 63, nb = 2 * ob + (o >> 5);
        if (nb < g.nb_f) {
            uint32_t *to = image_f + (size_t)grp * g.words_f + ((size_t)nb * g.kb_f + v0 / 8) * 64 + h * 32 + (o & 31);
#pragma unroll
            for (int kb = 0; kb < PREP_V / 8; ++kb) {
                const u32x2 b = *(const u32x2 *)&by_o[o][kb * 8];
                const uint32_t four = h ? __builtin_amdgcn_perm(b[0], b[1], 0x05070103u) : __builtin_amdgcn_perm(b[0], b[1], 0x04060002u);
                if (v0 / 8 + kb < g.kb_f) to[kb * 64] = word_of_nibbles(four);
            }
        }
    } else {
        // D, half h of the words of the eight inputs of a vector: outputs 16 s + 8 h + j, turned, then input by input
        const int h = (tid >> 6) & 1, v = tid & 63, nb = (v0 + v) / 4;
        if (nb < g.nb_d) {
            uint32_t lo[4], hi[4];                             // [s]: bytes 0 .. 3 and 4 .. 7 of the turned eight, that is by bit of a member
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const u32x2 b = *(const u32x2 *)&by_v[v][16 * s + 8 * h];
                lo[s] = __builtin_amdgcn_perm(b[1], b[0], 0x00020406u);       // outputs 6, 4, 2, 0: bits 0 .. 3 of a byte of the word
                hi[s] = __builtin_amdgcn_perm(b[1], b[0], 0x01030507u);       // 7, 5, 3, 1
                turn_8x8(lo[s], hi[s]);
            }
            uint32_t word[8];                                  // by input j: odd ones from bit 7 - j / 2, even ones from bit 3 - j / 2
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const uint32_t *from = c < 4 ? lo : hi;
                const uint32_t sel = 0x0c0c0000u | (uint32_t)(c & 3) | (uint32_t)(4 + (c & 3)) << 8;
                const uint32_t top = __builtin_amdgcn_perm(from[0], from[1], sel), low = __builtin_amdgcn_perm(from[2], from[3], sel);
                word[c >= 4 ? 2 * (7 - c) + 1 : 2 * (3 - c)] = word_of_nibbles(top << 16 | low);
            }
            uint32_t *to = image_d + (size_t)grp * g.words_d + ((size_t)nb * g.kb_d + ob) * 64 + h * 32 + ((v0 + v) & 3) * 8;
            *(u32x4 *)to = u32x4{word[0], word[1], word[2], word[3]};
            *(u32x4 *)(to + 4) = u32x4{word[4], word[5], word[6], word[7]};
        }
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
__device__ inline bool find_tile(const int32_t *offsets, int groups, int rows, int col_tiles, const Divisor &col_div, uint32_t most, RowTile &tile)
{
    const int lane = threadIdx.x & 63;
    // (groups g0 .. g0 + 63, a lane each: their rows, and the tiles of those up to it)
    auto look = [&](int g0, int &lo, int &hi) {
        lo = hi = 0;
        if (g0 + lane < groups) group_rows(offsets, g0 + lane, rows, lo, hi);
        int upto = (hi - lo + BT - 1) / BT;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int v = __shfl_up(upto, d);
            if (lane >= d) upto += v;
        }
        return upto;
    };
    // No more tiles than the grid has workgroups (`most` of rows).  Offsets that do not decrease never name more (see tile_grid); those that go down and up
    // again can, up to the whole of the rows for every other group: then the surplus is dropped, and which group's result a row gets is not defined.
    uint32_t total;
    int lo = 0, hi = 0, upto = 0;
    if (!offsets) total = (uint32_t)(rows + BT - 1) / BT;
    else {
        upto = look(0, lo, hi);
        total = min((uint32_t)__builtin_amdgcn_readlane(upto, 63), most);
        for (int g0 = 64; g0 < groups; g0 += 64) {
            int l, h;
            total = min(total + (uint32_t)__builtin_amdgcn_readlane(look(g0, l, h), 63), most);
        }
    }
    const uint32_t tiles = total * (uint32_t)col_tiles;
    const uint32_t share = (tiles + 7) / 8, at = blockIdx.x / 8;
    const uint32_t id = (blockIdx.x % 8) * share + at;
    if (at >= share || id >= tiles) return false;
    int m = (int)fast_div(id, col_div);
    tile.col = (int)id - m * col_tiles;
    if (!offsets) {
        tile.group = 0;
        tile.t0 = m * BT;
        tile.t1 = min(tile.t0 + BT, rows);
        return true;
    }
    for (int g0 = 0;;) {
        const uint64_t past = __ballot(upto > m);
        if (past) {
            const int l = __builtin_ctzll(past);
            m -= l ? __builtin_amdgcn_readlane(upto, l - 1) : 0;
            tile.group = g0 + l;
            tile.t0 = __builtin_amdgcn_readlane(lo, l) + m * BT;
            tile.t1 = min(tile.t0 + BT, __builtin_amdgcn_readlane(hi, l));
            return true;
        }
        m -= __builtin_amdgcn_readlane(upto, 63);
        g0 += 64;
        if (g0 >= groups) return false;
        upto = look(g0, lo, hi);
    }
}

// The adapters' share as the rows kernels add it: up [n][N][rank] and the scaled inner products, fp32 [rows][rank].
struct AdapterShare {
    const void *up;
    const float *low;
    const int32_t *of_row;
    int n, rank;
    const void *down;                // OWN: the adapters' other matrix [n][rank][K], their scales, and where the unscaled inner products go
    const float *scale;
    float *low_out;
};

// How the adapters' share gets its inner products: not at all, from another launch, or by the kernel itself.
enum { NONE, GIVEN, OWN };

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
    Divisor col_div;                 // by col_tiles
    uint32_t most;                   // tiles of rows that the grid has workgroups for
    AdapterShare ad;
};

// out tile = rows x signs on the matrix cores (D[n][t]: n from the bits, t the rows).
//   - Rows go to LDS 64 channels at a time (128 bytes a row, 16-byte pieces xor-ed by half the row's number, so that the sixteen
//     rows that are read at once lie in sixteen different places of the 256 bytes of banks), with the 64-channel blocks of the bits; STAGES of these in flight, loaded without registers.
//   - Bits become operand registers by a shift and a masked xor (two VALU instructions for 128 weights): the weights cost LDS a
//     sixteenth of what the rows cost, and HBM as well.
//   - GRAD: the contracted axis is the output channels, and alpha, on that axis, is what the signs are put on: exact, and free.
// Bound: many rows by the matrix pipes at the clock that the chip's power leaves them (77 % busy; 16384 rows in 8 groups of uneven sizes, 4096 ->
// 4096, 413 us = 1.33 PFLOP/s, 16384 rows 8192 -> 8192 in one 1427 us = 1.54; input gradients 434 and 1490), few rows by a step's latency, 0.3 us:
// 1537 rows of 60 groups, 1032 -> 1416, 13.3 us.
template <class T, bool GRAD, int ADAPT, int BT, int BN, int WT, int WN, int STAGES, bool DEEP>
__global__ __launch_bounds__(64 * (BT / WT) * (BN / WN), 2)
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
    if (!find_tile<BT>(p.offsets, p.groups, p.rows, p.col_tiles, p.col_div, p.most, tile)) return;
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
    const int xr = tid >> 3, xc = (tid & 7) ^ ((xr >> 1) & 7); // (THREADS / 8 rows further on these bits of the row are the same)
#pragma unroll
    for (int i = 0; i < XL; ++i) {
        const int r = xr + i * (THREADS / 8);
        xo[i] = r < rows ? (uint32_t)r * row_bytes + xc * 16 : NOWHERE;
    }
    const uint32_t lds0 = lds_address(lds);
    // a quarter of a step's loads
    // Input gradients in tiles of 128 x 256 start each row of tiles at another channel: 2048 rows of 4096 -> 4096 68.7 -> 61.2 us, 8 experts of
    // 8192 rows 236 -> 230 (others lose by it: tiles of 32 x 128 14.2 -> 15.4, outputs 2 %).
    constexpr bool TURNED = GRAD && BT == 128 && BN == 256;
    const int turn = TURNED ? tile.t0 / BT * 5 % p.kbs : 0;
    auto issue = [&](int step, int slot, int part) {
        int kb = step;
        if constexpr (TURNED) kb = step >= p.kbs ? step : step + turn >= p.kbs ? step + turn - p.kbs : step + turn;
        const uint32_t at = __builtin_amdgcn_readfirstlane(lds0 + slot * STAGE);
        const bool in = kb * 64 + xc * 8 < p.K;                // (past the last channel: zeros, whatever the row holds there)
#pragma unroll
        for (int i = part * XL / 4; i < (part + 1) * XL / 4; ++i)
            load_lds16(at + i * THREADS * 16 + wave * 1024, in ? xo[i] + (uint32_t)kb * 128 : NOWHERE, rx);
        if (part == 0) {
#pragma unroll
            for (int i = 0; i < BL; ++i) {
                const int nb = n0 / 32 + wave * BL + i;
                load_lds4(at + X_BYTES + (wave * BL + i) * 256, kb < p.kbs ? (uint32_t)((nb * p.kbs + kb) * 64 + lane) * 4 : NOWHERE, rb);
            }
            if constexpr (GRAD) load_lds4(at + X_BYTES + BIT_BYTES + wave * 256, kb < p.kbs ? (uint32_t)kb * 128 + lane * 4 : NOWHERE, ra);
        }
    };

    f32x16 acc[NB][TB] = {};
    for (int s = 0; s < (DEEP ? STAGES : STAGES - 1); ++s)
        for (int q = 0; q < 4; ++q) issue(s, s, q);
    const int h = lane >> 5, ln = lane & 31;
    uint32_t piece[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) piece[s] = (uint32_t)(wt * WT + ln) * 128 + (((2 * s + h) ^ ((ln >> 1) & 7)) << 4);

    uint32_t ones = H::ONES;
    asm("" : "+v"(ones));                                      // (known to be constant, the masked xor would take two instructions)
    if constexpr (DEEP) {
        // Small tiles: a wave has too few products to hide LDS behind 16 channels at a time, and there may be no other wave on its SIMD.  All
        // fragments of the next 64 channels are read while these are multiplied; a slot is free as soon as it has been read.  512 rows, 4096 -> 4096 in
        // 64 x 128: outputs 22.6 -> 19.7 us, input gradients 29.5 -> 21.0.  (128 x 128 loses by it: 26.3 -> 30.7.)
        v8 x[2][4][TB];
        uint32_t word[2][NB];
        u32x4 one[2][4];
        auto fetch = [&](int slot, int to) {
            const char *at = lds + slot * STAGE;
#pragma unroll
            for (int i = 0; i < NB; ++i) word[to][i] = *(const uint32_t *)(at + X_BYTES + ((wn * NB + i) * 64 + lane) * 4);
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                one[to][s] = u32x4{ones, ones, ones, ones};
                if constexpr (GRAD) one[to][s] = *(const u32x4 *)(at + X_BYTES + BIT_BYTES + wave * 256 + (2 * s + h) * 16);
#pragma unroll
                for (int i = 0; i < TB; ++i) x[to][s][i] = *(const v8 *)(at + piece[s] + i * 4096);
            }
        };
        int slot = 0;
        auto step = [&](int kb, auto which) {
            constexpr int from = decltype(which)::value;
            // the next step's loads have landed, and everyone has read this step's
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS * (STAGES - 2)) : "memory");
            const int next = slot == STAGES - 1 ? 0 : slot + 1;
            fetch(next, from ^ 1);
#pragma unroll
            for (int q = 0; q < 4; ++q) issue(kb + STAGES, slot, q);
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int i = 0; i < NB; ++i) {
                    const v8 w = signed_operand<T>(word[from][i], s, one[from][s]);
#pragma unroll
                    for (int j = 0; j < TB; ++j) acc[i][j] = H::mfma(w, x[from][s][j], acc[i][j]);
                }
            slot = next;
        };
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(LOADS * (STAGES - 1)) : "memory");
        fetch(0, 0);
        for (int kb = 0; kb < p.kbs; kb += 2) {                // (a step past the last: zeros)
            step(kb, std::integral_constant<int, 0>{});
            step(kb + 1, std::integral_constant<int, 1>{});
        }
    } else {
        // While the products of 16 channels run, the operands of the next 16 are made: fragments are read from LDS, bits turned into registers.  The
        // instructions are dealt out between the matrix instructions, in whose shadow they issue.
        v8 x[2][TB], w[2][NB];
        uint32_t word[NB];
        auto read_x = [&](int slot, int s, int to) {
#pragma unroll
            for (int i = 0; i < TB; ++i) x[to][i] = *(const v8 *)(lds + slot * STAGE + piece[s] + i * 4096);
        };
        auto read_word = [&](int slot) {
#pragma unroll
            for (int i = 0; i < NB; ++i) word[i] = *(const uint32_t *)(lds + slot * STAGE + X_BYTES + ((wn * NB + i) * 64 + lane) * 4);
        };
        uint32_t word_next[NB];
        auto read_word_next = [&](int slot) {
#pragma unroll
            for (int i = 0; i < NB; ++i) word_next[i] = *(const uint32_t *)(lds + slot * STAGE + X_BYTES + ((wn * NB + i) * 64 + lane) * 4);
        };
        auto make_w = [&](int slot, int s, int to) {
            u32x4 one = {ones, ones, ones, ones};
            if constexpr (GRAD) one = *(const u32x4 *)(lds + slot * STAGE + X_BYTES + BIT_BYTES + wave * 256 + (2 * s + h) * 16);
#pragma unroll
            for (int i = 0; i < NB; ++i) w[to][i] = signed_operand<T>(word[i], s, one);
        };
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(LOADS * (STAGES - 2)) : "memory");
        read_word(0);
        read_x(0, 0, 0);
        make_w(0, 0, 0);
        int slot = 0;
        for (int kb = 0; kb < p.kbs; ++kb) {
            // the next step's loads have landed (the ones behind it may be in flight), and everyone is done with the slot that is loaded next
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS * (STAGES - 3)) : "memory");
            const int free = slot == 0 ? STAGES - 1 : slot - 1, next = slot == STAGES - 1 ? 0 : slot + 1;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                issue(kb + STAGES - 1, free, s);
                if (s == 2) read_word_next(next);
                if (s < 3) {
                    read_x(slot, s + 1, (s + 1) & 1);
                    make_w(slot, s + 1, (s + 1) & 1);
                } else {
                    read_x(next, 0, 0);
#pragma unroll
                    for (int i = 0; i < NB; ++i) word[i] = word_next[i];
                    make_w(next, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < NB; ++i)
#pragma unroll
                    for (int j = 0; j < TB; ++j) acc[i][j] = H::mfma(w[s & 1][i], x[s & 1][j], acc[i][j]);
#pragma unroll
                for (int i = 0; i < NB * TB; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);           // a matrix instruction
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);           // an LDS read
                    __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);           // VALU
                }
            }
            slot = next;
        }
    }
    int ids[TB];                                               // the adapters of the rows 32 j + ln
    if constexpr (ADAPT) {
#pragma unroll
        for (int j = 0; j < TB; ++j) {
            const int t = tile.t0 + wt * WT + j * 32 + ln;
            ids[j] = t < tile.t1 ? p.ad.of_row[t] : -1;
        }
    }
    // nothing of this workgroup writes to LDS any more, and every wave is done reading
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");

    // Lane: row ln of a block of 32, columns 8 g + 4 h + i of register 4 g + i.  Through LDS (a wave's own 32 rows) to whole lines.
    constexpr int PITCH = WN * 2 + 16;
    char *mine = lds + wave * 32 * PITCH;
    const int nw = n0 + wn * WN;
    // (With adapters every register counts: what would be kept for the next 32 rows, scales and addresses, would put others into scratch memory, and
    // waves with scratch start later.  Hence the empty assembly statements, past which nothing is kept.)
    u32x4 u[4][NB] = {};
    int held = -1;
#pragma unroll
    for (int j = 0; j < TB; ++j) {
        const int tj = tile.t0 + wt * WT + j * 32;
        if constexpr (!GRAD) {
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    int n = min(nw + i * 32 + g * 8, p.N - 8) + 4 * h;
                    if constexpr (ADAPT) asm volatile("" : "+v"(n));
                    const typename H::v4 a = *(const typename H::v4 *)(alpha + n);
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[i][j][4 * g + k] *= (float)a[k];
                }
        }
        if constexpr (ADAPT) {
            // For each adapter of these 32 rows in turn: its product with the rows' inner products, added where the row is its own.  (Tiles start at
            // multiples of 32; a matrix of the rank 64 or less stays for the next rows when they have the same adapter.)
            const int id = ids[j];
            uint64_t left = __ballot(id >= 0 && id < p.ad.n);
            while (left) {
                const int a = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
                const bool own = id == a;
                left &= ~__ballot(own);
                int rank = p.ad.rank;
                asm volatile("" : "+s"(rank));
                const __amdgpu_buffer_rsrc_t ru = buffer((const T *)p.ad.up + (int64_t)a * p.N * rank, (uint32_t)p.N * rank * 2);
                const __amdgpu_buffer_rsrc_t rz = buffer(p.ad.low + scaled_at(tj, 0, rank), 32u * rank * 4);
                const uint32_t zo = own ? (uint32_t)(8 * h * 32 + ln * 4) * 4 : NOWHERE;
                for (int r0 = 0; r0 < rank; r0 += 64) {
                    // 64 of the rank: all loads before the first product
                    u32x4 z[4][2];
                    const bool load_u = a != held;
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        const int r = r0 + 16 * s + 8 * h;
                        if (load_u)
#pragma unroll
                            for (int i = 0; i < NB; ++i)
                                u[s][i] = __builtin_amdgcn_raw_buffer_load_b128(ru, r < rank ? (uint32_t)((nw + i * 32 + ln) * rank + r) * 2 : NOWHERE, 0, 0);
#pragma unroll
                        for (int i = 0; i < 2; ++i) z[s][i] = __builtin_amdgcn_raw_buffer_load_b128(rz, zo + (uint32_t)(r0 + 16 * s + 4 * i) * 128, 0, 0);
                    }
                    // (a power of two a row, whose column of D the lanes ln and ln + 32 hold)
                    float up = 1.0f, down = 1.0f;
                    if constexpr (Pieces<T>::SCALED) {
                        float top = 0.0f;
#pragma unroll
                        for (int s = 0; s < 4; ++s) {
                            if (r0 + 16 * s >= rank) break;
#pragma unroll
                            for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(__uint_as_float(z[s][i >> 2][i & 3])));
                        }
                        const int e = piece_exponent(larger_half(top));
                        up = power_of_two(e);
                        down = power_of_two(-e);
                    }
                    f32x16 d[NB] = {};
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        if (r0 + 16 * s >= rank) break;
                        float zf[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) zf[i] = __uint_as_float(z[s][i >> 2][i & 3]);
                        const Pieces<T> piece = split8<T>(zf, up);
#pragma unroll
                        for (int i = 0; i < NB; ++i)
#pragma unroll
                            for (int k = 0; k < Pieces<T>::N; ++k) d[i] = H::mfma(__builtin_bit_cast(v8, u[s][i]), piece.of[k], d[i]);
                    }
#pragma unroll
                    for (int i = 0; i < NB; ++i)
#pragma unroll
                        for (int k = 0; k < 16; ++k) acc[i][j][k] += own ? d[i][k] * down : 0.0f;
                }
                held = p.ad.rank <= 64 ? a : -1;
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
// Few rows of small adapters need one launch, not two: eight more waves make the inner products beside the others, in every workgroup again, which is
// little as long as there are few of them (rows x rank x channels up to 64 K: 2048 -> 2048, one row of rank 8 4.3 us against 5.8, of rank 32 5.8 against 6.8,
// 64 (128 K) 8.0 against 7.9; 4096 -> 4096, two rows of rank 8 6.7 against 6.9, of rank 16 8.0 against 7.3).
constexpr int64_t OWN_PRODUCTS = 64 * 1024;
// OWN: wave `first` of eight takes NR inner products of a row at a time, to LDS with the adapter's scale and, from one workgroup, to memory without.
constexpr int OWN_DOTS = 256;
template <class T, int NR>
__device__ inline void own_dots(const RowsArgs &p, int first, int lane, bool out, float *own)
{
    using v8 = typename Half<T>::v8;
    const int rank = p.ad.rank;
    for (int i = first * NR; i < p.rows * rank; i += 8 * NR) { // (rank is a multiple of NR)
        const int t = i / rank, r = i - t * rank, a = p.ad.of_row[t];
        const bool some = a >= 0 && a < p.ad.n;
        float sum[NR] = {}, scale = 0.0f;
        if (some) {
            scale = p.ad.scale[a];
            const T *x = (const T *)p.in + t * p.ld_in, *down = (const T *)p.ad.down + ((int64_t)a * rank + r) * p.K;
#pragma unroll(NR == 1 ? 4 : 2)
            for (int k = lane * 8; k < p.K; k += 512) {
                const v8 u = *(const v8 *)(x + k);
#pragma unroll
                for (int j = 0; j < NR; ++j) {
                    const v8 v = *(const v8 *)(down + (int64_t)j * p.K + k);
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[j] = fmaf((float)u[e], (float)v[e], sum[j]);
                }
            }
#pragma unroll
            for (int d = 32; d; d >>= 1)
#pragma unroll
                for (int j = 0; j < NR; ++j) sum[j] += __shfl_xor(sum[j], d);
        }
        if (lane == 0) {
#pragma unroll
            for (int j = 0; j < NR; ++j) {
                own[i + j] = sum[j] * scale;
                if (out && p.ad.low_out) p.ad.low_out[i + j] = sum[j];
            }
        }
    }
}

// 16 rows by 16 NB columns a workgroup: its eight waves take the contracted channels in turn (blocks of 64) and their sums are joined in
// LDS in the order of the waves.  The weights are read once, one bit each; what counts is how fast a CU gets at the rows, which every
// workgroup reads (they stay in L2): neighbouring lanes have to load neighbouring bytes (150 GB/s a CU; with a row a lane, as the operand
// wants them, 38), so the rows go through LDS, without registers, a wave's own part of it, AHEAD blocks at once.  Bound by latency: 16 rows
// 4096 -> 4096 4.7 us, of which the 2 MB of weights are 0.4 at the memory's rate; 32 rows of 32 groups 2048 -> 1024 (5 MB) 6.1 with its launch.
template <class T, bool GRAD, int ADAPT, int NB, int AHEAD>
__global__ __launch_bounds__(ADAPT == OWN ? 1024 : 512)
void linear_few_kernel(RowsArgs p)
{
    using H = Half<T>;
    using v8 = typename H::v8;
    constexpr int WAVES = 8;
    // the rows on their way; then the sums
    constexpr int IN = WAVES * AHEAD * 2048, SUMS = WAVES * 16 * (16 * NB + 1) * 4;
    __shared__ __align__(16) char lds[IN > SUMS ? IN : SUMS];
    float(*const part)[16][16 * NB + 1] = (float(*)[16][16 * NB + 1])lds;
    __shared__ __align__(16) float own[ADAPT == OWN ? OWN_DOTS : 1];         // scaled inner products [rows][rank]
    RowTile tile;
    if (!find_tile<16>(p.offsets, p.groups, p.rows, p.col_tiles, p.col_div, p.most, tile)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int q = lane >> 4, ln = lane & 15, n0 = tile.col * 16 * NB;
    const s32x4 rx = resource((const T *)p.in + (int64_t)tile.t0 * p.ld_in, (uint32_t)(tile.t1 - tile.t0 - 1) * (uint32_t)p.ld_in * 2 + p.K * 2);
    // a load: 16 rows of 64 bytes, four lanes a row, their 16-byte pieces xor-ed by a quarter of the row's number against bank conflicts
    const int lr = lane >> 2, lp = (lane & 3) ^ ((lane >> 4) & 3);
    const uint32_t xo = tile.t0 + lr < tile.t1 ? (uint32_t)lr * (uint32_t)p.ld_in * 2 + lp * 16 : NOWHERE;
    char *mine = lds + wave * AHEAD * 2048;
    const uint32_t mine0 = __builtin_amdgcn_readfirstlane(lds_address(mine));
    const char *from = mine + (4 * ln + (q ^ (ln >> 2))) * 16;
    // Channels 64 kb + 32 m + 8 q + j of a lane: the half q % 2 of the block's words, steps 2 m + q / 2.
    const __amdgpu_buffer_rsrc_t rb = buffer(p.image + (size_t)tile.group * p.words, p.words * 4);
    uint32_t bo[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        const int n = n0 + 16 * i;
        bo[i] = ((uint32_t)(n >> 5) * p.kbs * 64 + (q & 1) * 32 + (n & 16) + ln) * 4;
    }
    const T *alpha = (const T *)p.alpha + (size_t)tile.group * p.alpha_stride;
    const __amdgpu_buffer_rsrc_t ra = buffer(alpha, p.alpha_stride * 2);

    f32x4 acc[NB] = {};
    if constexpr (ADAPT == OWN) {
        // the upper eight waves: inner products with the adapters' matrices
        if (wave >= WAVES) {
            if (p.rows * p.ad.rank <= 2 * WAVES) own_dots<T, 1>(p, wave - WAVES, lane, tile.col == 0, own);
            else own_dots<T, 4>(p, wave - WAVES, lane, tile.col == 0, own);
        }
    }
    for (int k0 = wave; k0 < (ADAPT == OWN && wave >= WAVES ? 0 : p.kbs); k0 += WAVES * AHEAD) {
        uint32_t word[AHEAD][NB];
        u32x4 one[AHEAD][2];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int kb = k0 + a * WAVES;                     // (blocks past the last: zeros for rows)
#pragma unroll
            for (int i = 0; i < NB; ++i) word[a][i] = __builtin_amdgcn_raw_buffer_load_b32(rb, bo[i] + kb * 256, 0, 0);
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                one[a][m] = u32x4{H::ONES, H::ONES, H::ONES, H::ONES};
                if constexpr (GRAD) one[a][m] = __builtin_amdgcn_raw_buffer_load_b128(ra, kb * 128 + m * 64 + 16 * q, 0, 0);
                load_lds16(mine0 + (a * 2 + m) * 1024, kb * 64 + 32 * m + 8 * lp < p.K ? xo + kb * 128 + m * 64 : NOWHERE, rx);
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
        for (int a = 0; a < AHEAD; ++a)
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const v8 x = *(const v8 *)(from + (a * 2 + m) * 1024);
#pragma unroll
                for (int i = 0; i < NB; ++i) acc[i] = H::mfma16(signed_operand<T>(word[a][i] << (4 * (q >> 1)), 2 * m, one[a][m]), x, acc[i]);
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    __syncthreads();
    if (ADAPT != OWN || wave < WAVES)
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) part[wave][ln][16 * i + 4 * q + r] = acc[i][r];
    __syncthreads();

    if (tid >= 128 * NB) return;
    const int r = tid / (8 * NB), c = tid % (8 * NB) * 2, t = tile.t0 + r, n = n0 + c;
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
            for (int k = 0; k < p.ad.rank; k += 8) {
                const v8 u0 = *(const v8 *)(u + k), u1 = *(const v8 *)(u + p.ad.rank + k);
                float z[8];
#pragma unroll
                for (int i = 0; i < 8; i += 4)
                    *(f32x4 *)(z + i) = ADAPT == OWN ? *(const f32x4 *)(own + t * p.ad.rank + k + i) : *(const f32x4 *)(p.ad.low + scaled_at(t, k + i, p.ad.rank));
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v0 = fmaf(z[i], (float)u0[i], v0);
                    v1 = fmaf(z[i], (float)u1[i], v1);
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

template <class T, bool GRAD, int ADAPT, int BT, int BN, int WT, int WN, int STAGES, bool DEEP>
int launch_tiles(RowsArgs p, hipStream_t s)
{
    constexpr int WAVES = (BT / WT) * (BN / WN);
    constexpr size_t LDS = (size_t)STAGES * (BT * 128 + BN * 8 + (GRAD ? 256 * WAVES : 0));
    static_assert(LDS >= (size_t)WAVES * 32 * (WN * 2 + 16) && LDS <= 160 * 1024, "LDS");
    static LdsGrant grant;
    const auto kernel = linear_rows_kernel<T, GRAD, ADAPT, BT, BN, WT, WN, STAGES, DEEP>;
    const int rc = grant_dynamic_lds((const void *)kernel, LDS, grant);
    if (rc != SNN_OK) return rc;
    p.col_tiles = (p.N + BN - 1) / BN;
    p.col_div = make_divisor(p.col_tiles);
    const int64_t grid = tile_grid(p.rows, p.groups, BT, p.col_tiles);
    if (grid >= ((int64_t)1 << 31)) return SNN_ERR_UNSUPPORTED;
    p.most = (uint32_t)(grid / p.col_tiles);
    kernel<<<dim3((unsigned)grid), 64 * WAVES, LDS, s>>>(p);
    return check_launch();
}

template <class T, bool GRAD, int ADAPT, int NB>
int launch_few(RowsArgs p, hipStream_t s)
{
    p.col_tiles = (p.N + 16 * NB - 1) / (16 * NB);
    p.col_div = make_divisor(p.col_tiles);
    const int64_t grid = tile_grid(p.rows, p.groups, 16, p.col_tiles);
    if (grid >= ((int64_t)1 << 31)) return SNN_ERR_UNSUPPORTED;
    p.most = (uint32_t)(grid / p.col_tiles);
    // (up to eight blocks of 64 channels a wave has one: 98 rows of 14 groups 512 -> 2800 6.1 us, 7.3 with loads for two)
    if (p.kbs <= 8)
        linear_few_kernel<T, GRAD, ADAPT, NB, 1><<<dim3((unsigned)grid), ADAPT == OWN ? 1024 : 512, 0, s>>>(p);
    else
        linear_few_kernel<T, GRAD, ADAPT, NB, 2><<<dim3((unsigned)grid), ADAPT == OWN ? 1024 : 512, 0, s>>>(p);
    return check_launch();
}

// Which tile a call of many rows takes.  Costs in microseconds, fitted to 59 calls and their gradients of 320 to 16384 rows, of 1 to 60 groups of
// even, random and skewed sizes, 776 to 4096 channels wide (its choice is more than 5 % slower than the best form in five of 118): for
// 64 contracted channels a tile alone on its CU with most CUs idle, and its share of a CU when all are busy (then the clock is down to
// 1.8 - 1.9 GHz: such calls are bound by power, and what moves fewer bytes for a product is faster); and once for a tile.  Adapters add 0.9 us for every
// 32 rows of a tile, whose loads wait for each other, and 0.3 when other tiles fill the wait (rank 64 or less): 1111 rows of rank 24, 1352 ->
// 2056, 22.9 us in 128 x 128, 19.7 in 32 x 128; 3636 rows, 880 -> 4096, 43 and 44, and 39 in 128 x 256.  The input's gradient also
// scales its weights, which makes small tiles dearer.  A tile is small to spread few rows over the chip and large to be fed with fewer
// reads; two of 128 x 256 stay on a CU and fill each other's waits (one of 256 x 256 instead: 72 / 69 us, 69 / 69, 100 / 104, 381 / 385).
// One group, 4096 -> 4096, outputs / input gradients in us:
//   rows    128 x 256   128 x 128   64 x 128   32 x 128
//    512      38 / 46     26 / 36    20 / 23    22 / 26
//   1024      41 / 47     32 / 39    33 / 36    39 / 45
//   4096     100 / 104   110 / 121  116 / 126  136 / 155
//  16384     376 / 390   418 / 461  441 / 478  521 / 590
struct TileForm {
    int rows, cols;
    float alone[2], share[2], once[2];                         // [input's gradient]
};
constexpr TileForm TILE_FORMS[] = {{128, 256, {0.44f, 0.66f}, {0.718f, 0.819f}, {4.3f, 1.8f}},
                                   {128, 128, {0.30f, 0.52f}, {0.412f, 0.449f}, {1.4f, 2.2f}},
                                   {64, 128, {0.28f, 0.29f}, {0.209f, 0.223f}, {1.2f, 1.5f}},
                                   {32, 128, {0.29f, 0.37f}, {0.134f, 0.142f}, {0.8f, 0.9f}}};

int tile_form(int64_t rows, int groups, int N, int blocks, bool grad, int adapter_rank)
{
    int best = 0;
    float least = 0.0f;
    for (int i = 0; i < (int)(sizeof(TILE_FORMS) / sizeof(TILE_FORMS[0])); ++i) {
        const TileForm &f = TILE_FORMS[i];
        const float adapters = (float)(f.rows / 32 * ((adapter_rank + 63) / 64));
        const float alone = f.alone[grad] * blocks + f.once[grad] + 0.9f * adapters, share = f.share[grad] * blocks + f.once[grad] + 0.3f * adapters;
        // (of several groups, the last tile of each is half full on average)
        const float used = (float)(rows < groups ? rows : groups);
        const float down = groups > 1 ? (float)rows / f.rows + 0.5f * used : (float)((rows + f.rows - 1) / f.rows);
        const float tiles = down * (float)((N + f.cols - 1) / f.cols);
        const float turns = ceilf(tiles / 256.0f), full = turns * share > alone ? turns * share : alone;
        const float time = alone + (full - alone) * tiles / (256.0f * turns);
        if (i == 0 || time < least) {
            best = i;
            least = time;
        }
    }
    return best;
}

template <class T, bool GRAD, int ADAPT>
int launch_rows(RowsArgs p, hipStream_t s)
{
    // Few rows: as long as there are not many workgroups of 16 rows x 64 columns.  Outputs / input gradients in us, so and in tiles: 4096 -> 4096, 64
    // rows 8.1 / 8.6 and 18.5 / 19.9, 256 rows (1024 workgroups) 19.2 / 17.1 and 18.9 / 20.2, 320 rows 21.5 / 19.9 and 18.8 / 20.2; 2048 -> 2048, 384 rows
    // (768) 9.7 / 9.1 and 9.9 / 11.8, 640 rows (1280) 13.4 / 12.2 and 12.3 / 11.9; 60 groups 1032 -> 1416, 1537 rows 20.1 / 19.7 and 11.5 / 14.4.
    const int64_t used = p.rows < p.groups ? p.rows : p.groups, tiles = (p.rows + used * 15) / 16;
    if (tiles * ((p.N + 63) / 64) <= (GRAD ? 1280 : 896)) {
        // Narrower ones where they would leave CUs idle (of several groups, some 0.6 tiles end in each).  Outputs / input gradients in workgroups of 16, 32 and
        // 64 columns: 4096 -> 4096, 16 rows 5.0 / 5.1, 5.4 / 5.3, 7.2 / 7.1; 48 rows (768 of the narrowest) 8.5 / 9.5, 7.5 / 7.9, 7.3 / 7.1; 100 rows
        // (1792) 14.1 / 16.8, 10.9 / 11.7, 10.6 / 9.9; 32 rows of 32 groups 2048 -> 1024 7.7, 6.5, 7.0.
        const float ends = p.groups > 1 ? p.rows / 16.0f + 0.6f * (float)used : (float)tiles;
        const float narrow = ends * (float)((p.N + 15) / 16);
        if (narrow <= 256.0f) return launch_few<T, GRAD, ADAPT, 1>(p, s);
        if (narrow <= (GRAD ? 640.0f : 1500.0f)) return launch_few<T, GRAD, ADAPT, 2>(p, s);
        return launch_few<T, GRAD, ADAPT, 4>(p, s);
    }
    switch (tile_form(p.rows, p.groups, p.N, p.kbs, GRAD, ADAPT ? p.ad.rank : 0)) {
    case 0: return launch_tiles<T, GRAD, ADAPT, 128, 256, 128, 64, 4, false>(p, s);
    case 1: return launch_tiles<T, GRAD, ADAPT, 128, 128, 128, 32, 4, false>(p, s);
    case 2: return launch_tiles<T, GRAD, ADAPT, 64, 128, 64, 32, 4, true>(p, s);
    default: return launch_tiles<T, GRAD, ADAPT, 32, 128, 32, 32, 4, !GRAD>(p, s);
    }
}

template <class T>
int launch_typed(const RowsArgs &p, bool grad, hipStream_t s)
{
    if (p.ad.up) return grad ? launch_rows<T, true, GIVEN>(p, s) : launch_rows<T, false, GIVEN>(p, s);
    return grad ? launch_rows<T, true, NONE>(p, s) : launch_rows<T, false, NONE>(p, s);
}

RowsArgs rows_args(const LinearGeom &g, bool grad, const void *in, int64_t ld_in, int64_t rows, const int32_t *offsets, const void *weights, void *out,
                   int64_t ld_out)
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
    return p;
}

}  // namespace

int launch_linear_rows(const LinearGeom &g, bool grad, const void *in, int64_t ld_in, int64_t rows, const int32_t *offsets,
                       const void *weights, void *out, int64_t ld_out, const Adapters *ad, const void *up, const float *low, hipStream_t s)
{
    RowsArgs p = rows_args(g, grad, in, ld_in, rows, offsets, weights, out, ld_out);
    if (ad) p.ad = {up, low, ad->of_row, ad->n, ad->rank, nullptr, nullptr, nullptr};
    return g.dtype == SNN_DTYPE_BF16 ? launch_typed<__bf16>(p, grad, s) : launch_typed<_Float16>(p, grad, s);
}

bool adapters_in_one_launch(const LinearGeom &g, int64_t rows, int rank)
{
    return rows > 0 && rows <= 16 && g.C_out <= 4096 && rows * rank <= OWN_DOTS && rows * rank * g.C_in <= OWN_PRODUCTS;
}

int launch_adapters_in_one(const LinearGeom &g, const Adapters &ad, const void *x, int64_t ldx, int64_t rows, const void *weights, void *y, int64_t ldy,
                           float *low, hipStream_t s)
{
    RowsArgs p = rows_args(g, false, x, ldx, rows, nullptr, weights, y, ldy);
    p.ad = {ad.B, nullptr, ad.of_row, ad.n, ad.rank, ad.A, ad.scale, low};
    return g.dtype == SNN_DTYPE_BF16 ? launch_few<__bf16, false, OWN, 1>(p, s) : launch_few<_Float16, false, OWN, 1>(p, s);
}

}  // namespace snn
