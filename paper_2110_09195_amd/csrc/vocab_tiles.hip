// The products of the losses over a vocabulary: one tile kernel with four endings.
#include "linear_device.h"
#include "vocab_loss.h"

#include <math.h>

namespace snn {

namespace {

// An operand whose contracted axis lies along memory: R rows of 32 of it a step, 64 bytes a row in LDS, their 16-byte pieces xor-ed by a quarter of the
// row's number, so that sixteen rows read at once lie in sixteen different places of the banks.
template <int R, int THREADS, bool TURNED>
struct Operand {
    static constexpr int L = R * 4 / THREADS, BYTES = R * 64;
    static_assert(L * THREADS == R * 4, "whole loads");
    s32x4 from;
    uint32_t offset[L];
    int k, piece, width;

    // `width` of the axis count; what lies behind gives zeros
    __device__ void begin(const void *p, int64_t ld, int row0, int rows, int width_, int k0)
    {
        const int tid = threadIdx.x, left = min(rows - row0, R);
        from = resource((const char *)p + (int64_t)row0 * ld * 2, left > 0 ? (uint32_t)(left - 1) * (uint32_t)(ld * 2) + (uint32_t)width_ * 2 : 0);
        width = width_;
        k = k0;
        piece = (tid & 3) ^ ((tid >> 4) & 3);
#pragma unroll
        for (int i = 0; i < L; ++i) offset[i] = (uint32_t)(tid / 4 + i * (THREADS / 4)) * (uint32_t)(ld * 2) + piece * 16;
    }
    __device__ void issue(uint32_t lds, int wave)
    {
        const bool in = k + piece * 8 < width;
#pragma unroll
        for (int i = 0; i < L; ++i) load_lds16(lds + i * THREADS * 16 + wave * 1024, in ? offset[i] + (uint32_t)k * 2 : NOWHERE, from);
        k += 32;
    }
    static __device__ uint32_t at(int row0, int lane)
    {
        return (uint32_t)(row0 + (lane & 31)) * 64 + (((lane >> 5) ^ ((lane >> 2) & 3)) << 4);
    }
    // eight values of 16 s .. 16 s + 15 of the step
    template <class T>
    static __device__ typename Half<T>::v8 read(const char *base, uint32_t at, int s)
    {
        return *(const typename Half<T>::v8 *)(base + (at ^ (uint32_t)(s << 5)));
    }
};

// An operand whose contracted axis lies across memory: 32 of its rows a step, R columns each; 32-byte pieces xor-ed with the row's low two bits, fragments
// turned by the reads that fetch them.
template <int R, int THREADS>
struct Operand<R, THREADS, true> {
    static constexpr int P = R / 8, L = 32 * P / THREADS, BYTES = R * 64;
    static_assert(L * THREADS == 32 * P && THREADS % P == 0, "whole loads");
    const char *from;
    uint32_t offset[L];
    int left, row_bytes, gap;

    // `cols` columns; rows k0 .. rows - 1 of the axis count, what lies behind gives zeros
    __device__ void begin(const void *p, int64_t ld, int col0, int cols, int rows, int k0)
    {
        row_bytes = (int)ld * 2;
        gap = row_bytes - (cols - col0) * 2;
        left = rows - k0;
        from = (const char *)p + ((int64_t)k0 * ld + col0) * 2;
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const int r = (i * THREADS + (int)threadIdx.x) / P, c = threadIdx.x % P;
            offset[i] = (uint32_t)r * (uint32_t)row_bytes + ((((c >> 1) ^ ((r & 3) << 1)) << 1) | (c & 1)) * 16;
        }
    }
    __device__ void issue(uint32_t lds, int wave)
    {
        const s32x4 r = resource(from, (uint32_t)max(min(max(left, 0), 32) * row_bytes - gap, 0));
#pragma unroll
        for (int i = 0; i < L; ++i) load_lds16(lds + i * THREADS * 16 + wave * 1024, offset[i], r);
        from += 32 * (int64_t)row_bytes;
        left -= 32;
    }
    static __device__ uint32_t at(int col0, int lane)
    {
        const int q = lane >> 4, rr = (lane & 15) >> 2, h = lane >> 5;
        return (8 * h + rr) * (R * 2) + (((2 * (col0 / 32) + (q & 1)) ^ (rr << 1)) * 32) + (lane & 3) * 8;
    }
    template <class T>
    static __device__ typename Half<T>::v8 read(const char *base, uint32_t at, int s)
    {
        return read_turned<T>(base + at + s * 16 * (R * 2), 4 * (R * 2));
    }
};

// The tile of a workgroup: groups of eight tiles of rows, within a group the columns' tiles, the group's eight innermost; XCDs (workgroups in
// turn) take runs of that order, so that what an XCD works on at one time reads few different operands.
struct Place {
    int m, n, split;
};

__device__ inline bool find_place(int tm, int tn, int splits, Place &at)
{
    const uint32_t each = (uint32_t)tm * tn, total = each * splits, share = (total + 7) / 8, turn = blockIdx.x >> 3;
    const uint32_t id = (blockIdx.x & 7) * share + turn;
    if (turn >= share || id >= total) return false;
    at.split = id / each;
    const uint32_t r = id - at.split * each, group = r / (8 * tn), first = group * 8, rest = r - first * tn;
    const uint32_t wide = min(8u, (uint32_t)tm - first);
    at.n = rest / wide;
    at.m = first + (rest - at.n * wide);
    return true;
}

// D[m][n] over 32 of the contracted axis at a time.  Tiles go to LDS as they lie, without registers, STAGES in flight; while the products of
// 16 run, the fragments of the next 16 are read, in the shadow of the matrix instructions.
template <class T, int KIND, int BM, int BN, int WM, int WN, int STAGES>
__global__ __launch_bounds__(64 * (BM / WM) * (BN / WN))
void vocab_tiles_kernel(TilesArgs p)
{
    using H = Half<T>;
    using v8 = typename H::v8;
    constexpr int WAVES_M = BM / WM, WAVES = WAVES_M * (BN / WN), THREADS = 64 * WAVES;
    constexpr int MB = WM / 32, NB = WN / 32;
    using A = Operand<BM, THREADS, KIND == ROWS || KIND == TABLE>;
    using B = Operand<BN, THREADS, KIND == TABLE>;
    constexpr int STAGE = A::BYTES + B::BYTES, LOADS = A::L + B::L;
    extern __shared__ __align__(16) char lds[];

    const int count = p.head ? __builtin_amdgcn_readfirstlane(p.head->count) : KIND == TABLE ? p.K : p.N;
    const int N = KIND == TABLE ? p.N : count, K = KIND == TABLE ? count : p.K;
    const int tm = (p.M + BM - 1) / BM, tn = (N + BN - 1) / BN;
    int steps = (K + 31) / 32;
    const int splits = KIND == ROWS ? row_splits(tm * tn, p.steps, p.most_splits) : 1;
    Place at;
    if (!find_place(tm, tn, splits, at)) return;
    int first = 0;
    if constexpr (KIND == ROWS) {
        const int run = (steps + splits - 1) / splits;
        first = at.split * run;
        steps = max(min(steps - first, run), 0);
    }
    const int m0 = at.m * BM, n0 = at.n * BN;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave % WAVES_M, wn = wave / WAVES_M;
    const uint32_t lds0 = lds_address(lds);

    A a;
    B b;
    if constexpr (KIND == ROWS || KIND == TABLE) a.begin(p.a, p.lda, m0, p.M, K, first * 32);
    else a.begin(p.a, p.lda, m0, p.M, K, 0);
    // (probabilities are zeros behind the piece's last token: whole loads of them)
    if constexpr (KIND == TABLE) b.begin(p.b, p.ldb, n0, (N + 7) & ~7, K, 0);
    else if constexpr (KIND == ROWS) b.begin(p.b, p.ldb, n0, N, (K + 31) & ~31, first * 32);
    else b.begin(p.b, p.ldb, n0, N, K, 0);
    auto issue = [&](int slot, int part) {
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds0 + slot * STAGE);
        if (part == 0) a.issue(to, wave);
        else b.issue(to + A::BYTES, wave);
    };

    f32x16 acc[MB][NB] = {};
    uint32_t am[MB], bn[NB];
#pragma unroll
    for (int i = 0; i < MB; ++i) am[i] = A::at(wm * WM + i * 32, lane);
#pragma unroll
    for (int i = 0; i < NB; ++i) bn[i] = B::at(wn * WN + i * 32, lane);
    v8 x[2][MB], y[2][NB];
    auto read = [&](const char *base, int s, int to) {
#pragma unroll
        for (int i = 0; i < MB; ++i) x[to][i] = A::template read<T>(base, am[i], s);
#pragma unroll
        for (int i = 0; i < NB; ++i) y[to][i] = B::template read<T>(base + A::BYTES, bn[i], s);
    };
    auto multiply = [&](int from) {
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = H::mfma(x[from][i], y[from][j], acc[i][j]);
#pragma unroll
        for (int i = 0; i < MB * NB; ++i) {
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
        const char *here = lds + slot * STAGE;
        const int free = slot == 0 ? STAGES - 1 : slot - 1;
        slot = slot == STAGES - 1 ? 0 : slot + 1;
        issue(free, 0);
        read(here, 1, 1);
        multiply(0);
        issue(free, 1);
        read(lds + slot * STAGE, 0, 0);
        multiply(1);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");

    // Lane: column ln of a block of 32, rows 8 g + 4 h + i of register 4 g + i.
    const int h = lane >> 5, ln = lane & 31;
    if constexpr (KIND == STATS || KIND == PROBS) {
        const int mw = m0 + wm * WM;                           // the wave's first token, of the piece
        const bool edge = mw + WM > p.M;
        float top[NB], sum[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int t = n0 + wn * WN + j * 32 + ln;
            const bool row = t < N;
            float g = 0.0f;
            if constexpr (KIND == PROBS) {
                const float lse2 = row ? p.lse2[t] : 0.0f;
                g = row ? p.g[t] : 0.0f;
#pragma unroll
                for (int i = 0; i < MB; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int v = mw + i * 32 + 8 * (r >> 2) + 4 * h + (r & 3);
                        const float e = __builtin_amdgcn_exp2f(fmaf(acc[i][j][r], p.c, -lse2)) * g;
                        acc[i][j][r] = edge && v >= p.M ? 0.0f : e;
                    }
            } else if (edge)
#pragma unroll
                for (int i = 0; i < MB; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (mw + i * 32 + 8 * (r >> 2) + 4 * h + (r & 3) >= p.M) acc[i][j][r] = -INFINITY;
            // the listed tokens of the row that are among the wave's
            const int most = min(p.M - mw, WM);
            for (int k0 = 0; k0 < p.k; k0 += 8) {
                int local[8];
                bool some = false;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    local[e] = row && k0 + e < p.k ? p.ids[t * p.id_row + (k0 + e) * p.id_k] : -1;
                    local[e] = local[e] < 0 ? -1 : local[e] - p.v0 - mw;
                    some |= (uint32_t)local[e] < (uint32_t)max(most, 0);
                }
                if (!__any(some)) continue;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool hit = (uint32_t)local[e] < (uint32_t)max(most, 0) && ((local[e] >> 2) & 1) == h;
                    if (!__any(hit)) continue;
                    const int mine = hit ? local[e] - 4 * h : -1;
                    if constexpr (KIND == STATS) {
                        float z = 0.0f;
#pragma unroll
                        for (int i = 0; i < MB; ++i)
#pragma unroll
                            for (int r = 0; r < 16; ++r) z = mine == i * 32 + 8 * (r >> 2) + (r & 3) ? acc[i][j][r] : z;
                        if (hit) p.picked[(p.list ? p.list[t] : t) * (int64_t)p.k + k0 + e] = z;
                    } else {
                        const float q = hit ? g * (p.q ? p.q[t * p.id_row + (k0 + e) * p.id_k] : 1.0f) : 0.0f;
#pragma unroll
                        for (int i = 0; i < MB; ++i)
#pragma unroll
                            for (int r = 0; r < 16; ++r) acc[i][j][r] -= mine == i * 32 + 8 * (r >> 2) + (r & 3) ? q : 0.0f;
                    }
                }
            }
            if constexpr (KIND == STATS) {
                float m = -INFINITY, s = 0.0f;
#pragma unroll
                for (int i = 0; i < MB; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) m = fmaxf(m, acc[i][j][r]);
                m = fmaxf(m, __shfl_xor(m, 32)) * p.c;
                const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
                for (int i = 0; i < MB; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s += __builtin_amdgcn_exp2f(fmaf(acc[i][j][r], p.c, -base));
                top[j] = m;
                sum[j] = s + __shfl_xor(s, 32);
            }
        }
        if constexpr (KIND == STATS) {
            float2 *const stat = (float2 *)lds;                // [WAVES_M][BN]
            if (h == 0)
#pragma unroll
                for (int j = 0; j < NB; ++j) stat[wm * BN + wn * WN + j * 32 + ln] = make_float2(top[j], sum[j]);
            __syncthreads();
            if (tid < BN && n0 + tid < N) {
                float m = -INFINITY, s = 0.0f;
#pragma unroll
                for (int i = 0; i < WAVES_M; ++i) m = fmaxf(m, stat[i * BN + tid].x);
                const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
                for (int i = 0; i < WAVES_M; ++i) s += stat[i * BN + tid].y * __builtin_amdgcn_exp2f(stat[i * BN + tid].x - base);
                p.part[at.m * p.part_ld + n0 + tid] = make_float2(m, s);
            }
        } else {
            // through LDS (a wave's own 32 rows) to whole lines
            constexpr int PITCH = WM * 2 + 16, PIECES = WM / 8;
            char *const mine = lds + wave * 32 * PITCH;
#pragma unroll
            for (int j = 0; j < NB; ++j) {
#pragma unroll
                for (int i = 0; i < MB; ++i)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        typename H::v4 v;
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[k] = (T)acc[i][j][4 * g + k];
                        *(typename H::v4 *)(mine + ln * PITCH + (i * 32 + g * 8 + 4 * h) * 2) = v;
                    }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
                for (int i = 0; i < PIECES / 2; ++i) {
                    const int q = i * 64 + lane, r = q / PIECES, c = q % PIECES, t = n0 + wn * WN + j * 32 + r;
                    const u32x4 v = *(const u32x4 *)(mine + r * PITCH + c * 16);
                    if (t < N) *(u32x4 *)((T *)p.probs + (int64_t)t * p.ldp + mw + c * 8) = v;
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            }
        }
    } else {
        constexpr int PITCH = WM * 4 + 16;
        char *const mine = lds + wave * 32 * PITCH;
        const float down = KIND == TABLE ? p.head->down : 1.0f;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int o = n0 + wn * WN + j * 32;
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *(f32x4 *)(mine + ln * PITCH + (i * 32 + 8 * g + 4 * h) * 4) =
                        f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if constexpr (KIND == ROWS) {
                constexpr int PIECES = WM / 4;
#pragma unroll
                for (int i = 0; i < PIECES / 2; ++i) {
                    const int n = i * 64 + lane, r = n / PIECES, c = m0 + wm * WM + n % PIECES * 4;
                    f32x4 v = *(const f32x4 *)(mine + r * PITCH + n % PIECES * 16);
                    if (o + r < N && c < p.M) {
                        f32x4 *const to = (f32x4 *)(p.out + at.split * p.out_split + (int64_t)(o + r) * p.M + c);
                        if (p.add) v += *to;
                        *to = v;
                    }
                }
            } else {
                constexpr int PIECES = WM / 8;
#pragma unroll
                for (int i = 0; i < PIECES / 2; ++i) {
                    const int n = i * 64 + lane, r = n / PIECES, c = m0 + wm * WM + n % PIECES * 8;
                    const f32x4 v[2] = {*(const f32x4 *)(mine + r * PITCH + n % PIECES * 32), *(const f32x4 *)(mine + r * PITCH + n % PIECES * 32 + 16)};
                    if (o + r < N && c < p.M) {
                        v8 *const to = (v8 *)((T *)p.dtable + (int64_t)(p.v0 + o + r) * p.M + c);
                        const v8 had = p.accumulate ? *to : v8{};
                        v8 w;
#pragma unroll
                        for (int k = 0; k < 8; ++k) w[k] = (T)(p.accumulate ? fmaf(v[k >> 2][k & 3], down, (float)had[k]) : v[k >> 2][k & 3] * down);
                        *to = w;
                    }
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
    }
}

template <class T, int KIND, int BM, int BN, int WM, int WN, int STAGES>
int launch_tiles(const TilesArgs &p, hipStream_t s)
{
    constexpr int WAVES = (BM / WM) * (BN / WN);
    constexpr size_t TILES = (size_t)STAGES * (BM + BN) * 64;
    constexpr size_t OUT = KIND == STATS ? (size_t)(BM / WM) * BN * 8 : (size_t)WAVES * 32 * (WM * (KIND == PROBS ? 2 : 4) + 16);
    constexpr size_t LDS = TILES > OUT ? TILES : OUT;
    static_assert(LDS <= 160 * 1024, "LDS");
    static LdsGrant grant;
    const auto kernel = vocab_tiles_kernel<T, KIND, BM, BN, WM, WN, STAGES>;
    const int rc = grant_dynamic_lds((const void *)kernel, LDS, grant);
    if (rc != SNN_OK) return rc;
    const int64_t tiles = (int64_t)((p.M + BM - 1) / BM) * ((p.N + BN - 1) / BN) * (KIND == ROWS ? p.most_splits : 1);
    if (tiles >= ((int64_t)1 << 30)) return SNN_ERR_UNSUPPORTED;
    if (tiles == 0) return SNN_OK;
    kernel<<<dim3((unsigned)((tiles + 7) / 8 * 8)), 64 * WAVES, LDS, s>>>(p);
    return check_launch();
}

template <class T, int KIND>
int launch_form(int form, const TilesArgs &p, hipStream_t s)
{
    if constexpr (KIND == STATS)
        if (form == TILE_FEW) return launch_tiles<T, KIND, 128, 64, 32, 64, 4>(p, s);
    return form == TILE_256 ? launch_tiles<T, KIND, 256, 256, 128, 64, 4>(p, s) : launch_tiles<T, KIND, 128, 128, 64, 64, 4>(p, s);
}

template <class T>
int launch_kind(int kind, int form, const TilesArgs &p, hipStream_t s)
{
    switch (kind) {
    case STATS: return launch_form<T, STATS>(form, p, s);
    case PROBS: return launch_form<T, PROBS>(form, p, s);
    case ROWS: return launch_form<T, ROWS>(form, p, s);
    default: return launch_form<T, TABLE>(form, p, s);
    }
}

}  // namespace

int launch_vocab_tiles(int kind, int form, int dtype, const TilesArgs &p, hipStream_t s)
{
    return dtype == SNN_DTYPE_BF16 ? launch_kind<__bf16>(kind, form, p, s) : launch_kind<_Float16>(kind, form, p, s);
}

}  // namespace snn
