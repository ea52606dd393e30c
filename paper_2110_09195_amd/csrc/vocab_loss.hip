// Losses of rows over a vocabulary and their gradients, in pieces of the vocabulary: no logits are kept.  The products are in vocab_tiles.hip.
#include "linear_device.h"
#include "vocab_loss.h"

#include <math.h>

namespace snn {

namespace {

constexpr float LOG2E = 1.44269504088896f, LN2 = 0.693147180559945f;

// ---- which rows count --------------------------------------------------------------------------------------------
// A row counts when its target is a token; with a teacher, when one of the row's listed tokens is one and has a logit above -infinity; and for the
// gradients, when its loss's gradient is not zero.  The others take no part in any product, whatever they hold.

__device__ inline bool listed(int id, int V) { return (uint32_t)id < (uint32_t)V; }

// One wave: a row with a teacher.
__device__ inline bool row_counts(const Targets &t, int V, int64_t row, int lane)
{
    bool some = false;
    for (int k = lane; k < t.k; k += 64) some |= listed(t.ids[row * t.k + k], V) && !(t.logits[row * t.k + k] == -INFINITY);
    return __any(some);
}

// Flags of rows with a teacher, a wave each; and the outputs of what does not count.
__global__ __launch_bounds__(256)
void loss_flags_kernel(Targets t, int V, int rows, uint8_t *__restrict__ flags, float *__restrict__ loss, float *__restrict__ lse, float *__restrict__ picked)
{
    const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    const bool counts = row_counts(t, V, row, lane);
    if (lane == 0) flags[row] = counts;
    if (!picked) return;
    if (!counts && lane == 0) loss[row] = lse[row] = 0.0f;
    for (int k = lane; k < t.k; k += 64)
        if (!counts || !listed(t.ids[(int64_t)row * t.k + k], V)) picked[(int64_t)row * t.k + k] = 0.0f;
}

// The rows that count, in their order, and each row's place among them (-1: none).  One workgroup.  flags = nullptr: by the targets.
__global__ __launch_bounds__(1024)
void loss_list_kernel(const int32_t *__restrict__ ids, const uint8_t *__restrict__ flags, const float *__restrict__ g, float temperature, int rows, int V,
                      bool scaled, LossHead *__restrict__ head, int *__restrict__ list, int *__restrict__ place, float *__restrict__ loss, float *__restrict__ lse)
{
    __shared__ int waves[16];
    __shared__ float tops[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int before = 0;
    float top = 0.0f;
    for (int r0 = 0; r0 < rows; r0 += 1024) {
        const int r = r0 + threadIdx.x;
        bool counts = r < rows && (flags ? flags[r] != 0 : listed(ids[r], V));
        if (g && counts) {
            const float v = g[r] / temperature;
            counts = v != 0.0f;
            if (fabsf(v) < INFINITY) top = fmaxf(top, fabsf(v));
        }
        const uint64_t all = __ballot(counts);
        if (lane == 0) waves[wave] = __popcll(all);
        __syncthreads();
        int at = before + __popcll(all & ((1ull << lane) - 1)), sum = 0;
#pragma unroll
        for (int w = 0; w < 16; ++w) {
            at += w < wave ? waves[w] : 0;
            sum += waves[w];
        }
        before += sum;
        if (r < rows) place[r] = counts ? at : -1;
        if (counts) list[at] = r;
        else if (loss && !flags && r < rows) loss[r] = lse[r] = 0.0f;
        __syncthreads();
    }
    top = wave_top(top);
    if (lane == 0) tops[wave] = top;
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < 16; ++w) top = fmaxf(top, tops[w]);
    // (values of f16 reach from 2^-24 to 2^16: the largest gradient is brought to 2^14 .. 2^15; bf16 has fp32's range)
    const int e = scaled ? piece_exponent(top) : 0;
    head->count = before;
    head->up = power_of_two(e);
    head->down = power_of_two(-e);
}

struct GatherArgs {
    Targets t;
    const void *x;
    int64_t ldx;
    int rows, V, C;
    const LossHead *head;
    const int *place;
    void *xc;
    int32_t *ids;                     // [k][ld]
    float *q;                         // [k][ld], or nullptr
    int64_t ld;
    const float *lse, *g;             // nullptr: forward
    float *lse2, *gc;
    void *dx;                         // rows of zeros for what does not count; nullptr: not wanted
    int64_t lddx;
};

// Rows that count next to each other, with what belongs to them.  A wave a row.
template <class T>
__global__ __launch_bounds__(256)
void loss_gather_kernel(GatherArgs p)
{
    using v8 = typename Half<T>::v8;
    const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= p.rows) return;
    const int at = __builtin_amdgcn_readfirstlane(p.place[row]);
    if (at < 0) {
        if (p.dx)
            for (int c = lane * 8; c < p.C; c += 512) *(v8 *)((T *)p.dx + (int64_t)row * p.lddx + c) = v8{};
        return;
    }
    const T *const from = (const T *)p.x + (int64_t)row * p.ldx;
    T *const to = (T *)p.xc + (int64_t)at * p.C;
#pragma unroll 4
    for (int c = lane * 8; c < p.C; c += 512) *(v8 *)(to + c) = *(const v8 *)(from + c);
    if (p.g && lane == 0) {
        p.lse2[at] = p.lse[row] * LOG2E;
        p.gc[at] = p.g[row] / p.t.temperature * p.head->up;
    }
    if (!p.t.logits) {
        if (lane == 0) p.ids[at] = p.t.ids[row];
        return;
    }
    float top = -INFINITY, sum = 0.0f;
    const int32_t *const ids = p.t.ids + (int64_t)row * p.t.k;
    const float *const logits = p.t.logits + (int64_t)row * p.t.k;
    if (p.q) {
        for (int k = lane; k < p.t.k; k += 64)
            if (listed(ids[k], p.V)) top = fmaxf(top, logits[k] / p.t.temperature);
#pragma unroll
        for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
        for (int k = lane; k < p.t.k; k += 64)
            if (listed(ids[k], p.V)) sum += expf(logits[k] / p.t.temperature - top);
#pragma unroll
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    }
    for (int k = lane; k < p.t.k; k += 64) {
        const bool in = listed(ids[k], p.V);
        p.ids[k * p.ld + at] = in ? ids[k] : -1;
        if (p.q) p.q[k * p.ld + at] = in ? expf(logits[k] / p.t.temperature - top) / sum : 0.0f;
    }
}

// ---- from tiles to rows --------------------------------------------------------------------------------------------

struct JoinArgs {
    Targets t;
    int rows, V;
    const LossHead *head;             // nullptr: all rows, of which some may not count
    const int *list;
    const float2 *part;
    int64_t part_ld;
    int tiles;
    float c;
    const float *pick;                // of targets, by place
    float *loss, *lse, *picked;
};

__device__ inline void join(float &m, float &s, float m2, float s2)
{
    const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.0f : top;
    s = s * __builtin_amdgcn_exp2f(m - base) + s2 * __builtin_amdgcn_exp2f(m2 - base);
    m = top;
}

// Sums of exponentials of RT rows from those of the tiles, and their losses.  The loss is formed from what the row's logits fall short of the largest
// one, not from the sum's logarithm as a whole: small losses keep their digits.
template <int RT>
__global__ __launch_bounds__(256)
void loss_join_kernel(JoinArgs p)
{
    constexpr int SLICES = 256 / RT;
    __shared__ float2 stat[SLICES][RT];
    const int tid = threadIdx.x, rt = tid % RT, slice = tid / RT;
    const int rows = p.head ? p.head->count : p.rows, t0 = blockIdx.x * RT;
    if (t0 >= rows) return;
    float m = -INFINITY, s = 0.0f;
    if (t0 + rt < rows) {
        constexpr int N = 8;
        for (int i0 = slice; i0 < p.tiles; i0 += N * SLICES) {
            float2 v[N];
#pragma unroll
            for (int n = 0; n < N; ++n)
                v[n] = i0 + n * SLICES < p.tiles ? p.part[(i0 + n * SLICES) * p.part_ld + t0 + rt] : make_float2(-INFINITY, 0.0f);
#pragma unroll
            for (int n = 0; n < N; ++n) join(m, s, v[n].x, v[n].y);
        }
    }
    stat[slice][rt] = make_float2(m, s);
    for (int half = SLICES / 2; half; half >>= 1) {
        __syncthreads();
        if (slice < half) {
            join(m, s, stat[slice + half][rt].x, stat[slice + half][rt].y);
            stat[slice][rt] = make_float2(m, s);
        }
    }
    __syncthreads();
    if (!p.t.logits) {
        if (tid >= RT || t0 + tid >= rows) return;
        const int t = t0 + tid, row = p.list ? p.list[t] : t;
        m = stat[0][tid].x;
        s = log2f(stat[0][tid].y);
        const bool counts = listed(p.t.ids[row], p.V);
        p.lse[row] = counts ? LN2 * (m + s) : 0.0f;
        p.loss[row] = counts ? LN2 * (s - fmaf(p.pick[t], p.c, -m)) : 0.0f;
        return;
    }
    const int lane = tid & 63;
    for (int r = tid >> 6; r < RT && t0 + r < rows; r += 4) {
        const int t = t0 + r;
        const int64_t row = p.list ? p.list[t] : t;
        const bool counts = p.list || row_counts(p.t, p.V, row, lane);
        const int32_t *const ids = p.t.ids + row * p.t.k;
        const float *const logits = p.t.logits + row * p.t.k;
        float *const picked = p.picked + row * p.t.k;
        if (!p.list)
            for (int k = lane; k < p.t.k; k += 64)
                if (!counts || !listed(ids[k], p.V)) picked[k] = 0.0f;
        if (!counts) {
            if (lane == 0) p.loss[row] = p.lse[row] = 0.0f;
            continue;
        }
        m = stat[0][r].x;
        s = log2f(stat[0][r].y);
        float top = -INFINITY, sum = 0.0f, far = 0.0f;
        for (int k = lane; k < p.t.k; k += 64)
            if (listed(ids[k], p.V)) top = fmaxf(top, logits[k] / p.t.temperature);
#pragma unroll
        for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
        for (int k = lane; k < p.t.k; k += 64)
            if (listed(ids[k], p.V)) sum += expf(logits[k] / p.t.temperature - top);
#pragma unroll
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
        const float all = log2f(sum);
        for (int k = lane; k < p.t.k; k += 64)
            if (listed(ids[k], p.V)) {
                const float d = logits[k] / p.t.temperature - top, q = expf(d) / sum;
                // (a share of zero counts for nothing, whatever the row's logit)
                if (!(q == 0.0f)) far += q * ((d * LOG2E - all) + (s - fmaf(picked[k], p.c, -m)));
            }
#pragma unroll
        for (int d = 32; d; d >>= 1) far += __shfl_xor(far, d);
        if (lane == 0) {
            p.lse[row] = LN2 * (m + s);
            p.loss[row] = LN2 * far;
        }
    }
}

// Gradients of rows from their parts: a wave a row.
template <class T>
__global__ __launch_bounds__(256)
void loss_rows_kernel(const float *__restrict__ part, int64_t split, int C, int tile_m, int tile_n, int steps, int most, const LossHead *__restrict__ head,
                      const int *__restrict__ list, T *__restrict__ dx, int64_t lddx)
{
    using v8 = typename Half<T>::v8;
    const int lane = threadIdx.x & 63, t = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), count = head->count;
    if (t >= count) return;
    const int splits = row_splits((C + tile_m - 1) / tile_m * ((count + tile_n - 1) / tile_n), steps, most);
    const float down = head->down;
    T *const to = dx + (int64_t)list[t] * lddx;
    for (int c = lane * 8; c < C; c += 512) {
        float sum[8] = {};
#pragma unroll 4
        for (int s = 0; s < splits; ++s) {
            const float *const from = part + s * split + (int64_t)t * C + c;
            const f32x4 a = *(const f32x4 *)from, b = *(const f32x4 *)(from + 4);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                sum[k] += a[k];
                sum[4 + k] += b[k];
            }
        }
        v8 v;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = (T)(sum[k] * down);
        *(v8 *)(to + c) = v;
    }
}

// ---- plans -------------------------------------------------------------------------------------------------------

// What a piece of the vocabulary may hold of probabilities, in bytes (at least 256 tokens are a piece, at most all)
constexpr size_t PIECE_BYTES = (size_t)512 << 20;
// and the parts of the rows' gradients beyond the first
constexpr size_t PARTS_BYTES = (size_t)64 << 20;

struct LossPlan {
    bool gather;                      // rows that count are copied next to each other
    int form, form_rows, form_table;
    int64_t ld;                       // rows, in whole blocks of 64
    int tiles;                        // of the vocabulary (forward)
    int piece, most_splits;
    size_t list, place, flags, pick, ids, q, lse2, g, xc, part, probs, out, bytes;
};

int form_of(int64_t m, int64_t n, int64_t enough)
{
    return (m + 255) / 256 * ((n + 255) / 256) >= enough && n > 128 && m > 128 ? TILE_256 : TILE_128;
}

LossPlan loss_plan(const Vocab &v, int64_t rows, int k, bool backward)
{
    LossPlan p = {};
    p.ld = (rows + 63) / 64 * 64;
    // (two launches and a copy pay where the product takes longer than some 50 us)
    p.gather = backward || (rows > 256 && (double)rows * v.V * v.C > 3e10);
    size_t at = 256;                                           // the head
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += align_up(bytes, 256);
        return here;
    };
    if (p.gather) {
        p.list = take(p.ld * 4);
        p.place = take(p.ld * 4);
        p.flags = take(p.ld);
        p.ids = take((size_t)k * p.ld * 4);
        p.xc = take((size_t)rows * v.C * 2);
    }
    if (!backward) {
        p.form = rows <= 64 ? TILE_FEW : form_of(v.V, rows, 200);
        p.tiles = (v.V + tile_m(p.form) - 1) / tile_m(p.form);
        p.pick = take(p.ld * 4);
        p.part = take((size_t)p.tiles * p.ld * 8);
    } else {
        const size_t all = ((size_t)v.V + 255) / 256, most = PIECE_BYTES / 512 / (size_t)(p.ld ? p.ld : 64);
        const size_t pieces = most < 1 ? all : (all + most - 1) / most;
        p.piece = (int)((all + pieces - 1) / pieces * 256);
        p.form = form_of(p.piece, rows, 200);
        p.form_rows = form_of(v.C, rows, 1);
        p.form_table = form_of(v.C, p.piece, 200);
        const size_t part = (size_t)rows * v.C * 4;
        p.most_splits = (int)(part * 64 <= PARTS_BYTES ? 64 : part * 2 > PARTS_BYTES ? 1 : PARTS_BYTES / part);
        p.q = take((size_t)k * p.ld * 4);
        p.lse2 = take(p.ld * 4);
        p.g = take(p.ld * 4);
        p.probs = take((size_t)p.ld * p.piece * 2);
        p.out = take(part * p.most_splits);
    }
    p.bytes = at;
    return p;
}

// The rows that count, their number and the gradients' scale, and what belongs to them.
int launch_rows(const Vocab &v, const LossPlan &plan, const Rows16 &x, int64_t rows, const Targets &t, const float *lse, const float *dloss, void *dx,
                int64_t lddx, float *loss, float *lse_out, float *picked, char *ws, hipStream_t s)
{
    uint8_t *const flags = t.logits ? (uint8_t *)(ws + plan.flags) : nullptr;
    LossHead *const head = (LossHead *)ws;
    int *const list = (int *)(ws + plan.list), *const place = (int *)(ws + plan.place);
    const unsigned blocks = (unsigned)((rows + 3) / 4);
    if (flags && rows) loss_flags_kernel<<<dim3(blocks), 256, 0, s>>>(t, v.V, (int)rows, flags, loss, lse_out, picked);
    loss_list_kernel<<<1, 1024, 0, s>>>(t.ids, flags, dloss, t.temperature, (int)rows, v.V, dloss && v.dtype == SNN_DTYPE_F16, head, list, place, loss,
                                          lse_out);
    if (rows) {
        GatherArgs g = {};
        g.t = t; g.x = x.p; g.ldx = x.ld; g.rows = (int)rows; g.V = v.V; g.C = v.C; g.head = head; g.place = place;
        g.xc = ws + plan.xc; g.ids = (int32_t *)(ws + plan.ids); g.ld = plan.ld;
        if (dloss) {
            g.q = (float *)(ws + plan.q);
            g.lse = lse; g.g = dloss; g.lse2 = (float *)(ws + plan.lse2); g.gc = (float *)(ws + plan.g);
            g.dx = dx; g.lddx = lddx;
        }
        if (v.dtype == SNN_DTYPE_BF16) loss_gather_kernel<__bf16><<<dim3(blocks), 256, 0, s>>>(g);
        else loss_gather_kernel<_Float16><<<dim3(blocks), 256, 0, s>>>(g);
    }
    return check_launch();
}

}  // namespace

size_t loss_workspace_bytes(const Vocab &v, int64_t rows, int k, bool backward) { return loss_plan(v, rows, k, backward).bytes; }

int launch_loss_forward(const Vocab &v, const Rows16 &x, int64_t rows, const Rows16 &table, const Targets &t, float *loss, float *lse, float *picked,
                        void *workspace, hipStream_t s)
{
    const LossPlan plan = loss_plan(v, rows, t.k, false);
    char *const ws = (char *)workspace;
    TilesArgs p = {};
    p.a = table.p; p.lda = table.ld; p.M = v.V;
    p.b = x.p; p.ldb = x.ld; p.N = (int)rows; p.K = v.C;
    p.c = LOG2E / t.temperature;
    p.ids = t.ids; p.id_row = t.k; p.id_k = 1; p.k = t.k;
    if (plan.gather) {
        const int rc = launch_rows(v, plan, x, rows, t, nullptr, nullptr, nullptr, 0, loss, lse, picked, ws, s);
        if (rc != SNN_OK) return rc;
        p.head = (const LossHead *)ws;
        p.b = ws + plan.xc; p.ldb = v.C;
        p.ids = (const int32_t *)(ws + plan.ids); p.id_row = 1; p.id_k = plan.ld;
    }
    const int *const list = plan.gather ? (const int *)(ws + plan.list) : nullptr;
    p.part = (float2 *)(ws + plan.part); p.part_ld = plan.ld;
    // (targets' logits stay in the workspace, by place)
    p.picked = t.logits ? picked : (float *)(ws + plan.pick);
    p.list = t.logits ? list : nullptr;
    const int rc = launch_vocab_tiles(STATS, plan.form, v.dtype, p, s);
    if (rc != SNN_OK) return rc;
    JoinArgs j = {};
    j.t = t; j.rows = (int)rows; j.V = v.V; j.head = p.head; j.list = list;
    j.part = p.part; j.part_ld = p.part_ld; j.tiles = plan.tiles; j.c = p.c;
    j.pick = (const float *)(ws + plan.pick);
    j.loss = loss; j.lse = lse; j.picked = picked;
    if (rows <= 256) loss_join_kernel<1><<<dim3((unsigned)rows), 256, 0, s>>>(j);
    else loss_join_kernel<32><<<dim3((unsigned)((rows + 31) / 32)), 256, 0, s>>>(j);
    return check_launch();
}

int launch_loss_backward(const Vocab &v, const Rows16 &x, int64_t rows, const Rows16 &table, const Targets &t, const float *lse, const float *dloss,
                         void *dx, int64_t lddx, void *dtable, bool accumulate, void *workspace, hipStream_t s)
{
    const LossPlan plan = loss_plan(v, rows, t.k, true);
    char *const ws = (char *)workspace;
    int rc = launch_rows(v, plan, x, rows, t, lse, dloss, dx, lddx, nullptr, nullptr, nullptr, ws, s);
    if (rc != SNN_OK) return rc;
    const int64_t split = (int64_t)rows * v.C;
    const int most = plan.most_splits;
    int steps = 0;
    for (int64_t v0 = 0; v0 < v.V; v0 += plan.piece) {
        const int n = (int)(v.V - v0 < plan.piece ? v.V - v0 : plan.piece);
        const char *const rows_of_piece = (const char *)table.p + v0 * table.ld * 2;
        TilesArgs p = {};
        p.head = (const LossHead *)ws;
        p.a = rows_of_piece; p.lda = table.ld; p.M = n;
        p.b = ws + plan.xc; p.ldb = v.C; p.N = (int)rows; p.K = v.C;
        p.c = LOG2E / t.temperature;
        p.v0 = (int)v0;
        p.ids = (const int32_t *)(ws + plan.ids); p.id_row = 1; p.id_k = plan.ld; p.k = t.k;
        p.q = t.logits ? (const float *)(ws + plan.q) : nullptr;
        p.lse2 = (const float *)(ws + plan.lse2); p.g = (const float *)(ws + plan.g);
        p.probs = ws + plan.probs; p.ldp = plan.piece;
        if ((rc = launch_vocab_tiles(PROBS, plan.form, v.dtype, p, s)) != SNN_OK) return rc;
        if (dx) {
            TilesArgs r = {};
            r.head = p.head;
            r.a = rows_of_piece; r.lda = table.ld; r.M = v.C;
            r.b = p.probs; r.ldb = p.ldp; r.N = (int)rows; r.K = n;
            r.out = (float *)(ws + plan.out); r.out_split = split; r.most_splits = most; r.add = v0 > 0;
            // (the number of parts is the first piece's in all of them: a shorter last piece leaves some empty)
            if (v0 == 0) steps = (n + 31) / 32;
            r.steps = steps;
            if ((rc = launch_vocab_tiles(ROWS, plan.form_rows, v.dtype, r, s)) != SNN_OK) return rc;
        }
        if (dtable) {
            TilesArgs w = {};
            w.head = p.head;
            w.a = p.b; w.lda = v.C; w.M = v.C;
            w.b = p.probs; w.ldb = p.ldp; w.N = n; w.K = (int)rows;
            w.v0 = (int)v0; w.dtable = dtable; w.accumulate = accumulate;
            if ((rc = launch_vocab_tiles(TABLE, plan.form_table, v.dtype, w, s)) != SNN_OK) return rc;
        }
    }
    if (!dx || rows == 0) return SNN_OK;
    const unsigned blocks = (unsigned)((rows + 3) / 4);
    const int tm = tile_m(plan.form_rows), tn = tile_n(plan.form_rows);
    const LossHead *const head = (const LossHead *)ws;
    const int *const list = (const int *)(ws + plan.list);
    if (v.dtype == SNN_DTYPE_BF16)
        loss_rows_kernel<__bf16><<<dim3(blocks), 256, 0, s>>>((const float *)(ws + plan.out), split, v.C, tm, tn, steps, most, head, list, (__bf16 *)dx, lddx);
    else
        loss_rows_kernel<_Float16><<<dim3(blocks), 256, 0, s>>>((const float *)(ws + plan.out), split, v.C, tm, tn, steps, most, head, list, (_Float16 *)dx,
                                                                lddx);
    return check_launch();
}

}  // namespace snn
