// Device pieces of the projections' kernels: 16-bit operands of the matrix cores, loads from memory into LDS.
#pragma once

#include "linear.h"

namespace snn {

using s32x4 = __attribute__((ext_vector_type(4))) int;
using u32x4 = __attribute__((ext_vector_type(4))) uint32_t;
using u32x2 = __attribute__((ext_vector_type(2))) uint32_t;
using f32x4 = __attribute__((ext_vector_type(4))) float;
using f32x16 = __attribute__((ext_vector_type(16))) float;

template <class T> struct Half;
template <> struct Half<__bf16> {
    using v8 = __attribute__((ext_vector_type(8))) __bf16;
    using v4 = __attribute__((ext_vector_type(4))) __bf16;
    using v2 = __attribute__((ext_vector_type(2))) __bf16;
    static constexpr uint32_t ONES = 0x3f803f80u;              // (1, 1)
    static __device__ f32x16 mfma(v8 a, v8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    static __device__ f32x4 mfma16(v8 a, v8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Half<_Float16> {
    using v8 = __attribute__((ext_vector_type(8))) _Float16;
    using v4 = __attribute__((ext_vector_type(4))) _Float16;
    using v2 = __attribute__((ext_vector_type(2))) _Float16;
    static constexpr uint32_t ONES = 0x3c003c00u;
    static __device__ f32x16 mfma(v8 a, v8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
    static __device__ f32x4 mfma16(v8 a, v8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

// A buffer resource for the loads below: what they load past `bytes` is zeros.  The vector unit writes its registers (readfirstlane), and a vector memory
// instruction may read such a register five wait states later at the earliest.  The compiler knows of its own loads, not of those in
// assembly text, so the wait is part of the resource: nobody gets at the registers before it is over.
__device__ inline s32x4 resource(const void *p, uint32_t bytes)
{
    const uint64_t a = (uint64_t)p;
    s32x4 r;
    r[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)a);
    r[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32));
    r[2] = __builtin_amdgcn_readfirstlane((int)bytes);
    r[3] = 0x00020000;
    asm("s_nop 4" : "+s"(r));
    return r;
}

// The same for the compiler's own loads.
__device__ inline __amdgpu_buffer_rsrc_t buffer(const void *p, uint32_t bytes)
{
    const uint64_t a = (uint64_t)p;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)a), hi = __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32));
    return __builtin_amdgcn_make_buffer_rsrc((void *)((uint64_t)lo | (uint64_t)hi << 32), 0, __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000);
}

__device__ inline uint32_t lds_address(const void *p) { return (uint32_t)(uint64_t)(__attribute__((address_space(3))) const void *)p; }

// Memory to LDS without registers: lane l's 16 (4) bytes go to lds + 16 l (4 l); `lds` is the wave's.  Not counted by the compiler: the
// kernel waits for them itself.
__device__ inline void load_lds16(uint32_t lds, uint32_t offset, s32x4 from)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(offset), "s"(from) : "memory");
}
__device__ inline void load_lds4(uint32_t lds, uint32_t offset, s32x4 from)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds), "v"(offset), "s"(from) : "memory");
}

// The adapters' scaled inner products as the rows kernels read them: blocks of 32 rows, of those pieces of 4 of the rank, so that the rows of a
// block lie next to each other (a load of a wave's operand is 512 bytes in a row then; with a row a lane, and the matrix read again for every 32 rows,
// the backward call of 8192 rows of rank 64, 4096 -> 4096 took 305 us, and takes 294).
__device__ inline int64_t scaled_at(int t, int r, int rank) { return ((int64_t)(t >> 5) * rank + (r & ~3)) * 32 + (t & 31) * 4 + (r & 3); }

constexpr uint32_t NOWHERE = 0x80000000u;                      // an offset past every resource

// Eight fp32 values as sums of values of the activations' type, for products that are to have fp32's precision.  Three of bf16 hold all 24 bits: the
// upper half of an fp32 value is a bf16 value, and what is left after two such cuts fits a third.  Two of f16, rounded, hold 22 where the value is in
// f16's range, which is why values are first multiplied by a power of two (SCALED) that brings the largest of them to 2^14 .. 2^15; what is
// smaller than that by more than 2^17 keeps an error of 2^-40 of the largest.
template <class T>
struct Pieces {
    static constexpr bool SCALED = !__is_same(T, __bf16);
    static constexpr int N = SCALED ? 2 : 3;
    typename Half<T>::v8 of[N];
};

// What is left of a value after a piece: nothing of an infinite one.
__device__ inline float rest_of(float v, float piece) { return fabsf(v) == INFINITY ? 0.0f : v - piece; }

template <class T>
__device__ inline Pieces<T> split8(const float *v, float scale)
{
    Pieces<T> p;
    if constexpr (!Pieces<T>::SCALED) {
        uint32_t rest[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) rest[j] = __float_as_uint(v[j]);
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            u32x4 half;
#pragma unroll
            for (int j = 0; j < 4; ++j) half[j] = __builtin_amdgcn_perm(rest[2 * j + 1], rest[2 * j], 0x07060302u);
            p.of[k] = __builtin_bit_cast(typename Half<T>::v8, half);
            if (k < 2)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float all = __uint_as_float(rest[j]), half = __uint_as_float(rest[j] & 0xffff0000u);
                    rest[j] = __float_as_uint(k == 0 ? rest_of(all, half) : all - half);     // (no rest is infinite)
                }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            p.of[0][j] = (T)(v[j] * scale);
            p.of[1][j] = (T)rest_of(v[j] * scale, (float)p.of[0][j]);
        }
    }
    return p;
}

// The exponent of the power of two for values whose largest magnitude is `top` (fp32's range needs -114 .. 141; what is below 2^-112 is brought as near
// to 2^14 as a power of two whose reciprocal is one, too), and that power.
__device__ inline int piece_exponent(float top) { return min(141 - (int)(__float_as_uint(top) >> 23), 126); }
__device__ inline float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

// The larger of lanes l and l + 32; and the largest of the wave.  (Magnitudes: as whole numbers they have the same order.)
__device__ inline float larger_half(float m)
{
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
    return __uint_as_float(max(both[0], both[1]));
}
__device__ inline float wave_top(float m)
{
    int v = __float_as_int(m);
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x128, 0xf, 0xf, true));     // sixteen lanes turned by 8, 4, 2, 1
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x124, 0xf, 0xf, true));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x122, 0xf, 0xf, true));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x121, 0xf, 0xf, true));
    return __int_as_float(max(max(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16)),
                              max(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48))));
}

// Eight values along the rows (the contracted axis) of a lane's channel, out of a tile of rows in LDS: two reads that exchange the axes
// of 4 x 16 values within 16 lanes.  `next` bytes further on lie the other four rows.
template <class T>
__device__ inline typename Half<T>::v8 read_turned(const char *at, int next)
{
    using v4s = __attribute__((ext_vector_type(4))) short;
    using lds_v4s = __attribute__((address_space(3))) v4s;
    const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)(at));
    const v4s b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)(at + next));
    return __builtin_bit_cast(typename Half<T>::v8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// ---- 8-bit activations ---------------------------------------------------------------------------------------

// Where a thread's pieces of 8 channels lie: rows of `pieces` (whole words of exponents: 16 pieces each), a grid's stride apart.
struct Walk {
    int64_t rows;
    int pieces;
    int64_t step_rows;
    int step_pieces;
};

// a grid of at most 8192 workgroups, and the walk of its threads
inline unsigned walk_of(int64_t rows, int C, Walk &w)
{
    w.rows = rows;
    w.pieces = (C + 127) / 128 * 16;
    const int64_t blocks = (rows * w.pieces + 255) / 256, grid = blocks < 8192 ? blocks : 8192;
    w.step_rows = grid * 256 / w.pieces;
    w.step_pieces = (int)(grid * 256 % w.pieces);
    return (unsigned)grid;
}

// Values from their 8-bit form, by workgroup `block` of the walk's grid.
template <class T>
__device__ inline void restore_rows(const int8_t *__restrict__ q, const uint8_t *__restrict__ e, const Walk &w, int C, T *__restrict__ x, int64_t ldx, int64_t block)
{
    using v8 = typename Half<T>::v8;
    const int64_t id = block * 256 + threadIdx.x;
    int64_t t = id / w.pieces;
    int p = (int)(id - t * w.pieces);
    for (; t < w.rows; t += w.step_rows) {
        if (p * 8 < C) {
            const uint2 raw = *(const uint2 *)(q + t * C + p * 8);
            const float u = unit_of(e[t * (w.pieces >> 2) + (p >> 2)]);
            v8 v;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (T)kept_value((int)(int8_t)((i < 4 ? raw.x : raw.y) >> (8 * (i & 3))), u);
            *(u32x4 *)(x + t * ldx + p * 8) = __builtin_bit_cast(u32x4, v);
        }
        p += w.step_pieces;
        if (p >= w.pieces) {
            p -= w.pieces;
            ++t;
        }
    }
}

}  // namespace snn
