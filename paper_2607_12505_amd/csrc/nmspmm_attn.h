// Device code shared by the kernels of differential attention: tiles of rows in
// LDS, operands of the 32 x 32 x 16 matrix instruction from them, the extent of
// a sequence and what its rows see.
//
// Operand maps (a lane is l, half h = l / 32, column or row r = l % 32):
//   A, B: 8 values of row (A) or column (B) r at k = 8 h .. 8 h + 7
//   C:    column r, value e of 16 at row 8 (e / 4) + 4 h + e % 4
// So the rows of C that a lane holds in values 8 c .. 8 c + 7 are the quads 16 c + 4 h
// and 16 c + 8 + 4 h: rounded to 16 bits they are a B operand of 16 rows of k as they
// lie, if the A operand takes its k in the same order.  turned() reads A that way
// from rows in LDS, so no value of the maps crosses lanes.
#pragma once

#include <hip/hip_runtime.h>

#include "nmspmm_attn_internal.h"
#include "nmspmm_values.h"

namespace nmspmm {
namespace {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));

template <class T>
struct Mfma;
template <>
struct Mfma<half_t> {
    typedef half_t v8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ v16f mul(v8s a, v8s b, v16f c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
};
template <>
struct Mfma<bf16_t> {
    typedef bf16_t v8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ v16f mul(v8s a, v8s b, v16f c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
};

// Values 8 c .. 8 c + 7 of C, rounded once: a B operand.
template <class T>
__device__ __forceinline__ v8s pack(const float (&f)[16], int c) {
    typedef T v8 __attribute__((ext_vector_type(8)));
    v8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (T)f[8 * c + e];
    return __builtin_bit_cast(v8s, r);
}

// Sum and larger of a lane's value and that of the lane 32 away, in both.
__device__ __forceinline__ float half_sum(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}
__device__ __forceinline__ float half_max(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}

// ---------------------------------------------------------------- tiles in LDS
// A tile is rows of CPR 16-byte pieces.  Piece c of row r lies at place c ^ swizzle(r):
// the rows of an A or B operand (16 lanes at one piece) and the 4 rows of a turned
// one (16 lanes at 32 bytes of each) then lie in distinct banks.
// LDS is addressed by bytes from its start.
template <class V>
__device__ __forceinline__ V lds_load(uint32_t at) {
    return *(const __attribute__((address_space(3))) V *)(uintptr_t)at;
}
__device__ __forceinline__ uint32_t lds_start(char *lds) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
}
template <int CPR>
__device__ __forceinline__ int swizzle(int r) {
    if constexpr (CPR == 4) return ((r >> 1 & 1) * 2) ^ (r >> 2 & 1) ^ ((r >> 3 & 1) * 2);
    if constexpr (CPR == 8) return ((r & 1) * 2) ^ ((r >> 1 & 1) * 4) ^ (r >> 2 & 1) ^ ((r >> 3 & 1) * 2);
    return ((r & 1) * 4) ^ ((r >> 1 & 1) * 10) ^ (r >> 2 & 1) ^ ((r >> 3 & 1) * 2);
}

// 16 bytes a lane straight to LDS, lane l's at lds + 16 l (lds wave-uniform); zeros
// where the offset lies past the buffer.  M0 holds the LDS address; the wait states
// cover its write and a vector instruction's write of the resource's registers.
__device__ __forceinline__ void dma16(v4i buffer, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(offset), "s"(buffer),
                 "s"(lds)
                 : "memory", "m0");
}
__device__ __forceinline__ void dma4(v4i buffer, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(offset), "s"(buffer),
                 "s"(lds)
                 : "memory", "m0");
}
__device__ __forceinline__ v4i buffer_of(const void *p, int64_t bytes) {
    const uint64_t at = (uint64_t)p;
    return v4i{__builtin_amdgcn_readfirstlane((int)(uint32_t)at),
               __builtin_amdgcn_readfirstlane((int)((uint32_t)(at >> 32) & 0xFFFFu)),
               __builtin_amdgcn_readfirstlane((int)(bytes < 0 ? 0 : bytes)), 0x00020000};
}
// All of this wave's loads have arrived, then the workgroup's barrier.
__device__ __forceinline__ void arrive() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// ROWS rows of `width` values into LDS: rows from `left` on and columns from `width` on
// are zero, whatever memory holds there.  In whole pieces at 16-byte boundaries the
// loads go straight to LDS and arrive later; otherwise a value at a time, at once.
template <class T, int CPR, int ROWS, int WAVES>
struct Tile {
    static constexpr int LOADS = ROWS * CPR / (64 * WAVES), BYTES = ROWS * CPR * 16;
    static_assert(LOADS * 64 * WAVES == ROWS * CPR, "whole loads");
    static __device__ __forceinline__ void load(const T *p, int64_t stride, int left, int width, bool vec, uint32_t lds,
                                                int wave, int lane) {
        left = left < 0 ? 0 : left < ROWS ? left : ROWS;
        if (vec) {
            const v4i buffer = buffer_of(p, left ? ((left - 1) * stride + width) * 2 : 0);
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int id = (i * WAVES + wave) * 64 + lane, row = id / CPR, c = (id % CPR) ^ swizzle<CPR>(row);
                const uint32_t offset = c * 8 < width ? (uint32_t)(row * (uint32_t)stride * 2 + c * 16) : 0x80000000u;
                dma16(buffer, offset, lds + (i * WAVES + wave) * 1024);
            }
        } else {
#pragma unroll 1
            for (int i = 0; i < LOADS; ++i) {
                const int id = (i * WAVES + wave) * 64 + lane, row = id / CPR, c = (id % CPR) ^ swizzle<CPR>(row);
                typedef T v8 __attribute__((ext_vector_type(8)));
                v8 v;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v[e] = (T)0.f;
                    if (row < left && c * 8 + e < width) v[e] = p[row * stride + c * 8 + e];
                }
                *(__attribute__((address_space(3))) v8 *)(uintptr_t)(lds + id * 16) = v;
            }
        }
    }
    // The A or B operand of 32 rows from `row` (a multiple of 32): k = 16 c .. 16 c + 15.
    static __device__ __forceinline__ v8s rows(uint32_t lds, int row, int c, int lane) {
        const int r = row + (lane & 31);
        return lds_load<v8s>(lds + (r * CPR + ((2 * c + (lane >> 5)) ^ swizzle<CPR>(r & 15))) * 16);
    }
    // The A operand of 32 columns from 32 x with k over the rows row .. row + 15 (row: a
    // multiple of 16) in the order that values of C have (above).
    static __device__ __forceinline__ v8s turned(uint32_t lds, int row, int x, int lane) {
        const int quad = (lane >> 5) * 4 + ((lane & 15) >> 2);
        const int piece = 4 * x + 2 * (lane >> 4 & 1) + (lane >> 1 & 1), low = 8 * (lane & 1);
        const v4s a = read4(lds + ((row + quad) * CPR + (piece ^ swizzle<CPR>(quad))) * 16 + low);
        const v4s b = read4(lds + ((row + 8 + quad) * CPR + (piece ^ swizzle<CPR>(8 + quad))) * 16 + low);
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    // 4 rows x 16 columns of 16 bits for 16 lanes: lane i gives the address of 4 columns of row
    // i / 4 and gets the 4 rows of column i.
    static __device__ __forceinline__ v4s read4(uint32_t at) {
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)(uintptr_t)at);
    }
};

// The B operand of a row in memory, k = 16 c .. 16 c + 15, zero from `width` on.
template <class T>
__device__ __forceinline__ v8s row_operand(const T *p, bool valid, int c, int width, bool vec, int lane) {
    const int at = 16 * c + 8 * (lane >> 5);
    v8s r = {0, 0, 0, 0, 0, 0, 0, 0};
    if (!valid || at >= width) return r;
    if (vec) return *(const v8s *)(p + at);
    typedef T v8 __attribute__((ext_vector_type(8)));
    v8 v = __builtin_bit_cast(v8, r);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (at + e < width) v[e] = p[at + e];
    return __builtin_bit_cast(v8s, v);
}

// 4 values of a row at column c of `width`.
template <class T>
__device__ __forceinline__ void store4(T *p, int c, int width, bool vec, float a, float b, float d, float e) {
    typedef T v4 __attribute__((ext_vector_type(4)));
    if (vec) {
        if (c < width) *(v4 *)(p + c) = v4{(T)a, (T)b, (T)d, (T)e};
        return;
    }
    if (c < width) p[c] = (T)a;
    if (c + 1 < width) p[c + 1] = (T)b;
    if (c + 2 < width) p[c + 2] = (T)d;
    if (c + 3 < width) p[c + 3] = (T)e;
}

// Codes in 16 bits of values of which `top` is the largest magnitude: what the backward pass
// keeps of both maps' products, whose sums with do are differences' small parts.
struct KeptScale {
    float scale, inv;
};
__device__ __forceinline__ KeptScale kept_scale(float top) {
    if (!(top < __builtin_inff())) return {__builtin_nanf(""), 0.f};
    if (top < 0x1p-100f) return {0.f, 0.f};
    return {top * (1.f / 32767.f), 32767.f / top};
}
__device__ __forceinline__ short kept_code(float x, float inv) {
    int r;
    asm("v_cvt_i32_f32 %0, %1" : "=v"(r) : "v"(__builtin_rintf(x * inv)));
    return (short)r;
}

// ---------------------------------------------------------------- sequences

// A sequence: its lengths, its tensors' first rows and the number of its first row.
// Lengths and offsets come from device memory: they are held within the tensors.
struct Sequence {
    int nq, nk;
    int64_t q0, k0;   // rows before it in packed tensors (else the batch's stride tells)
    int64_t row0;
    int batch;        // 0 where packed
};
__device__ __forceinline__ int64_t within(int64_t v, int64_t lo, int64_t hi) { return v < lo ? lo : v > hi ? hi : v; }
__device__ __forceinline__ Sequence sequence(const AttnArgs &a, int b) {
    Sequence s;
    s.q0 = s.k0 = 0;
    s.nq = a.tq;
    s.nk = a.tk;
    s.row0 = (int64_t)b * a.tq;
    s.batch = b;
    if (a.q_offsets) {
        s.q0 = within(a.q_offsets[b], 0, a.total_q);
        s.nq = (int)within(within(a.q_offsets[b + 1], s.q0, a.total_q) - s.q0, 0, a.tq);
        s.k0 = within(a.k_offsets[b], 0, a.total_k);
        s.nk = (int)within(within(a.k_offsets[b + 1], s.k0, a.total_k) - s.k0, 0, a.tk);
        s.row0 = s.q0;
        s.batch = 0;
    } else {
        if (a.q_lens) s.nq = (int)within(a.q_lens[b], 0, a.tq);
        if (a.k_lens) s.nk = (int)within(a.k_lens[b], 0, a.tk);
    }
    return s;
}
template <class T>
__device__ __forceinline__ T *head_of(const Heads &t, int batch, int64_t row, int head) {
    return (T *)t.p + batch * t.batch + row * t.token + head * t.head;
}

// First and last key that row t sees (last < first: none).
__device__ __forceinline__ int first_seen(const AttnArgs &a, const Sequence &s, int t) {
    const int at = t + s.nk - s.nq - a.left;
    return at > 0 ? at : 0;
}
__device__ __forceinline__ int last_seen(const AttnArgs &a, const Sequence &s, int t) {
    const int at = t + s.nk - s.nq + a.right;
    return at < s.nk - 1 ? at : s.nk - 1;
}

// lam of a head, by the whole wave: given, or exp(q1 . k1) - exp(q2 . k2) + init.
struct Weight {
    float lam, e1, e2;
};
__device__ __forceinline__ Weight weight_of(const nm_diff_weight &w, int head, int lane) {
    Weight r = {0.f, 0.f, 0.f};
    if (w.value) {
        r.lam = w.value[head];
        return r;
    }
    const int64_t at = w.per_head ? (int64_t)head * w.n : 0;
    float a = 0.f, b = 0.f;
    for (int i = lane; i < w.n; i += 64) {
        a += w.q1[at + i] * w.k1[at + i];
        b += w.q2[at + i] * w.k2[at + i];
    }
    r.e1 = expf(wave_sum(a));
    r.e2 = expf(wave_sum(b));
    r.lam = r.e1 - r.e2 + w.init;
    return r;
}

// Workgroups are dispatched round-robin over the 8 XCDs; those of one head (which share its
// keys) run on one of them, whose L2 then holds the keys.
__device__ __forceinline__ int near_block(int bid, int count) {
    const int xcd = bid & 7, local = bid >> 3, per = count >> 3, left = count & 7;
    return xcd < left ? xcd * (per + 1) + local : left * (per + 1) + (xcd - left) * per + local;
}

}  // namespace
}  // namespace nmspmm
