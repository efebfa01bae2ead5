// Activation types of the transformer-block kernels: loads to and stores from
// 32-bit floats, and the reductions of a wave and of the waves of a row.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace nmspmm {

typedef _Float16 half_t;
typedef __bf16 bf16_t;

// Eight values as they travel (16 bytes of a 16-bit type, 32 of binary32).
template <class T>
struct Raw8 {
    typedef T vec __attribute__((ext_vector_type(8), aligned(16)));
    vec v;
};

template <class T>
__device__ __forceinline__ Raw8<T> load8(const T *p) {
    return {*(const typename Raw8<T>::vec *)p};
}
template <class T>
__device__ __forceinline__ void store8(T *p, const float (&f)[8]) {
    typename Raw8<T>::vec v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (T)f[e];
    *(typename Raw8<T>::vec *)p = v;
}

// A cross-lane move within rows of 16 lanes and between them; lanes that have
// no source, and rows outside the mask, get `old`.
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ float dpp(float old, float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, old),
                                                                 __builtin_bit_cast(int, x), CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ float last_lane(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

// Sum and largest value (of values >= 0, or NaN) over the 64 lanes, the same in every lane and the
// same order of additions every time: xor 1, xor 2, half rows, rows, then rows
// 0 and 2 into 1 and 3, and row 1 into 2 and 3; lane 63 ends with all.
__device__ __forceinline__ float wave_sum(float x) {
    x += dpp<0xB1>(0.f, x);
    x += dpp<0x4E>(0.f, x);
    x += dpp<0x141>(0.f, x);
    x += dpp<0x140>(0.f, x);
    x += dpp<0x142, 0xA>(0.f, x);
    x += dpp<0x143, 0xC>(0.f, x);
    return last_lane(x);
}
// Two sums in one: lanes 0 to 31 end with that of a, the others with that of b.  After the
// swap of a's upper half with b's lower one an addition joins both halves of both; then
// rows 16 lanes apart, and the steps of wave_sum within a row.
__device__ __forceinline__ float wave_sums(float a, float b) {
    const auto half = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b),
                                                       false, false);
    const float y = __builtin_bit_cast(float, (uint32_t)half[0]) + __builtin_bit_cast(float, (uint32_t)half[1]);
    const auto row = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, y), __builtin_bit_cast(uint32_t, y),
                                                      false, false);
    float x = __builtin_bit_cast(float, (uint32_t)row[0]) + __builtin_bit_cast(float, (uint32_t)row[1]);
    x += dpp<0xB1>(0.f, x);
    x += dpp<0x4E>(0.f, x);
    x += dpp<0x141>(0.f, x);
    x += dpp<0x140>(0.f, x);
    return x;
}
__device__ __forceinline__ float lane_of(float x, int lane) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
}
// The larger of two magnitudes; a NaN, or an infinity, wins: the bits of a
// float without its sign are ordered as the values are, NaN above infinity.
__device__ __forceinline__ float larger(float a, float b) {
    const uint32_t x = __builtin_bit_cast(uint32_t, a), y = __builtin_bit_cast(uint32_t, b);
    return __builtin_bit_cast(float, x > y ? x : y);
}
__device__ __forceinline__ float magnitude(float a) {
    return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, a) & 0x7FFFFFFFu);
}
__device__ __forceinline__ float wave_largest(float x) {
    x = larger(x, dpp<0xB1>(0.f, x));
    x = larger(x, dpp<0x4E>(0.f, x));
    x = larger(x, dpp<0x141>(0.f, x));
    x = larger(x, dpp<0x140>(0.f, x));
    x = larger(x, dpp<0x142, 0xA>(0.f, x));
    x = larger(x, dpp<0x143, 0xC>(0.f, x));
    return last_lane(x);
}

// The same over the WPR waves of a row.  `box` is the row's LDS (2 x 2 x WPR floats):
// calls alternate between its halves, so one barrier each is enough.  Every
// thread of the workgroup calls it the same number of times.
template <int WPR>
struct RowReduce {
    float (*box)[2][WPR > 1 ? WPR : 1];
    int wave;          // of the row
    int turn = 0;
    __device__ void sum2(float &a, float &b) {
        const float both = wave_sums(a, b);
        if constexpr (WPR == 1) {
            a = lane_of(both, 0);
            b = lane_of(both, 32);
        } else {
            if ((threadIdx.x & 31) == 0) box[turn][(threadIdx.x >> 5) & 1][wave] = both;
            __syncthreads();
            a = b = 0.f;
#pragma unroll
            for (int w = 0; w < WPR; ++w) {
                a += box[turn][0][w];
                b += box[turn][1][w];
            }
            turn ^= 1;
        }
    }
    __device__ float sum(float a) {
        a = wave_sum(a);
        if constexpr (WPR > 1) {
            if ((threadIdx.x & 63) == 0) box[turn][0][wave] = a;
            __syncthreads();
            a = 0.f;
#pragma unroll
            for (int w = 0; w < WPR; ++w) a += box[turn][0][w];
            turn ^= 1;
        }
        return a;
    }
    __device__ float largest(float a) {
        a = wave_largest(a);
        if constexpr (WPR > 1) {
            if ((threadIdx.x & 63) == 0) box[turn][0][wave] = a;
            __syncthreads();
            a = 0.f;
#pragma unroll
            for (int w = 0; w < WPR; ++w) a = larger(a, box[turn][0][w]);
            turn ^= 1;
        }
        return a;
    }
};

// Row codes: scale = top / 127, code = rint(x * (127 / top)), decided in
// binary32 (both quotients correctly rounded).  Below 2^-100 the quotients
// would leave the normal range: such a row is all zero.  A row with an
// infinity or NaN has the scale NaN and zero codes, so its outputs are NaN.
struct RowScale {
    float scale, inv;
};
__device__ __forceinline__ RowScale row_scale(float top) {
    if (!(top < __builtin_inff())) return {__builtin_nanf(""), 0.f};
    if (top < 0x1p-100f) return {0.f, 0.f};
    return {top / 127.f, 127.f / top};
}
// |x * inv| <= 127 * (1 + 2^-23), whose nearest integer is in range.  In a row that has an
// infinity or NaN the products may be NaN: they convert to 0 (v_cvt_i32_f32).
__device__ __forceinline__ int row_code(float x, float inv) {
    int r;
    asm("v_cvt_i32_f32 %0, %1" : "=v"(r) : "v"(__builtin_rintf(x * inv)));
    return r;
}
__device__ __forceinline__ uint32_t pack4(int a, int b, int c, int d) {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm((uint32_t)d, (uint32_t)c, 0x0C0C0400u),
                                 __builtin_amdgcn_perm((uint32_t)b, (uint32_t)a, 0x0C0C0400u), 0x05040100u);
}

}  // namespace nmspmm
