// Rotary positions with several axes.  Pair i of a head's channels (u, w) turns
// by a = pos[axis[i]][token] * freq[i]:
//   (u cos a - w sin a, u sin a + w cos a)
// The gradient is the rotation by -a.
//
// An angle is made in turns in 64 bits (pos * freq / 2 pi), of which the whole turns are
// taken off before it goes to 32 bits: far positions keep their angle to 2^-25 of
// a turn.  The angles of a token are made once, in LDS, for all of its heads.
//
// Bound by memory: every value is read and written once.  18464 x 32 x 64 bf16 in halves 24.2 us,
// 12544 x 24 x 64 fp16 in pairs 15.7 us,
// 4.9 TB/s, 8192 x 16 x 91 bf16 (odd rows: pieces of 1, 2 and 4 values at their
// ends) 16.0 us, 3.0 TB/s; a pair a thread took 31 us there.  One token: the launch (2.3 us).  Few tokens take what a
// workgroup takes for its angles and items one after another: 5 heads of 91 channels, 37 pairs, fp32, 18 tokens a
// workgroup, 7.6 us for 18 tokens (one workgroup), 8.0 for 1021 (57), 9.1 for 4000.
#include <hip/hip_runtime.h>

#include "nmspmm_attn_internal.h"
#include "nmspmm_values.h"

namespace nmspmm {
namespace {

constexpr int kRotaryThreads = 256;

// Up to 8 values at any alignment of their type (the hardware's loads and stores take it), in pieces of 8, 4, 2 and 1.
template <class T>
struct Some {
    typedef T vec __attribute__((ext_vector_type(8)));
    template <int N>
    using any = T __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    template <int N, int AT = 0>
    static __device__ __forceinline__ void get(const T *p, vec &v) {
        constexpr int W = N >= 8 ? 8 : N >= 4 ? 4 : N >= 2 ? 2 : 1;
        const any<W> x = *(const any<W> *)(p + AT);
#pragma unroll
        for (int j = 0; j < W; ++j) v[AT + j] = x[j];
        if constexpr (N > W) get<N - W, AT + W>(p, v);
    }
    template <int N, int AT = 0>
    static __device__ __forceinline__ void put(T *p, const vec &v) {
        constexpr int W = N >= 8 ? 8 : N >= 4 ? 4 : N >= 2 ? 2 : 1;
        any<W> x;
#pragma unroll
        for (int j = 0; j < W; ++j) x[j] = v[AT + j];
        *(any<W> *)(p + AT) = x;
        if constexpr (N > W) put<N - W, AT + W>(p, v);
    }
    static __device__ __forceinline__ vec load(const T *p, int n) {
        vec v = {};
        if (n >= 8) {
            get<8>(p, v);
            return v;
        }
        switch (n) {
            case 1: get<1>(p, v); break;
            case 2: get<2>(p, v); break;
            case 3: get<3>(p, v); break;
            case 4: get<4>(p, v); break;
            case 5: get<5>(p, v); break;
            case 6: get<6>(p, v); break;
            case 7: get<7>(p, v); break;
            default: break;
        }
        return v;
    }
    static __device__ __forceinline__ void store(T *p, int n, const vec &v) {
        if (n >= 8) return put<8>(p, v);
        switch (n) {
            case 1: put<1>(p, v); break;
            case 2: put<2>(p, v); break;
            case 3: put<3>(p, v); break;
            case 4: put<4>(p, v); break;
            case 5: put<5>(p, v); break;
            case 6: put<6>(p, v); break;
            case 7: put<7>(p, v); break;
            default: break;
        }
    }
};

__host__ __device__ constexpr int angles_of(int pairs) { return (pairs + 7) & ~7; }

// Tokens of a workgroup: `per` of them, whose angles lie in LDS.  An item is two pieces of 8
// channels: 8 pairs, or channels past the pairs, which are copied.
template <class T>
__global__ __launch_bounds__(kRotaryThreads) void k_rotary(RotaryArgs a, int per) {
    using vec = typename Some<T>::vec;
    extern __shared__ __attribute__((aligned(16))) float2 turn[];       // angles of a token: whole items of pairs
    const int row = angles_of(a.pairs);
    const int64_t t0 = (int64_t)blockIdx.x * per;
    const int n = (int)(a.tokens - t0 < per ? a.tokens - t0 : per);
    for (int e = threadIdx.x; e < n * a.pairs; e += kRotaryThreads) {
        const int t = e / a.pairs, i = e - t * a.pairs;
        const int axis = a.axis[i] < 0 ? 0 : a.axis[i] < a.axes ? a.axis[i] : a.axes - 1;
        const int64_t at = axis * a.ld_pos + t0 + t;
        const double pos = a.pos_float ? (double)((const float *)a.pos)[at] : (double)((const int32_t *)a.pos)[at];
        const double turns = pos * a.freq[i] * 0.15915494309189533577;
        float s, c;
        sincospif((float)(2.0 * (turns - __builtin_rint(turns))), &s, &c);
        turn[t * row + i] = make_float2(c, s * a.sign);
    }
    __syncthreads();
    const int heads = a.part[0].heads + a.part[1].heads;
    // items of a head: the pairs' and those of the channels behind them
    const int rest = a.d - 2 * a.pairs, turned = (a.pairs + 7) / 8, copied = (rest + 15) / 16;
    const int items = turned + copied, token_items = heads * items;
    for (int e = threadIdx.x; e < n * token_items; e += kRotaryThreads) {
        const int t = e / token_items, r = e - t * token_items;
        int h = r / items;
        const int i = r - h * items;
        const bool second = h >= a.part[0].heads;
        const RotaryPart &p = a.part[second];
        if (second) h -= a.part[0].heads;
        const T *x = (const T *)p.x + (t0 + t) * p.x_token + h * p.x_head;
        T *out = (T *)p.out + (t0 + t) * p.out_token + h * p.out_head;
        const float2 *at = turn + t * row;
        // the item's pieces, neighbours' side by side
        const bool turns = i < turned;
        const int first = turns ? 8 * i : 2 * a.pairs + 8 * (i - turned), end = turns ? 2 * a.pairs : a.d;
        const bool halves = turns && !a.interleaved;
        const int c0 = first, c1 = first + (halves ? a.pairs : 8 * (turns ? turned : copied));
        const int n0 = (halves ? a.pairs : end) - c0, n1 = end - c1;
        vec v0 = Some<T>::load(x + c0, n0), v1 = Some<T>::load(x + c1, n1);
        if (halves) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float2 z = at[8 * i + j];
                const float u = (float)v0[j], w = (float)v1[j];
                v0[j] = (T)(u * z.x - w * z.y);
                v1[j] = (T)(u * z.y + w * z.x);
            }
        } else if (turns) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 z0 = at[4 * i + j], z1 = at[4 * (i + turned) + j];
                const float u0 = (float)v0[2 * j], w0 = (float)v0[2 * j + 1], u1 = (float)v1[2 * j], w1 = (float)v1[2 * j + 1];
                v0[2 * j] = (T)(u0 * z0.x - w0 * z0.y);
                v0[2 * j + 1] = (T)(u0 * z0.y + w0 * z0.x);
                v1[2 * j] = (T)(u1 * z1.x - w1 * z1.y);
                v1[2 * j + 1] = (T)(u1 * z1.y + w1 * z1.x);
            }
        }
        Some<T>::store(out + c0, n0, v0);
        Some<T>::store(out + c1, n1, v1);
    }
}

template <class T>
int launch(const RotaryArgs &a, hipStream_t stream) {
    const int heads = a.part[0].heads + a.part[1].heads;
    // as many tokens as give every thread two items, within the angles' room
    const int64_t items = (int64_t)heads * ((a.d + 15) / 16);
    int64_t per = (2 * kRotaryThreads + items - 1) / items;
    const int64_t room = 16384 / (8 * angles_of(a.pairs));
    per = per < 1 ? 1 : per > room ? room : per;
    const int64_t grid = (a.tokens + per - 1) / per;
    if (grid >= (1ll << 24)) return (int)hipErrorInvalidConfiguration;   // a launch's threads are counted in 32 bits
    const size_t lds = (size_t)per * angles_of(a.pairs) * 8;
    k_rotary<T><<<dim3((unsigned)grid), kRotaryThreads, lds, stream>>>(a, (int)per);
    return (int)hipGetLastError();
}

}  // namespace

int launch_rotary(int type, const RotaryArgs &a, void *stream) {
    const hipStream_t s = (hipStream_t)stream;
    return type == NM_TYPE_F16 ? launch<half_t>(a, s) : type == NM_TYPE_BF16 ? launch<bf16_t>(a, s) : launch<float>(a, s);
}

}  // namespace nmspmm
