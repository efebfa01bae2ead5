// Rotary positions with several axes.  Pair i of a head's channels (u, w) turns
// by a = pos[axis[i]][token] * freq[i]:
//   (u cos a - w sin a, u sin a + w cos a)
// The gradient is the rotation by -a.
//
// An angle is made in turns in 64 bits (pos * freq / 2 pi), of which the whole turns are
// taken off before it goes to 32 bits: far positions keep their angle to 2^-25 of
// a turn.  The angles of a token are made once, in LDS, for all of its heads.
#include <hip/hip_runtime.h>

#include "nmspmm_attn_internal.h"
#include "nmspmm_values.h"

namespace nmspmm {
namespace {

constexpr int kRotaryThreads = 256;

// Tokens of a workgroup: `per` of them, whose angles lie in LDS.
// VEC: items of 8 channels at 16-byte boundaries (halves: 8 pairs as two pieces; pairs: 4
// pairs in one), else of one pair; the channels past the pairs are copied by the same piece.
template <class T, bool VEC>
__global__ __launch_bounds__(kRotaryThreads) void k_rotary(RotaryArgs a, int per) {
    extern __shared__ float2 turn[];
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
        turn[e] = make_float2(c, s * a.sign);
    }
    __syncthreads();
    const int heads = a.part[0].heads + a.part[1].heads;
    // items of a head: the pairs' and those of the channels behind them
    const int turned = !VEC ? a.pairs : a.interleaved ? a.pairs / 4 : a.pairs / 8;
    const int rest = VEC ? (a.d - 2 * a.pairs) / 8 : a.d - 2 * a.pairs;
    const int items = turned + rest, token_items = heads * items;
    for (int e = threadIdx.x; e < n * token_items; e += kRotaryThreads) {
        const int t = e / token_items, r = e - t * token_items;
        int h = r / items;
        const int i = r - h * items;
        const bool second = h >= a.part[0].heads;
        const RotaryPart &p = a.part[second];
        if (second) h -= a.part[0].heads;
        const T *x = (const T *)p.x + (t0 + t) * p.x_token + h * p.x_head;
        T *out = (T *)p.out + (t0 + t) * p.out_token + h * p.out_head;
        const float2 *at = turn + t * a.pairs;
        if constexpr (!VEC) {
            if (i >= turned) {
                const int c = 2 * a.pairs + i - turned;
                out[c] = x[c];
                continue;
            }
            const int cu = a.interleaved ? 2 * i : i, cw = a.interleaved ? 2 * i + 1 : i + a.pairs;
            const float u = (float)x[cu], w = (float)x[cw];
            const float2 z = at[i];
            out[cu] = (T)(u * z.x - w * z.y);
            out[cw] = (T)(u * z.y + w * z.x);
        } else {
            if (i >= turned) {
                const int c = 2 * a.pairs + (i - turned) * 8;
                *(typename Raw8<T>::vec *)(out + c) = load8(x + c).v;
            } else if (a.interleaved) {
                const auto v = load8(x + 8 * i).v;
                float f[8];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 z = at[4 * i + j];
                    const float u = (float)v[2 * j], w = (float)v[2 * j + 1];
                    f[2 * j] = u * z.x - w * z.y;
                    f[2 * j + 1] = u * z.y + w * z.x;
                }
                store8(out + 8 * i, f);
            } else {
                const auto vu = load8(x + 8 * i).v, vw = load8(x + a.pairs + 8 * i).v;
                float fu[8], fw[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float2 z = at[8 * i + j];
                    const float u = (float)vu[j], w = (float)vw[j];
                    fu[j] = u * z.x - w * z.y;
                    fw[j] = u * z.y + w * z.x;
                }
                store8(out + 8 * i, fu);
                store8(out + a.pairs + 8 * i, fw);
            }
        }
    }
}

template <class T>
int launch(bool vec, const RotaryArgs &a, hipStream_t stream) {
    const int heads = a.part[0].heads + a.part[1].heads;
    // as many tokens as give every thread two items, within the angles' room
    const int64_t items = (int64_t)heads * (vec ? (a.d + 15) / 16 : (a.d + 1) / 2);
    int64_t per = (2 * kRotaryThreads + items - 1) / items;
    const int64_t room = 16384 / (8 * a.pairs);
    per = per < 1 ? 1 : per > room ? room : per;
    const int64_t grid = (a.tokens + per - 1) / per;
    if (grid >= (1ll << 24)) return (int)hipErrorInvalidConfiguration;   // a launch's threads are counted in 32 bits
    const size_t lds = (size_t)per * a.pairs * 8;
    if (vec)
        k_rotary<T, true><<<dim3((unsigned)grid), kRotaryThreads, lds, stream>>>(a, (int)per);
    else
        k_rotary<T, false><<<dim3((unsigned)grid), kRotaryThreads, lds, stream>>>(a, (int)per);
    return (int)hipGetLastError();
}

}  // namespace

int launch_rotary(int type, bool vec, const RotaryArgs &a, void *stream) {
    const hipStream_t s = (hipStream_t)stream;
    return type == NM_TYPE_F16 ? launch<half_t>(vec, a, s)
                               : type == NM_TYPE_BF16 ? launch<bf16_t>(vec, a, s) : launch<float>(vec, a, s);
}

}  // namespace nmspmm
