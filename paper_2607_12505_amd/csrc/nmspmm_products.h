// Epilogues of the products of a transformer block, on the k-loop of
// nmspmm_gemm.h: scales for each token and channel, the gate of a gated
// feed-forward block, its gradients, and plain 16-bit results.
//
// Large products are bound by the k-loop, whose matrix instructions run 43 % of the
// time, waits and LDS reads taking the rest: 18464 x 1024 -> 4096 dense to fp16 93 to 96 us,
// 1.65 POP/s of the 3.65 that the int8 instructions reach on such data in a bare loop
// (without its loads, or without its products, the loop still takes 75 to 85 us).
#pragma once

#include "nmspmm_block.h"
#include "nmspmm_gemm.h"
#include "nmspmm_values.h"

namespace nmspmm {
namespace {

// Pieces of rows whose start has only the alignment of their values (the
// hardware takes wide global accesses at any address of 2 bytes or more).
typedef unsigned int v4u_any __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned int v2u_any __attribute__((ext_vector_type(2), aligned(2)));

template <class T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    typedef T v2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, v2{(T)a, (T)b});
}
template <class T>
__device__ __forceinline__ v2u pack4_of(const v4f &f) {
    return v2u{pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3])};
}

// 16 bytes (16 / sizeof(T) channels from ch) of a row of n channels.
template <class T>
__device__ __forceinline__ void store_piece(T *row, int ch, int n, const v4i &v, bool stream) {
    constexpr int PER = 16 / sizeof(T);
    if (ch + PER <= n) {
        if (stream)
            __builtin_nontemporal_store(__builtin_bit_cast(v4u, v), (v4u_any *)(row + ch));
        else
            *(v4u_any *)(row + ch) = __builtin_bit_cast(v4u, v);
    } else {
        typedef T vec __attribute__((ext_vector_type(PER)));
        const vec t = __builtin_bit_cast(vec, v);
#pragma unroll
        for (int e = 0; e < PER; ++e)
            if (ch + e < n) row[ch + e] = t[e];
    }
}

// The wave's accumulators (or what was made of them) as rows of type T.
template <class G, class T, class Acc, class Value, class Row>
__device__ __forceinline__ void store_tile(int8_t *stg, int lane, const Acc (&acc)[G::FN][G::FM], int ch0, int n,
                                           bool stream, const Value &value, const Row &row_of) {
    store_rows<G, (int)sizeof(T)>(
        stg, lane, acc,
        [&](int i, int j, const Acc &v, int8_t *dst) {
            const v4f f = value(i, j, v);
            if constexpr (sizeof(T) == 4)
                *(v4f *)dst = f;
            else
                *(v2u *)dst = pack4_of<T>(f);
        },
        [&](int row, int ch, const v4i &v) {
            T *p = (T *)row_of(row, (T *)nullptr);
            if (p && ch0 + ch < n) store_piece<T>(p, ch0 + ch, n, v, stream);
        });
}

template <class F>
__device__ __forceinline__ void by_type(int type, const F &f) {
    if (type == NM_TYPE_F16)
        f((half_t *)nullptr);
    else if (type == NM_TYPE_BF16)
        f((bf16_t *)nullptr);
    else
        f((float *)nullptr);
}

// The scales of the wave's tokens: token fragment j, lane % 16.
template <class G>
__device__ __forceinline__ void load_row_scales(const BlockArgs &a, const TileAt &at, float (&sx)[G::FM]) {
#pragma unroll
    for (int j = 0; j < G::FM; ++j) {
        const int tok = at.tok + j * 16 + (at.lane & 15);
        sx[j] = a.row_scale[tok < a.m ? tok : a.m - 1];
    }
}

// The empty statement keeps the value in binary32: left alone, the compiler
// rounds some products straight to binary16, and a token would not have the same
// bits from every kernel.
__device__ __forceinline__ v4f scaled_value(const v4i &v, float sx, const v4f &c, const v4f &b) {
    v4f f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float x = __builtin_fmaf((float)v[e] * sx, c[e], b[e]);
        asm("" : "+v"(x));
        f[e] = x;
    }
    return f;
}

// The k-sliced tile: the sum of its four waves' parts for 4 channels of a token,
// and where they go.
template <class G>
__device__ __forceinline__ v4i sum_ks(const int8_t *lds, int row, int cc) {
    v4i v = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < 4; ++w) v += *(const v4i *)(lds + w * G::BM * G::ROWB + row * G::ROWB + cc * 16);
    return v;
}
template <class T>
__device__ __forceinline__ void store_four(const BlockArgs &a, int tok, int ch, const v4f &f) {
    T *row = (T *)a.out + (int64_t)tok * a.ldo;
    if (ch + 4 <= a.n_out) {
        if constexpr (sizeof(T) == 4)
            *(v4u_any *)(row + ch) = __builtin_bit_cast(v4u, f);
        else
            *(v2u_any *)(row + ch) = pack4_of<T>(f);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (ch + e < a.n_out) row[ch + e] = (T)f[e];
    }
}

// y = T(acc * sx[token] * c[channel] + b[channel]): the int32 sum is exact, three
// roundings in binary32 and the one to T.  The scales run along m and n, so they
// cost one multiplication each in the epilogue and nothing in the loop.
struct ScaledOut {
    static __device__ bool scaled(const BlockArgs &) { return true; }
    static __device__ const float *first(const BlockArgs &a) { return a.scale; }
    static __device__ const float *second(const BlockArgs &a) { return a.qscale; }

    template <class G, class Mul>
    static __device__ __forceinline__ void finish(const BlockArgs &a, const TileAt &at,
                                                  const v4i (&acc)[G::FN][G::FM], int8_t *stg, const Mul &multiplier,
                                                  int *) {
        float sx[G::FM];
        load_row_scales<G>(a, at, sx);
        by_type(a.type, [&](auto *t) {
            using T = typename std::remove_pointer<decltype(t)>::type;
            store_tile<G, T>(
                stg, at.lane, acc, at.ch, a.n_out, (a.stream_out & sizeof(T)) != 0,
                [&](int i, int j, const v4i &v) {
                    return scaled_value(v, sx[j], multiplier(0, i), a.qscale ? multiplier(1, i) : v4f{0, 0, 0, 0});
                },
                [&](int row, T *) -> T * {
                    return at.tok + row < a.m ? (T *)a.out + (int64_t)(at.tok + row) * a.ldo : nullptr;
                });
        });
    }

    template <class G>
    static __device__ __forceinline__ void finish_ks(const BlockArgs &a, const TileAt &at, const int8_t *lds, int *) {
        const int cc = threadIdx.x % G::CPR, ch = at.ch + cc * 4;   // the same channels for every row of this thread
        const int c = ch < a.n ? ch : 0;
        const v4f scale = *(const v4f *)(a.scale + c), bias = a.qscale ? *(const v4f *)(a.qscale + c) : v4f{0, 0, 0, 0};
        by_type(a.type, [&](auto *t) {
            using T = typename std::remove_pointer<decltype(t)>::type;
            for (int p = threadIdx.x; p < G::BM * G::CPR; p += 256) {
                const int row = p / G::CPR, tok = at.tok + row;
                if (tok >= a.m || ch >= a.n_out) continue;
                store_four<T>(a, tok, ch, scaled_value(sum_ks<G>(lds, row, cc), a.row_scale[tok], scale, bias));
            }
        });
    }
};

// act(g) and its derivative.  In steps of 2^-24 of the value: the exponential of sigmoid
// is the hardware's (2^x within an ulp, 2 steps) of an argument that is rounded to binary32, the
// reciprocal within an ulp, so silu and sigmoid are within 6 + 2 |g| steps and
// tanh gelu within 6 + 8 a, a = 2 sqrt(2 / pi) (|g| + 0.044715 |g|^3) its sigmoid's argument: under the
// rounding to binary16 or bfloat16 wherever the value is above 2^-100, in binary32 a few bits
// less in the far negative tail.
//   The normal distribution function of gelu: its tail at x = |g| is exp(-x^2 / 2) r(t), r a
// polynomial of t = 1 / (1 + p x).  p and the eight coefficients were fitted here (least squares,
// weighted until the largest relative error was least) to exp(x^2 / 2) erfc(x / sqrt(2)) / 2 for x to 16:
// 1.3e-7 of its value.  The roundings of the square and of its product with log2(e) / 2
// come back as a correction of the exponential, so gelu is within 32 steps down to g = -12,
// and 0 past -13.  (Formula 7.1.26 of Abramowitz and Stegun, Handbook of Mathematical
// Functions, 1964, is shorter but holds in absolute terms only: 1.6e-3 of gelu(-5).  erfcf of the
// library took half of the backward pass's first kernel.)
__device__ __forceinline__ float sigmoid(float g) {
    return __builtin_amdgcn_rcpf(1.f + __expf(-g));
}
__device__ __forceinline__ void act_and_slope(int act, float g, float &f, float &df) {
    if (act == NM_ACT_SILU) {
        const float s = sigmoid(g);
        f = g * s;
        df = s * __builtin_fmaf(g, 1.f - s, 1.f);
    } else if (act == NM_ACT_SIGMOID) {
        f = sigmoid(g);
        df = f * (1.f - f);
    } else if (act == NM_ACT_RELU) {
        f = g > 0.f || g != g ? g : 0.f;
        df = g > 0.f ? 1.f : 0.f;
    } else if (act == NM_ACT_GELU) {
        // past 16 the tail is 0, and an infinite square would make NaN of its correction
        const float x = __builtin_fminf(__builtin_fabsf(g), 16.f), h = x * x, h_lost = __builtin_fmaf(x, x, -h);
        constexpr float kHalf = -0.72134752f, kHalfLost = -9.6298e-9f;        // -log2(e) / 2
        const float y = kHalf * h;
        float lost = __builtin_fmaf(kHalf, h, -y);
        lost = __builtin_fmaf(kHalf, h_lost, lost);
        lost = __builtin_fmaf(kHalfLost, h, lost);
        float e = __builtin_amdgcn_exp2f(y);
        e = __builtin_fmaf(e, 0.69314718f * lost, e);
        const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.30759144f, x, 1.f));
        float q = __builtin_fmaf(0.03628652f, t, -0.14714111f);
        q = __builtin_fmaf(q, t, 0.16965123f);
        q = __builtin_fmaf(q, t, -0.025647799f);
        q = __builtin_fmaf(q, t, 0.11512103f);
        q = __builtin_fmaf(q, t, 0.10576676f);
        q = __builtin_fmaf(q, t, 0.12327715f);
        q = __builtin_fmaf(q, t, 0.12268628f);
        const float tail = q * t * e;                 // of the side that g is on
        const float p = g > 0.f ? 1.f - tail : tail;
        f = g * p;
        df = __builtin_fmaf(0.39894228040143268f * g, e, p);
    } else {   // NM_ACT_GELU_TANH: tanh(v) = 2 sigmoid(2 v) - 1
        const float in = 0.79788456080286536f * __builtin_fmaf(0.044715f * g * g, g, g);
        const float p = sigmoid(2.f * in);   // (1 + tanh) / 2
        f = g * p;
        df = __builtin_fmaf(2.f * g * p * (1.f - p), 0.79788456080286536f * __builtin_fmaf(0.134145f * g, g, 1.f), p);
    }
}
__device__ __forceinline__ float act_of(int act, float g) {
    float f, df;
    act_and_slope(act, g, f, df);
    return f;
}

// The activation as a constant to f: decided once for all values that f makes, whose
// exponentials then overlap (decided at each value they ran one after the other).
template <class F>
__device__ __forceinline__ void by_act(int act, const F &f) {
    switch (act) {
        case NM_ACT_SILU: f(std::integral_constant<int, NM_ACT_SILU>{}); break;
        case NM_ACT_GELU: f(std::integral_constant<int, NM_ACT_GELU>{}); break;
        case NM_ACT_GELU_TANH: f(std::integral_constant<int, NM_ACT_GELU_TANH>{}); break;
        case NM_ACT_RELU: f(std::integral_constant<int, NM_ACT_RELU>{}); break;
        default: f(std::integral_constant<int, NM_ACT_SIGMOID>{}); break;
    }
}

__device__ __forceinline__ float gate_times(int act, float g, float u) {
    float x = act_of(act, g) * u;
    asm("" : "+v"(x));   // in binary32 before its rounding to T, as scaled_value
    return x;
}

// A tile's rows of the interleaved weight: 16 gate channels, the same 16 up
// channels, the next 16 ...  So fragments 2 i and 2 i + 1 of a wave hold g and u
// of the same channels in the same lanes.
template <class G>
struct HalfTile {
    static constexpr int FN = G::FN / 2, FM = G::FM;
    static constexpr int stage_rows(int eb) { return 16 * FN * eb >= 64 ? 16 : 1024 / (16 * FN * eb); }
    static constexpr int stage_bytes(int eb) { return stage_rows(eb) * (FN * 16 * eb + 16); }
    static_assert(G::FN % 2 == 0 && stage_bytes(2) <= G::STG && stage_bytes(4) <= G::STG, "gated tile");
};

// Two fragments of a wave's channels.
template <class G>
struct PairTile {
    static constexpr int FN = 2, FM = G::FM;
    static constexpr int stage_rows(int eb) { return 16 * FN * eb >= 64 ? 16 : 1024 / (16 * FN * eb); }
    static constexpr int stage_bytes(int eb) { return stage_rows(eb) * (FN * 16 * eb + 16); }
    static_assert(G::FN % 2 == 0 && stage_bytes(2) <= G::STG, "gated tile");
};

// h = T(act(g) * u).  g and u never reach memory: a product of both and an elementwise pass
// after it would write and read 4 m n values more.  18464 x 1024 -> 2736 dense 120 us on the
// tile of nmspmm_rows.h, 1.72 POP/s, with gelu 5 % more; 1576 x 768 -> 2048 13.2 us.
struct GatedOut {
    static __device__ bool scaled(const BlockArgs &) { return true; }
    static __device__ const float *first(const BlockArgs &a) { return a.scale; }
    static __device__ const float *second(const BlockArgs &a) { return a.qscale; }

    template <class G, class Mul>
    static __device__ __forceinline__ void finish(const BlockArgs &a, const TileAt &at,
                                                  const v4i (&acc)[G::FN][G::FM], int8_t *stg, const Mul &multiplier,
                                                  int *) {
        using H = HalfTile<G>;
        float sx[G::FM];
        load_row_scales<G>(a, at, sx);
        v4f h[H::FN][H::FM];
#pragma unroll
        for (int i = 0; i < H::FN; ++i) {
            const v4f cg = multiplier(0, 2 * i), cu = multiplier(0, 2 * i + 1);
            const v4f zero = {0, 0, 0, 0};
            const v4f bg = a.qscale ? multiplier(1, 2 * i) : zero, bu = a.qscale ? multiplier(1, 2 * i + 1) : zero;
#pragma unroll
            for (int j = 0; j < H::FM; ++j) {
                const v4f g = scaled_value(acc[2 * i][j], sx[j], cg, bg);
                const v4f u = scaled_value(acc[2 * i + 1][j], sx[j], cu, bu);
                by_act(a.act, [&](auto act) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) h[i][j][e] = gate_times(decltype(act)::value, g[e], u[e]);
                });
            }
        }
        by_type(a.type, [&](auto *t) {
            using T = typename std::remove_pointer<decltype(t)>::type;
            store_tile<H, T>(
                stg, at.lane, h, at.ch / 2, a.n_out, (a.stream_out & sizeof(T)) != 0,
                [&](int, int, const v4f &v) { return v; },
                [&](int row, T *) -> T * {
                    return at.tok + row < a.m ? (T *)a.out + (int64_t)(at.tok + row) * a.ldo : nullptr;
                });
        });
    }

    template <class G>
    static __device__ __forceinline__ void finish_ks(const BlockArgs &a, const TileAt &at, const int8_t *lds, int *) {
        constexpr int HPR = G::CPR / 2;                            // 4-channel chunks of a row of h
        const int hc = threadIdx.x % HPR, cc = hc / 4 * 8 + hc % 4, ch = at.ch / 2 + hc * 4;
        const int c = at.ch + cc * 4 < a.n ? at.ch + cc * 4 : 0;   // gate; the up channels are 16 rows on
        const v4f zero = {0, 0, 0, 0}, cg = *(const v4f *)(a.scale + c), cu = *(const v4f *)(a.scale + c + 16);
        const v4f bg = a.qscale ? *(const v4f *)(a.qscale + c) : zero;
        const v4f bu = a.qscale ? *(const v4f *)(a.qscale + c + 16) : zero;
        by_type(a.type, [&](auto *t) {
            using T = typename std::remove_pointer<decltype(t)>::type;
            for (int p = threadIdx.x; p < G::BM * HPR; p += 256) {
                const int row = p / HPR, tok = at.tok + row;
                if (tok >= a.m || ch >= a.n_out) continue;
                const float sx = a.row_scale[tok];
                const v4f g = scaled_value(sum_ks<G>(lds, row, cc), sx, cg, bg);
                const v4f u = scaled_value(sum_ks<G>(lds, row, cc + 4), sx, cu, bu);
                v4f h;
                by_act(a.act, [&](auto act) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) h[e] = gate_times(decltype(act)::value, g[e], u[e]);
                });
                store_four<T>(a, tok, ch, h);
            }
        });
    }
};

// A scale as power of two, with its sign, times a value in [1, 2): codes times the
// power are exact in 16 bits, so a product with a scale along the reduction needs no
// rounding but that of the other operand.  0 and NaN: 0 and NaN times 1.
__device__ __forceinline__ float scale_power(float s) {
    return s != s ? s : __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, s) & 0xFF800000u);
}
__device__ __forceinline__ float scale_part(float s) {
    const uint32_t b = __builtin_bit_cast(uint32_t, s) & 0x7FFFFFFFu;
    return b < 0x00800000u || b >= 0x7F800000u ? 1.f : __builtin_bit_cast(float, (b & 0x007FFFFFu) | 0x3F800000u);
}

// Four values of dh from channel ch of a token; zero past the last token and channel.
template <class T>
__device__ __forceinline__ void load_four(const BlockArgs &a, int tok, int ch, float (&f)[4]) {
    typedef T v4t __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = 0.f;
    if (tok >= a.m) return;
    const T *p = (const T *)a.dh + (int64_t)tok * a.lddh + ch;
    if (ch + 4 <= a.n_out) {
        const v4t t = __builtin_bit_cast(v4t, (v2u)(*(const v2u_any *)p));
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = (float)t[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (ch + e < a.n_out) f[e] = (float)p[e];
    }
}

// From the recomputed g and u and dh:  dg = dh u act'(g), du = dh act(g), written
// for the two products that follow, with the part of the scale that their 16-bit
// codes leave out: by rows for dx (times the channel's), transposed for the
// weights' gradients (times the token's).  Their sums over the wave's tokens
// go to bias_parts in binary32.  6304 x 768 -> 2048 bf16 with gelu 60 us: bound by this
// epilogue (act and slope of 12.9 M values, 103 MB written and 26 read); its int8
// products are 11 at the rate of a bare loop of them.
template <class T>
struct GatedGradOut {
    static __device__ bool scaled(const BlockArgs &) { return true; }
    static __device__ const float *first(const BlockArgs &a) { return a.scale; }
    static __device__ const float *second(const BlockArgs &a) { return a.qscale; }

    template <class G, class Mul>
    static __device__ __forceinline__ void finish(const BlockArgs &a, const TileAt &at,
                                                  const v4i (&acc)[G::FN][G::FM], int8_t *stg, const Mul &multiplier,
                                                  int *) {
        // one pair of fragments (the same channels of both projections) at a time: 2 FM
        // fragments of gradients beside the accumulators still to come
        using P = PairTile<G>;
        constexpr int FM = G::FM;
        const int lane = at.lane, lg = lane >> 4, lt = lane & 15;
        float sx[FM];
        load_row_scales<G>(a, at, sx);
        float *parts = a.bias_parts ? a.bias_parts + (int64_t)(at.tok / (FM * 16)) * a.n : nullptr;
#pragma unroll
        for (int i = 0; i < G::FN; i += 2) {
            const v4f zero = {0, 0, 0, 0}, c[2] = {multiplier(0, i), multiplier(0, i + 1)};
            const v4f bg = a.qscale ? multiplier(1, i) : zero, bu = a.qscale ? multiplier(1, i + 1) : zero;
            v4f d[2][FM];
            float dh[FM][4];
#pragma unroll
            for (int j = 0; j < FM; ++j) load_four<T>(a, at.tok + j * 16 + lt, at.ch / 2 + i * 8 + 4 * lg, dh[j]);
            by_act(a.act, [&](auto act) {
#pragma unroll
                for (int j = 0; j < FM; ++j) {
                    const v4f g = scaled_value(acc[i][j], sx[j], c[0], bg);
                    const v4f u = scaled_value(acc[i + 1][j], sx[j], c[1], bu);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float f, df;
                        act_and_slope(decltype(act)::value, g[e], f, df);
                        d[0][j][e] = dh[j][e] * u[e] * df;
                        d[1][j][e] = dh[j][e] * f;
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            });
            // tokens past the last one have no gradient, whatever their row holds
            if (at.tok + FM * 16 > a.m) {
#pragma unroll
                for (int j = 0; j < FM; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool live = at.tok + j * 16 + lt < a.m;
                        d[0][j][e] = live ? d[0][j][e] : 0.f;
                        d[1][j][e] = live ? d[1][j][e] : 0.f;
                    }
            }
            const int ch0 = at.ch + i * 16;
            store_tile<P, T>(
                stg, lane, d, ch0, a.n, false,
                [&](int p, int, const v4f &v) {
                    return v4f{v[0] * scale_part(c[p][0]), v[1] * scale_part(c[p][1]), v[2] * scale_part(c[p][2]),
                               v[3] * scale_part(c[p][3])};
                },
                [&](int row, T *) -> T * {
                    return at.tok + row < a.m ? (T *)a.da + (int64_t)(at.tok + row) * a.n : nullptr;
                });
            // transposed: 16 channels x FM * 16 tokens at a time through the staging area
            constexpr int TROW = FM * 16 * 2 + 16;       // bytes of a staged channel, padded
            constexpr int CPR = FM * 2;                  // 16-byte pieces of it
            static_assert(16 * TROW <= G::STG, "transposed staging");
#pragma unroll
            for (int p = 0; p < 2; ++p) {
#pragma unroll
                for (int j = 0; j < FM; ++j) {
                    const float part = scale_part(sx[j]);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        *(T *)(stg + (4 * lg + e) * TROW + (j * 16 + lt) * 2) = (T)(d[p][j][e] * part);
                }
                for (int q = lane; q < 16 * CPR; q += 64) {
                    const int row = q / CPR, tok = at.tok + (q % CPR) * 8, ch = ch0 + p * 16 + row;
                    const v4i v = *(const v4i *)(stg + row * TROW + (q % CPR) * 16);
                    if (ch < a.n && tok < a.ldt) *(v4i *)((T *)a.dat + (int64_t)ch * a.ldt + tok) = v;
                }
                if (!parts) continue;
                v4f s = d[p][0];
#pragma unroll
                for (int j = 1; j < FM; ++j) s += d[p][j];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x = s[e];
                    x += dpp<0xB1>(0.f, x);
                    x += dpp<0x4E>(0.f, x);
                    x += dpp<0x141>(0.f, x);
                    x += dpp<0x140>(0.f, x);
                    s[e] = x;
                }
                const int ch = ch0 + p * 16 + 4 * lg;
                if (lt == 0 && ch < a.n) *(v4f *)(parts + ch) = s;
            }
        }
    }
};

// T(acc); interleaved rows go to two outputs.  dx and the weights' gradients of 6304 x 768 ->
// 2048 bf16 in one launch 85 us, 933 TFLOP/s; the library's product of the same
// operands takes 43 and 61 one after the other.  With split_k > 1 the splits' sums
// meet in the workspace as in the int8 kernels, added in their order.
template <class T>
struct CastOut {
    static __device__ bool scaled(const BlockArgs &) { return false; }
    static __device__ const float *first(const BlockArgs &) { return nullptr; }
    static __device__ const float *second(const BlockArgs &) { return nullptr; }

    static __device__ __forceinline__ T *row_at(const BlockArgs &a, int row) {
        if (row >= a.m) return nullptr;
        if (!a.interleaved) return (T *)a.out + (int64_t)row * a.ldo;
        const int r = (row >> 5) * 16 + (row & 15);
        return r < a.interleaved ? (T *)((row & 16) ? a.out2 : a.out) + (int64_t)r * a.ldo : nullptr;
    }

    template <class G, class Mul>
    static __device__ __forceinline__ void finish(const BlockArgs &a, const TileAt &at,
                                                  const v4f (&acc)[G::FN][G::FM], int8_t *stg, const Mul &,
                                                  int *s_last) {
        if (a.split_k == 1) {
            store_tile<G, T>(
                stg, at.lane, acc, at.ch, a.n_out, (a.stream_out & sizeof(T)) != 0,
                [&](int, int, const v4f &v) { return v; },
                [&](int row, T *) -> T * { return row_at(a, at.tok + row); });
            return;
        }
        const __amdgpu_buffer_rsrc_t r =
            __builtin_amdgcn_make_buffer_rsrc(a.partials, 0, a.split_k * a.m * a.n * 4, kBufferFlags);
        store_rows<G, 4>(
            stg, at.lane, acc, [&](int, int, const v4f &v, int8_t *dst) { *(v4f *)dst = v; },
            [&](int row, int ch, const v4i &v) {
                if (at.tok + row < a.m && at.ch + ch < a.n)
                    __builtin_amdgcn_raw_buffer_store_b128(
                        __builtin_bit_cast(v4u, v), r, ((at.split * a.m + at.tok + row) * a.n + at.ch + ch) << 2, 0, kSc1);
            });
        if (!arrive_last(a, at.tm * a.tiles_n + at.tn, s_last)) return;
        const int ch = at.ch + at.lane % G::CPR * 4;
        for (int r0 = at.lane / G::CPR; r0 < G::FM * 16; r0 += G::RPI) {
            const int row = at.tok + r0;
            if (row >= a.m || ch >= a.n) continue;
            v4f sum = {0, 0, 0, 0};
#pragma unroll 4
            for (int sp = 0; sp < a.split_k; ++sp)
                sum += __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(
                                                   r, ((sp * a.m + row) * a.n + ch) << 2, 0, kSc1));
            T *p = row_at(a, row);
            if (!p) continue;
            if (ch + 4 <= a.n_out) {
                *(v2u_any *)(p + ch) = pack4_of<T>(sum);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (ch + e < a.n_out) p[ch + e] = (T)sum[e];
            }
        }
    }
};

template <int KIND, int WN, int WM, int FN, int FM, int NST, class EPI>
__global__ __launch_bounds__(64 * WN * WM)
__attribute__((amdgpu_waves_per_eu(Geometry<KIND, WN, WM, FN, FM, NST>::WAVES))) void k_product(BlockArgs a) {
    using G = Geometry<KIND, WN, WM, FN, FM, NST>;
    __shared__ __attribute__((aligned(1024))) int8_t lds[G::LDSB + G::MULB];
    __shared__ uint2 lut[Kind<KIND>::LUT];
    __shared__ int s_last;
    gemm_tile<KIND, WN, WM, FN, FM, NST, EPI>(a, blockIdx.x, gridDim.x, lds, lut, &s_last);
}

template <int KIND, int FN, int FM, int NST, class EPI>
__global__ __launch_bounds__(256) void k_product_ks(BlockArgs a) {
    using G = GeometryKS<KIND, FN, FM, NST>;
    __shared__ __attribute__((aligned(1024))) int8_t lds[G::LDSB];
    __shared__ uint2 lut[Kind<KIND>::LUT];
    __shared__ int s_last;
    gemm_tile_ks<KIND, FN, FM, NST, EPI>(a, lds, lut, &s_last);
}

template <int KIND, class EPI, uint32_t TILES, int T = 0>
int launch_product(int tile, const BlockArgs &a, int grid, void *stream) {
    if constexpr (T < kNumSchedules) {
        if constexpr ((TILES >> T) & 1)
            if (tile == T) {
                constexpr TileCfg t = kTiles[T];
                if constexpr (t.layout == kKSliced)
                    hipLaunchKernelGGL((k_product_ks<KIND, t.fn, t.fm, t.nst, EPI>), dim3(grid), dim3(kThreads), 0,
                                       (hipStream_t)stream, a);
                else
                    hipLaunchKernelGGL((k_product<KIND, t.wn, t.wm, t.fn, t.fm, t.nst, EPI>), dim3(grid),
                                       dim3(64 * t.wn * t.wm), 0, (hipStream_t)stream, a);
                return (int)hipGetLastError();
            }
        return launch_product<KIND, EPI, TILES, T + 1>(tile, a, grid, stream);
    }
    return (int)hipErrorInvalidValue;
}

template <class EPI>
int launch_kinds(int kind, int tile, const BlockArgs &a, int grid, void *stream) {
    switch (kind) {
        case NM_KIND_SP42: return launch_product<NM_KIND_SP42, EPI, scaled_tiles(NM_KIND_SP42)>(tile, a, grid, stream);
        case NM_KIND_C14: return launch_product<NM_KIND_C14, EPI, scaled_tiles(NM_KIND_C14)>(tile, a, grid, stream);
        case NM_KIND_DENSE: return launch_product<NM_KIND_DENSE, EPI, scaled_tiles(NM_KIND_DENSE)>(tile, a, grid, stream);
        case NM_KIND_C18: return launch_product<NM_KIND_C18, EPI, scaled_tiles(NM_KIND_C18)>(tile, a, grid, stream);
        case NM_KIND_C28: return launch_product<NM_KIND_C28, EPI, scaled_tiles(NM_KIND_C28)>(tile, a, grid, stream);
        case NM_KIND_MK3: return launch_product<NM_KIND_MK3, EPI, scaled_tiles(NM_KIND_MK3)>(tile, a, grid, stream);
        case NM_KIND_MK4: return launch_product<NM_KIND_MK4, EPI, scaled_tiles(NM_KIND_MK4)>(tile, a, grid, stream);
        case NM_KIND_MK5: return launch_product<NM_KIND_MK5, EPI, scaled_tiles(NM_KIND_MK5)>(tile, a, grid, stream);
    }
    return (int)hipErrorInvalidValue;
}

}  // namespace
}  // namespace nmspmm
