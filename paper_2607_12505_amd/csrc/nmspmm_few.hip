// Scaled int8 products (plain or gated) of few tokens, bound by reading the
// weight once: every workgroup streams 16 output channels (gated: of both
// projections) from memory straight into the registers that the matrix
// instruction reads, its 8 waves taking the k-steps in turn, and the 8 partial
// sums meet in LDS.  A wave keeps 4 k-steps of weights in flight, 64 KB a compute
// unit, which covers the memory's latency; LDS holds no weight, so there is no
// barrier before the sums.  The sums are integers: a token has the same bits
// here and in a large batch.
//
// Activations come as codes (each wave reads its own k-steps of them, from L2),
// or, for the few tokens whose values fit 16 a thread, as values: every workgroup
// then makes the codes itself, in LDS, while its first weights are on their
// way.  That repeats a row's codes once for each 16 channels, and saves a launch.
//
// Measured: one token as values, dense 1024 -> 4096 4.3 us, gated 1024 -> 2736 (twice the
// weight rows) 4.8 us.  A token's weights are 4 to 6 MB, under 1 us at the memory's rate: what is
// left is the launch, the wait for x and the weights one after the other, and the sums.  From
// codes, weights from memory: dense 4096 -> 4096, 17 MB, 6.3 us (2.7 TB/s); 4:8 4096 ->
// 11008, 28 MB as stored, 8.6 us (3.3 TB/s).
#include "nmspmm_products.h"

namespace nmspmm {
namespace {

constexpr int kFewWaves = 8, kAhead = 4;

// A lane's weights of one (fragment, k-step), as stored.
template <int KIND>
struct FewOperand {
    WRegs<KIND> r;
};
template <>
struct FewOperand<NM_KIND_DENSE> {
    v4i lo, hi;
};

template <class T>
__device__ __forceinline__ void few_values(const void *x, int64_t at, float (&f)[8]) {
    const Raw8<T> t = load8((const T *)x + at);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (float)t.v[e];
}

// Codes of m rows of x (k a multiple of 8, at most 8 * kFewCodes * 512 values in
// all) into LDS rows of `pitch` bytes, zeros from k on, and their scales.
constexpr int kFewCodes = 2;
__device__ __forceinline__ void few_codes(const BlockArgs &a, int8_t *xs, int pitch, float *scales, uint32_t *tops) {
    const int tid = threadIdx.x, per = a.kx / 8, chunks = a.m * per;
    float f[kFewCodes][8];
    if (tid < 16) tops[tid] = 0;
    // the padding: from k to the end of the last k-step
    for (int i = tid; i < a.m * ((pitch - a.kx) / 8); i += kFewWaves * 64) {
        const int row = i / ((pitch - a.kx) / 8), c = i % ((pitch - a.kx) / 8);
        *(v2u *)(xs + row * pitch + a.kx + c * 8) = v2u{0, 0};
    }
#pragma unroll
    for (int i = 0; i < kFewCodes; ++i) {
        const int c = tid + i * kFewWaves * 64;
        if (c >= chunks) break;
        const int64_t at = (int64_t)(c / per) * a.ldx + (c % per) * 8;
        if (a.xtype == NM_TYPE_F16)
            few_values<half_t>(a.x, at, f[i]);
        else if (a.xtype == NM_TYPE_BF16)
            few_values<bf16_t>(a.x, at, f[i]);
        else
            few_values<float>(a.x, at, f[i]);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kFewCodes; ++i) {
        const int c0 = (tid & ~63) + i * kFewWaves * 64, c = tid + i * kFewWaves * 64;   // the wave's first chunk
        if (c0 >= chunks) break;
        float top = 0.f;
        if (c < chunks) {
#pragma unroll
            for (int e = 0; e < 8; ++e) top = larger(top, magnitude(f[i][e]));
        }
        const int last = c0 + 63 < chunks ? c0 + 63 : chunks - 1;
        if (c0 / per == last / per) {          // the wave's chunks are of one row
            top = wave_largest(top);
            if ((tid & 63) == 0) atomicMax(tops + c0 / per, __builtin_bit_cast(uint32_t, top));
        } else if (c < chunks) {
            atomicMax(tops + c / per, __builtin_bit_cast(uint32_t, top));
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kFewCodes; ++i) {
        const int c = tid + i * kFewWaves * 64;
        if (c >= chunks) break;
        const int row = c / per;
        const RowScale rs = row_scale(__builtin_bit_cast(float, tops[row]));
        if (c % per == 0) scales[row] = rs.scale;
        int q[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = row_code(f[i][e], rs.inv);
        *(v2u *)(xs + row * pitch + (c % per) * 8) = v2u{pack4(q[0], q[1], q[2], q[3]), pack4(q[4], q[5], q[6], q[7])};
    }
    __syncthreads();
}

// FN: 1, or 2 for the gate's and the up projection's fragments of the same
// channels; FM: 16-token fragments; CODES: activations come as codes.
template <int KIND, int FN, int FM, bool CODES>
__global__ __launch_bounds__(64 * kFewWaves) void k_few(BlockArgs a) {
    using K = Kind<KIND>;
    constexpr bool kDense = KIND == NM_KIND_DENSE, kMask = K::NV > 0;
    // the codes, then the partial sums; m * k <= 8192 codes and at most 136 bytes of padding a row
    constexpr int kSums = kFewWaves * FM * FN * 1024, kCodes = CODES ? 0 : 8 * kFewCodes * 64 * kFewWaves + 16 * 136;
    __shared__ __attribute__((aligned(16))) int8_t lds[kSums > kCodes ? kSums : kCodes];
    __shared__ uint2 lut[K::LUT];
    __shared__ float scales[16];
    __shared__ uint32_t tops[16];
    const int tid = threadIdx.x, lane = tid & 63, lg = lane >> 4, lt = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int f0 = blockIdx.x * FN;
    const int steps = a.k_steps > wave ? (a.k_steps - wave + kFewWaves - 1) / kFewWaves : 0;   // this wave's k-steps

    // --- weights: k-step wave + 8 t of fragment f0 + i
    FewOperand<KIND> w[kAhead][FN];
    const int8_t *wrow[FN];
    int64_t meta0[FN];
#pragma unroll
    for (int i = 0; i < FN; ++i) {
        if constexpr (kDense) {
            const int row = (f0 + i) * 16 + lt;
            wrow[i] = a.A + (int64_t)(row < a.n ? row : a.n - 1) * a.k;
        } else {
            const int64_t block = (int64_t)(f0 + i) * a.k_steps;
            wrow[i] = a.A + (block * 64 + lane) * K::VB;
            meta0[i] = (block * 64 + lane) * K::MB;
        }
    }
    auto load = [&](int t, FewOperand<KIND> (&o)[FN]) {
        const int s = wave + kFewWaves * t;
#pragma unroll
        for (int i = 0; i < FN; ++i) {
            if constexpr (kDense) {
                // past k (only in the last k-step) the row's last chunk instead: its codes are zero there
                const int c = s * 128 + lg * 16;
                o[i].lo = *(const v4i *)(wrow[i] + (c < a.k ? c : a.k - 16));
                o[i].hi = *(const v4i *)(wrow[i] + (c + 64 < a.k ? c + 64 : a.k - 16));
            } else {
                wload<KIND>(o[i].r, wrow[i] + (int64_t)s * 64 * K::VB, a.meta + meta0[i] + (int64_t)s * 64 * K::MB);
            }
        }
    };
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
        if (u < steps) load(u, w[u]);
    fill_lut<KIND>(lut, tid, 64 * kFewWaves);

    const int pitch = a.k_steps * 128 + 16;
    if constexpr (!CODES)
        few_codes(a, lds, pitch, scales, tops);
    else if constexpr (K::LUT > 1)
        __syncthreads();

    v4i acc[FN][FM];
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) acc[i][j] = v4i{0, 0, 0, 0};

    // --- the wave's k-steps.  A lane's columns: 16 lg and 64 + 16 lg as the
    // instructions order them, or its own 32 for the mask layouts.
    const int c0 = (kMask ? 2 * lg : lg) * 16, c1 = (kMask ? 2 * lg + 1 : lg + 4) * 16;
    auto multiply = [&](int t, const FewOperand<KIND> (&o)[FN]) {
        const int col = (wave + kFewWaves * t) * 128;
        v4i lo[FN], hi[FN];
        int idx[FN];
#pragma unroll
        for (int i = 0; i < FN; ++i) {
            if constexpr (kDense) {
                lo[i] = o[i].lo;
                hi[i] = o[i].hi;
            } else if constexpr (KIND == NM_KIND_SP42) {
                lo[i] = v4i{(int)o[i].r.v[0], (int)o[i].r.v[1], (int)o[i].r.v[2], (int)o[i].r.v[3]};
                idx[i] = (int)o[i].r.m;
            } else if constexpr (K::kSp) {
                uint32_t x;
                expand_sp42<KIND>(o[i].r, lut, lo[i], x);
                idx[i] = (int)x;
            } else {
                expand_dense<KIND>(o[i].r, lut, lo[i], hi[i]);
            }
        }
#pragma unroll
        for (int j = 0; j < FM; ++j) {
            const int tok = 16 * j + lt < a.m ? 16 * j + lt : a.m - 1;
            v4i xlo = {0, 0, 0, 0}, xhi = {0, 0, 0, 0};
            if constexpr (CODES) {
                const int8_t *row = a.X + (int64_t)tok * a.k + col;
                if (col + c0 < a.k) xlo = *(const v4i *)(row + c0);
                if (col + c1 < a.k) xhi = *(const v4i *)(row + c1);
            } else {
                xlo = *(const v4i *)(lds + tok * pitch + col + c0);
                xhi = *(const v4i *)(lds + tok * pitch + col + c1);
            }
            const v8i x = {xlo[0], xlo[1], xlo[2], xlo[3], xhi[0], xhi[1], xhi[2], xhi[3]};
#pragma unroll
            for (int i = 0; i < FN; ++i) {
                if constexpr (K::kSp) {
                    acc[i][j] = __builtin_amdgcn_smfmac_i32_16x16x128_i8(lo[i], x, acc[i][j], idx[i], 0, 0);
                } else {
                    acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(lo[i], xlo, acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(hi[i], xhi, acc[i][j], 0, 0, 0);
                }
            }
        }
    };
    for (int t0 = 0; t0 < steps; t0 += kAhead)
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (t0 + u < steps) {
                multiply(t0 + u, w[u]);
                if (t0 + u + kAhead < steps) load(t0 + u + kAhead, w[u]);
            }

    // --- the waves' sums, then 4 channels of one token a thread
    if constexpr (!CODES) __syncthreads();     // every wave has read its codes
    v4i *sums = (v4i *)lds;
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) sums[((wave * FM + j) * FN + i) * 64 + lane] = acc[i][j];
    __syncthreads();
    if (wave >= FM) return;
    const int tok = wave * 16 + lt;
    if (tok >= a.m) return;
    const float sx = CODES ? a.row_scale[tok] : scales[tok];
    v4f v[FN];
#pragma unroll
    for (int i = 0; i < FN; ++i) {
        v4i s = {0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < kFewWaves; ++u) s += sums[((u * FM + wave) * FN + i) * 64 + lane];
        const int ch = (f0 + i) * 16 + 4 * lg < a.n ? (f0 + i) * 16 + 4 * lg : 0;
        v[i] = scaled_value(s, sx, *(const v4f *)(a.scale + ch),
                            a.qscale ? *(const v4f *)(a.qscale + ch) : v4f{0, 0, 0, 0});
    }
    int ch = f0 * 16 + 4 * lg;
    if constexpr (FN == 2) {
        ch = blockIdx.x * 16 + 4 * lg;
        by_act(a.act, [&](auto act) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[0][e] = gate_times(decltype(act)::value, v[0][e], v[1][e]);
        });
    }
    by_type(a.type, [&](auto *p) {
        using T = typename std::remove_pointer<decltype(p)>::type;
        store_four<T>(a, tok, ch, v[0]);
    });
}

template <int KIND, int FN, int FM, bool CODES>
int few_one(const BlockArgs &a, void *stream) {
    hipLaunchKernelGGL((k_few<KIND, FN, FM, CODES>), dim3((a.n_frags + FN - 1) / FN), dim3(64 * kFewWaves), 0,
                       (hipStream_t)stream, a);
    return (int)hipGetLastError();
}
template <int KIND, int FN>
int few_shape(const BlockArgs &a, void *stream) {
    if (a.x) return few_one<KIND, FN, 1, false>(a, stream);
    if (a.m <= 16) return few_one<KIND, FN, 1, true>(a, stream);
    return few_one<KIND, FN, kFewTokens / 16, true>(a, stream);
}
template <int KIND>
int few_kind(bool gated, const BlockArgs &a, void *stream) {
    return gated ? few_shape<KIND, 2>(a, stream) : few_shape<KIND, 1>(a, stream);
}

}  // namespace

// Values: up to 8192 of them.  At 16384 (m 4, k 4096) one launch took 7.2 us against
// 5.7 to 6.5 for the codes and the product; at 4096 2.7 to 3.3 us against 5.
bool few_takes_values(int m, int k) { return m <= 16 && k % 8 == 0 && (int64_t)m * (k / 8) <= kFewCodes * 64 * kFewWaves; }

int launch_few(int kind, bool gated, const BlockArgs &a, void *stream) {
    switch (kind) {
        case NM_KIND_SP42: return few_kind<NM_KIND_SP42>(gated, a, stream);
        case NM_KIND_C14: return few_kind<NM_KIND_C14>(gated, a, stream);
        case NM_KIND_DENSE: return few_kind<NM_KIND_DENSE>(gated, a, stream);
        case NM_KIND_C18: return few_kind<NM_KIND_C18>(gated, a, stream);
        case NM_KIND_C28: return few_kind<NM_KIND_C28>(gated, a, stream);
        case NM_KIND_MK3: return few_kind<NM_KIND_MK3>(gated, a, stream);
        case NM_KIND_MK4: return few_kind<NM_KIND_MK4>(gated, a, stream);
        case NM_KIND_MK5: return few_kind<NM_KIND_MK5>(gated, a, stream);
    }
    return (int)hipErrorInvalidValue;
}

}  // namespace nmspmm
