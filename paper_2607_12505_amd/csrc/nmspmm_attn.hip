// Differential attention, forward: per head two softmax maps over the keys that a
// row sees, o = (p1 - lam p2) v.
//
// One pass over the keys.  The ratio of the maps' sums is not known before the last
// key, so each map has its own running maximum, sum and product with v; both products
// share v's operands.  Scores are made transposed (keys x rows): a lane holds
// keys of one row of q, so maximum and sum are a lane's own but for one exchange of
// halves, and the maps go into the product with v as they lie (nmspmm_attn.h).
// The maps' values are rounded to 16 bits before that product (the matrix instructions
// take no more): half an ulp of each value, the same size as the output's own rounding.
// Sums, maxima and products are in 32 bits.
//
// The rows of a workgroup are those of all heads that share a key head: row (token
// t, head g of the group) is number t * group + g, so shared keys are read once.
#include "nmspmm_attn.h"

namespace nmspmm {
namespace {

// WAVES 4: 128 rows, 32 a wave, share tiles of 64 keys.  WAVES 1: 32 rows, tiles of 32
// keys, for few rows: the keys are split over workgroups, whose sums k_diff_join joins.
template <class T, int D, int DV, int WAVES>
__global__ __launch_bounds__(64 * WAVES, D <= 64 ? 2 : 1) void k_diff_forward(AttnArgs a) {
    constexpr int KT = WAVES == 4 ? kKeyTileWide : kKeyTileNarrow;
    using KTile = Tile<T, D / 8, KT, WAVES>;
    using VTile = Tile<T, DV / 8, KT, WAVES>;
    constexpr int STAGE = 2 * KTile::BYTES + VTile::BYTES;
    __shared__ __attribute__((aligned(1024))) char shared[2 * STAGE];
    const uint32_t lds = lds_start(shared);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);

    // workgroup -> (sequence, key head, row tile, split); long rows of a causal mask first
    int id = near_block(blockIdx.x, gridDim.x);
    const int split = id % a.splits;
    id /= a.splits;
    const int chunk = id % a.chunks;
    id /= a.chunks;
    const int tile = a.row_tiles - 1 - id % a.row_tiles;
    id /= a.row_tiles;
    const int hk = id % a.Hk, b = id / a.Hk;
    const int v0 = chunk * DV, width = a.dv - v0 < DV ? a.dv - v0 : DV;   // its channels of v
    const Sequence s = sequence(a, b);
    const int64_t wide_rows = (int64_t)s.nq * a.group;
    const int64_t start = (int64_t)tile * (32 * WAVES);
    if (start >= wide_rows) return;
    const int rows = (int)(wide_rows - start < 32 * WAVES ? wide_rows - start : 32 * WAVES);

    // this lane's row; lanes behind the last row repeat it and store nothing
    const int mine = wave * 32 + (lane & 31);
    const bool valid = mine < rows;
    const int64_t number = start + (valid ? mine : rows - 1);
    const int t = (int)(number / a.group), g = (int)(number - (int64_t)t * a.group), head = hk * a.group + g;
    const int first = first_seen(a, s, t), last = last_seen(a, s, t);
    // what the wave's and the workgroup's rows see: rows rise with t, and so do both ends
    const int wave_low = __builtin_amdgcn_readlane(first, 0), wave_full = __builtin_amdgcn_readlane(first, 31);
    const int wave_end = __builtin_amdgcn_readlane(last, 0);
    const int wave_high = wave * 32 < rows ? __builtin_amdgcn_readlane(last, 31) : -1;
    const int low = first_seen(a, s, (int)(start / a.group));
    const int high = last_seen(a, s, (int)((start + rows - 1) / a.group));
    int tile0 = low / KT, tiles = high >= low ? high / KT + 1 - tile0 : 0;
    {   // this split's part of them
        const int from = (int)((int64_t)tiles * split / a.splits), to = (int)((int64_t)tiles * (split + 1) / a.splits);
        tile0 += from;
        tiles = to - from;
    }

    const T *kp = head_of<T>(a.k, s.batch, s.k0, 2 * hk), *vp = head_of<T>(a.v, s.batch, s.k0, hk) + v0;
    auto stage = [&](int n) {
        const int64_t j = (int64_t)(tile0 + n) * KT;
        const uint32_t to = lds + (n & 1) * STAGE;
        const int left = (int)(s.nk - j);
        KTile::load(kp + j * a.k.token, a.k.token, left, a.d, a.vec, to, wave, lane);
        KTile::load(kp + a.k.head + j * a.k.token, a.k.token, left, a.d, a.vec, to + KTile::BYTES, wave, lane);
        VTile::load(vp + j * a.v.token, a.v.token, left, width, a.vec, to + 2 * KTile::BYTES, wave, lane);
    };
    if (tiles > 0) stage(0);

    v8s q[2][D / 16];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
            q[i][c] = row_operand(head_of<T>(a.q, s.batch, s.q0 + t, 2 * head + i), valid, c, a.d, a.vec, lane);

    v16f o[2][DV / 32];
    float top[2], sum[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        top[i] = -__builtin_inff();
        sum[i] = 0.f;
#pragma unroll
        for (int x = 0; x < DV / 32; ++x) o[i][x] = v16f{};
    }

    for (int n = 0; n < tiles; ++n) {
        arrive();
        if (n + 1 < tiles) stage(n + 1);
        const uint32_t kt = lds + (n & 1) * STAGE, vt = kt + 2 * KTile::BYTES;
#pragma unroll 1
        for (int kb = 0; kb < KT; kb += 32) {
            const int j0 = (tile0 + n) * KT + kb;
            if (j0 > wave_high || j0 + 31 < wave_low) continue;
            v16f z[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                z[i] = v16f{};
#pragma unroll
                for (int c = 0; c < D / 16; ++c)
                    z[i] = Mfma<T>::mul(KTile::rows(kt + i * KTile::BYTES, kb, c, lane), q[i][c], z[i]);
            }
            if (j0 + 31 > wave_end || j0 < wave_full) {
                const int at = j0 + 4 * (lane >> 5);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int j = at + 8 * (e / 4) + e % 4;
                    const bool seen = j >= first && j <= last;
                    z[0][e] = seen ? z[0][e] : -__builtin_inff();
                    z[1][e] = seen ? z[1][e] : -__builtin_inff();
                }
            }
            // The maximum that the exponents are taken from follows the true one only when that has
            // grown by more than 2^8: a value is then at most 2^8, which 16 bits and the sums hold.  Each
            // row by itself: its bits do not depend on the rows beside it.
            float now[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float m = z[i][0];
#pragma unroll
                for (int e = 1; e < 16; ++e) m = fmaxf(m, z[i][e]);
                now[i] = half_max(m) * a.scale2;
            }
            if (__any(now[0] > top[0] + 8.f || now[1] > top[1] + 8.f)) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const bool grown = now[i] > top[i] + 8.f;
                    const float f = grown ? __builtin_amdgcn_exp2f(top[i] - now[i]) : 1.f;
                    top[i] = grown ? now[i] : top[i];
                    sum[i] *= f;
#pragma unroll
                    for (int x = 0; x < DV / 32; ++x) o[i][x] *= f;
                }
            }
            v8s p[2][2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float from = top[i] == -__builtin_inff() ? 0.f : top[i];
                float f[16], part = 0.f;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    f[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[i][e], a.scale2, -from));
                    part += f[e];
                }
                sum[i] += part;
                p[i][0] = pack<T>(f, 0);
                p[i][1] = pack<T>(f, 1);
            }
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int x = 0; x < DV / 32; ++x) {
                    const v8s w = VTile::turned(vt, kb + 16 * c, x, lane);
                    o[0][x] = Mfma<T>::mul(w, p[0][c], o[0][x]);
                    o[1][x] = Mfma<T>::mul(w, p[1][c], o[1][x]);
                }
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) sum[i] = half_sum(sum[i]);

    if (a.splits > 1) {
        if (!valid) return;
        // rows of a part: [sequence][key head][split][number]
        const int64_t part = (((int64_t)b * a.Hk + hk) * a.splits + split) * ((int64_t)a.tq * a.group) + number;
        float *ml = a.parts + (int64_t)a.batch * a.Hk * a.splits * a.tq * a.group * 2 * a.dv + part * 4;
        if (lane < 32 && chunk == 0) *(v4f *)ml = v4f{top[0], sum[0], top[1], sum[1]};
        const bool vec = a.dv % 4 == 0;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int x = 0; x < DV / 32; ++x)
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                    store4(a.parts + (part * 2 + i) * a.dv + v0, 32 * x + 2 * e + 4 * (lane >> 5), width, vec, o[i][x][e],
                           o[i][x][e + 1], o[i][x][e + 2], o[i][x][e + 3]);
        return;
    }
    float lam = 0.f;
    for (int k = 0; k < a.group; ++k) {   // the whole wave makes each head's weight
        const float w = weight_of(a.weight, hk * a.group + k, lane).lam;
        lam = k == g ? w : lam;
    }
    if (!valid) return;
    const float f1 = sum[0] == 0.f ? 0.f : 1.f / sum[0], f2 = sum[1] == 0.f ? 0.f : 1.f / sum[1];
    T *op = head_of<T>(a.o, s.batch, s.q0 + t, head) + v0;
#pragma unroll
    for (int x = 0; x < DV / 32; ++x) {
        o[0][x] *= f1;
        o[1][x] *= f2;
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const int c = 32 * x + 2 * e + 4 * (lane >> 5);
            float y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = o[0][x][e + j] - lam * o[1][x][e + j];
            store4(op, c, width, a.vec_out, y[0], y[1], y[2], y[3]);
        }
    }
    if (!a.kept) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float most = 0.f;
#pragma unroll
        for (int x = 0; x < DV / 32; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e) most = larger(most, magnitude(o[i][x][e]));
        most = larger(most, __shfl_xor(most, 32));
        const KeptScale k = kept_scale(most);
        int16_t *to = a.kept + (((s.row0 + t) * a.H + head) * 2 + i) * a.dv + v0;
        const bool vec = a.dv % 4 == 0;
#pragma unroll
        for (int x = 0; x < DV / 32; ++x)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int c = 32 * x + 2 * e + 4 * (lane >> 5);
                const v4s q4 = {kept_code(o[i][x][e], k.inv), kept_code(o[i][x][e + 1], k.inv),
                                kept_code(o[i][x][e + 2], k.inv), kept_code(o[i][x][e + 3], k.inv)};
                if (vec) {
                    if (c < width) *(v4s *)(to + c) = q4;
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (c + j < width) to[c + j] = q4[j];
                }
            }
        if (lane < 32) {
            float *at = a.stats + (2 * (int64_t)head + i) * a.stat_rows * a.rows + s.row0 + t;
            if (chunk == 0) at[0] = sum[i] == 0.f ? __builtin_inff() : top[i] + __builtin_amdgcn_logf(sum[i]);
            at[(1 + chunk) * a.rows] = k.scale;
        }
    }
}

// The splits' sums of one row and head, a wave each:  M = max of m_s,
// o_i = sum of 2^(m_s - M) O_s / sum of 2^(m_s - M) l_s.
template <class T>
__global__ __launch_bounds__(256) void k_diff_join(AttnArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t wide = (int64_t)a.tq * a.group, all = (int64_t)a.batch * a.Hk * wide;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= all) return;
    const int64_t number = row % wide, outer = row / wide;
    const int hk = (int)(outer % a.Hk), b = (int)(outer / a.Hk);
    const int t = (int)(number / a.group), head = hk * a.group + (int)(number - (int64_t)t * a.group);
    const Sequence s = sequence(a, b);
    if (t >= s.nq) return;
    const float *ml = a.parts + all * a.splits * 2 * a.dv;
    const int64_t part = outer * a.splits * wide + number;
    float top[2] = {-__builtin_inff(), -__builtin_inff()}, sum[2] = {0.f, 0.f};
    for (int n = 0; n < a.splits; ++n) {
        const v4f m = *(const v4f *)(ml + (part + n * wide) * 4);
        top[0] = fmaxf(top[0], m[0]);
        top[1] = fmaxf(top[1], m[2]);
    }
    const float lam = weight_of(a.weight, head, lane).lam;
    T *op = head_of<T>(a.o, s.batch, s.q0 + t, head);
    float y[2][kMaxValueWidth / 64];
#pragma unroll
    for (int n = 0; n < kMaxValueWidth / 64; ++n) y[0][n] = y[1][n] = 0.f;
    for (int n = 0; n < a.splits; ++n) {
        const v4f m = *(const v4f *)(ml + (part + n * wide) * 4);
        const float *p = a.parts + (part + n * wide) * 2 * a.dv;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (m[2 * i + 1] == 0.f) continue;     // a split that saw no key
            const float f = __builtin_amdgcn_exp2f(m[2 * i] - top[i]);
            sum[i] += f * m[2 * i + 1];
#pragma unroll
            for (int x = 0; x < kMaxValueWidth / 64; ++x)
                if (lane + 64 * x < a.dv) y[i][x] += f * p[i * a.dv + lane + 64 * x];
        }
    }
#pragma unroll
    for (int x = 0; x < kMaxValueWidth / 64; ++x) {
#pragma unroll
        for (int i = 0; i < 2; ++i) y[i][x] = sum[i] == 0.f ? 0.f : y[i][x] / sum[i];
        if (lane + 64 * x < a.dv) op[lane + 64 * x] = (T)(y[0][x] - lam * y[1][x]);
    }
    if (!a.kept) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float *at = a.stats + (2 * (int64_t)head + i) * a.stat_rows * a.rows + s.row0 + t;
        if (lane == 0) at[0] = sum[i] == 0.f ? __builtin_inff() : top[i] + __builtin_amdgcn_logf(sum[i]);
        int16_t *to = a.kept + (((s.row0 + t) * a.H + head) * 2 + i) * a.dv;
#pragma unroll
        for (int c = 0; c < kMaxValueWidth / kScaleWidth; ++c) {
            if (c * kScaleWidth >= a.dv) break;
            const KeptScale k = kept_scale(wave_largest(larger(magnitude(y[i][2 * c]), magnitude(y[i][2 * c + 1]))));
            if (lane == 0) at[(1 + c) * a.rows] = k.scale;
#pragma unroll
            for (int x = 2 * c; x < 2 * c + 2; ++x)
                if (lane + 64 * x < a.dv) to[lane + 64 * x] = kept_code(y[i][x], k.inv);
        }
    }
}

template <class T, int WAVES>
int forward(int cls, const AttnArgs &a, hipStream_t s) {
    const dim3 grid((unsigned)((int64_t)a.batch * a.Hk * a.row_tiles * a.chunks * a.splits)), block(64 * WAVES);
    if (cls == 0)
        hipLaunchKernelGGL((k_diff_forward<T, 32, 64, WAVES>), grid, block, 0, s, a);
    else if (cls == 1)
        hipLaunchKernelGGL((k_diff_forward<T, 64, 128, WAVES>), grid, block, 0, s, a);
    else
        hipLaunchKernelGGL((k_diff_forward<T, 128, 128, WAVES>), grid, block, 0, s, a);
    return (int)hipGetLastError();
}

}  // namespace

int launch_diff_forward(int type, int cls, bool wide, const AttnArgs &a, void *stream) {
    const hipStream_t s = (hipStream_t)stream;
    if (type == NM_TYPE_F16) return wide ? forward<half_t, 4>(cls, a, s) : forward<half_t, 1>(cls, a, s);
    return wide ? forward<bf16_t, 4>(cls, a, s) : forward<bf16_t, 1>(cls, a, s);
}

int launch_diff_join(int type, const AttnArgs &a, void *stream) {
    const int64_t rows = (int64_t)a.batch * a.Hk * a.tq * a.group;
    const dim3 grid((unsigned)((rows + 3) / 4));
    if (type == NM_TYPE_F16)
        hipLaunchKernelGGL(k_diff_join<half_t>, grid, dim3(256), 0, (hipStream_t)stream, a);
    else
        hipLaunchKernelGGL(k_diff_join<bf16_t>, grid, dim3(256), 0, (hipStream_t)stream, a);
    return (int)hipGetLastError();
}

}  // namespace nmspmm
