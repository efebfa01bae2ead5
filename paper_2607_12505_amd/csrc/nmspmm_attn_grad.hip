// Differential attention's backward pass, from do (dp = do v^T, D_i = sum over keys of p_i dp):
//   dv   = (p1 - lam p2)^T do
//   ds1  = p1 (dp - D1),  ds2 = -lam p2 (dp - D2)
//   dq_i = scale ds_i k_i,  dk_i = scale ds_i^T q_i,  dlam = -sum over rows of D2
// The maps are made again from the scores and the forward pass's logarithms of their sums.
// D1 and D2 enter ds as do . (p_i v), of the codes that the forward pass kept: 16 bits with a
// scale for each row, 2^-16 of its largest value.  (Products rounded to the type, and the output among
// them, put dq and dk at up to 2.5 times the error of a form in 32 bits.)  dlam takes the sums of p2 dp
// themselves, in 32 bits.
// ds and p1 - lam p2 are rounded to 16 bits once, for the matrix instructions.
//
// Two kernels, each with its sums in registers in a fixed order: one over keys for the
// rows of q (which also makes D1, D2 and the parts of dlam), one over rows for the
// keys.  The second makes scores and dp again: 512 of 1792 operations a pair at width
// 64 + 128, against sums of dq in memory by atomics, whose order would change results.
#include "nmspmm_attn.h"

namespace nmspmm {
namespace {

// dq, D1, D2 and the parts of dlam: rows as in the forward pass, scores transposed, so a
// lane's keys are of one row and ds is the operand of dq as it lies.
template <class T, int D, int DV>
__global__ __launch_bounds__(256, DV <= 128 ? 2 : 1) void k_diff_grad_q(AttnArgs a) {
    constexpr int KT = kKeyTileWide;
    using KTile = Tile<T, D / 8, KT, 4>;
    using VTile = Tile<T, DV / 8, KT, 4>;
    constexpr int STAGE = 2 * KTile::BYTES + VTile::BYTES;
    __shared__ __attribute__((aligned(1024))) char shared[2 * STAGE];
    const uint32_t lds = lds_start(shared);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    int id = near_block(blockIdx.x, gridDim.x);
    const int tile = a.row_tiles - 1 - id % a.row_tiles;
    id /= a.row_tiles;
    const int hk = id % a.Hk, b = id / a.Hk;
    const Sequence s = sequence(a, b);
    const int64_t wide_rows = (int64_t)s.nq * a.group;
    const int64_t start = (int64_t)tile * 128;
    float *lam_part = a.dlam_parts + (int64_t)hk * a.group * a.dlam_count + ((int64_t)b * a.row_tiles + tile) * 4 + wave;
    if (start >= wide_rows) {
        for (int k = lane; k < a.group; k += 64) lam_part[(int64_t)k * a.dlam_count] = 0.f;
        return;
    }
    const int rows = (int)(wide_rows - start < 128 ? wide_rows - start : 128);
    const int mine = wave * 32 + (lane & 31);
    const bool valid = mine < rows;
    const int64_t number = start + (valid ? mine : rows - 1);
    const int t = (int)(number / a.group), g = (int)(number - (int64_t)t * a.group), head = hk * a.group + g;
    const int first = first_seen(a, s, t), last = last_seen(a, s, t);
    const int wave_low = __builtin_amdgcn_readlane(first, 0), wave_full = __builtin_amdgcn_readlane(first, 31);
    const int wave_end = __builtin_amdgcn_readlane(last, 0);
    const int wave_high = wave * 32 < rows ? __builtin_amdgcn_readlane(last, 31) : -1;
    const int low = first_seen(a, s, (int)(start / a.group));
    const int high = last_seen(a, s, (int)((start + rows - 1) / a.group));
    const int tile0 = low / KT, tiles = high >= low ? high / KT + 1 - tile0 : 0;

    const T *kp = head_of<T>(a.k, s.batch, s.k0, 2 * hk), *vp = head_of<T>(a.v, s.batch, s.k0, hk);
    auto stage = [&](int n) {
        const int64_t j = (int64_t)(tile0 + n) * KT;
        const uint32_t to = lds + (n & 1) * STAGE;
        const int left = (int)(s.nk - j);
        KTile::load(kp + j * a.k.token, a.k.token, left, a.d, a.vec, to, wave, lane);
        KTile::load(kp + a.k.head + j * a.k.token, a.k.token, left, a.d, a.vec, to + KTile::BYTES, wave, lane);
        VTile::load(vp + j * a.v.token, a.v.token, left, a.dv, a.vec, to + 2 * KTile::BYTES, wave, lane);
    };
    if (tiles > 0) stage(0);

    v8s q[2][D / 16], grad[DV / 16];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
            q[i][c] = row_operand(head_of<T>(a.q, s.batch, s.q0 + t, 2 * head + i), valid, c, a.d, a.vec, lane);
    float lam = 0.f;
    for (int k = 0; k < a.group; ++k) {
        const float w = weight_of(a.weight, hk * a.group + k, lane).lam;
        lam = k == g ? w : lam;
    }
    float d[2], lse[2];
    {
        typedef T v8 __attribute__((ext_vector_type(8)));
        const T *gp = head_of<T>(a.grad, s.batch, s.q0 + t, head);
        const int16_t *kept = a.kept + ((s.row0 + t) * a.H + head) * 2 * a.dv;
        float sums[2][(DV + kScaleWidth - 1) / kScaleWidth] = {};
#pragma unroll
        for (int c = 0; c < DV / 16; ++c) {
            grad[c] = row_operand(gp, valid, c, a.dv, a.vec, lane);
            const v8 x = __builtin_bit_cast(v8, grad[c]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const v8s y = row_operand(kept + i * a.dv, valid, c, a.dv, a.dv % 8 == 0, lane);
#pragma unroll
                for (int e = 0; e < 8; ++e) sums[i][c * 16 / kScaleWidth] += (float)x[e] * (float)y[e];
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t at = (2 * (int64_t)head + i) * a.stat_rows * a.rows + s.row0 + t;
            lse[i] = a.stats[at];
            d[i] = 0.f;
#pragma unroll
            for (int c = 0; c < (DV + kScaleWidth - 1) / kScaleWidth; ++c)
                if (c * kScaleWidth < a.dv) d[i] += half_sum(sums[i][c]) * a.stats[at + (1 + c) * a.rows];
            if (valid && lane < 32) a.delta[(2 * (int64_t)head + i) * a.rows + s.row0 + t] = d[i];
        }
    }
    v16f dq[2][D / 32];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int x = 0; x < D / 32; ++x) dq[i][x] = v16f{};
    float second = 0.f;   // sum of p2 dp over this lane's keys

    for (int n = 0; n < tiles; ++n) {
        arrive();
        if (n + 1 < tiles) stage(n + 1);
        const uint32_t kt = lds + (n & 1) * STAGE, vt = kt + 2 * KTile::BYTES;
#pragma unroll 1
        for (int kb = 0; kb < KT; kb += 32) {
            const int j0 = (tile0 + n) * KT + kb;
            if (j0 > wave_high || j0 + 31 < wave_low) continue;
            v16f z[2], dp = v16f{};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                z[i] = v16f{};
#pragma unroll
                for (int c = 0; c < D / 16; ++c)
                    z[i] = Mfma<T>::mul(KTile::rows(kt + i * KTile::BYTES, kb, c, lane), q[i][c], z[i]);
            }
#pragma unroll
            for (int c = 0; c < DV / 16; ++c) dp = Mfma<T>::mul(VTile::rows(vt, kb, c, lane), grad[c], dp);
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
            float ds1[16], ds2[16], part = 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[0][e], a.scale2, -lse[0]));
                const float p2 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[1][e], a.scale2, -lse[1]));
                part = __builtin_fmaf(p2, dp[e], part);
                ds1[e] = p1 * (dp[e] - d[0]);
                ds2[e] = p2 * (dp[e] - d[1]);
            }
            second += part;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const v8s b1 = pack<T>(ds1, c), b2 = pack<T>(ds2, c);
#pragma unroll
                for (int x = 0; x < D / 32; ++x) {
                    dq[0][x] = Mfma<T>::mul(KTile::turned(kt, kb + 16 * c, x, lane), b1, dq[0][x]);
                    dq[1][x] = Mfma<T>::mul(KTile::turned(kt + KTile::BYTES, kb + 16 * c, x, lane), b2, dq[1][x]);
                }
            }
        }
    }
    if (!valid) second = 0.f;
    for (int k = 0; k < a.group; ++k) {
        const float w = wave_sum(g == k ? second : 0.f);
        if (lane == 0) lam_part[(int64_t)k * a.dlam_count] = w;
    }
    if (!valid) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        T *out = head_of<T>(a.dq, s.batch, s.q0 + t, 2 * head + i);
        const float f = i ? -lam * a.scale : a.scale;
#pragma unroll
        for (int x = 0; x < D / 32; ++x)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                store4(out, 32 * x + 2 * e + 4 * (lane >> 5), a.d, a.vec_out, dq[i][x][e] * f, dq[i][x][e + 1] * f,
                       dq[i][x][e + 2] * f, dq[i][x][e + 3] * f);
    }
}

// dlam and the learned vectors' gradients from the parts, by one workgroup.
__device__ __forceinline__ void weight_grads(const AttnArgs &a, int lane, int wave) {
    __shared__ float totals[4];
    float total = 0.f;
    for (int h = wave; h < a.H; h += 4) {
        float sum = 0.f;
        for (int64_t i = lane; i < a.dlam_count; i += 64) sum += a.dlam_parts[(int64_t)h * a.dlam_count + i];
        sum = -wave_sum(sum);
        total += sum;
        if (lane == 0) a.dlam[h] = sum;
        if (!a.weight.value && a.weight.per_head) {
            const Weight w = weight_of(a.weight, h, lane);
            const int64_t at = (int64_t)h * a.weight.n;
            for (int64_t i = at + lane; i < at + a.weight.n; i += 64) {
                a.dq1[i] = sum * w.e1 * a.weight.k1[i];
                a.dk1[i] = sum * w.e1 * a.weight.q1[i];
                a.dq2[i] = -sum * w.e2 * a.weight.k2[i];
                a.dk2[i] = -sum * w.e2 * a.weight.q2[i];
            }
        }
    }
    if (a.weight.value || a.weight.per_head) return;
    if (lane == 0) totals[wave] = total;
    __syncthreads();
    total = (totals[0] + totals[1]) + (totals[2] + totals[3]);
    const Weight w = weight_of(a.weight, 0, lane);
    for (int i = threadIdx.x; i < a.weight.n; i += 256) {
        a.dq1[i] = total * w.e1 * a.weight.k1[i];
        a.dk1[i] = total * w.e1 * a.weight.q1[i];
        a.dq2[i] = -total * w.e2 * a.weight.k2[i];
        a.dk2[i] = -total * w.e2 * a.weight.q2[i];
    }
}

// dk and dv: 128 keys a workgroup, 32 a wave, over the rows of all heads that share them.
// Scores as rows x keys, so a lane's rows are of one key and the maps are the operands of dv
// and dk as they lie.  DK, DV_: which of the two a workgroup makes.
template <class T, int D, int DV>
struct KeySteps {
    static constexpr int QT = 64;
    using QTile = Tile<T, D / 8, QT, 4>;
    using GTile = Tile<T, DV / 8, QT, 4>;
    static constexpr int TILES = 2 * QTile::BYTES + GTile::BYTES, STAGE = TILES + 4 * QT * 4;
};
template <class T, int D, int DV, bool DK, bool DV_>
__device__ __forceinline__ void key_grads(const AttnArgs &a, uint32_t lds, int id, int lane, int wave) {
    using S = KeySteps<T, D, DV>;
    using QTile = typename S::QTile;
    using GTile = typename S::GTile;
    constexpr int QT = S::QT, TILES = S::TILES, STAGE = S::STAGE;
    const int tile = id % a.key_tiles;
    id /= a.key_tiles;
    const int hk = id % a.Hk, b = id / a.Hk;
    const Sequence s = sequence(a, b);
    const int64_t begin = (int64_t)tile * kGradKeys;
    if (begin >= s.nk) return;
    const int key0 = (int)begin + wave * 32, key = key0 + (lane & 31);
    const bool valid = key < s.nk;
    const int off = s.nk - s.nq;
    // rows that see any of the workgroup's keys, of the wave's, and each of the wave's
    const int end = s.nk - 1 < (int)begin + kGradKeys - 1 ? s.nk - 1 : (int)begin + kGradKeys - 1;
    auto clip = [&](int64_t t) { return (int)(t < 0 ? 0 : t < s.nq ? t : s.nq - 1); };
    const int64_t low = begin - off - a.right, high = (int64_t)end - off + a.left;
    const int t0 = clip(low) / QT * QT;
    const int tiles = s.nq > 0 && high >= 0 && low < s.nq ? (clip(high) - t0) / QT + 1 : 0;
    const int64_t wave_low = (int64_t)key0 - off - a.right, wave_high = (int64_t)key0 + 31 - off + a.left;
    const int64_t full_low = wave_low + 31, full_high = wave_high - 31;

    auto stage = [&](int n) {
        const int head = hk * a.group + n / tiles;
        const int64_t t = t0 + (int64_t)(n % tiles) * QT;
        const uint32_t to = lds + (n & 1) * STAGE;
        const int left = (int)(s.nq - t);
        const T *qp = head_of<T>(a.q, s.batch, s.q0 + t, 2 * head);
        QTile::load(qp, a.q.token, left, a.d, a.vec, to, wave, lane);
        QTile::load(qp + a.q.head, a.q.token, left, a.d, a.vec, to + QTile::BYTES, wave, lane);
        GTile::load(head_of<T>(a.grad, s.batch, s.q0 + t, head), a.grad.token, left, a.dv, a.vec, to + 2 * QTile::BYTES,
                    wave, lane);
        // a wave each: logarithms of both maps' sums, D1 and D2
        const int64_t map = 2 * (int64_t)head + (wave & 1);
        const float *from = (wave < 2 ? a.stats + map * a.stat_rows * a.rows : a.delta + map * a.rows) + s.row0 + t;
        dma4(buffer_of(from, (int64_t)(left < QT ? left : QT) * 4), lane * 4, to + TILES + wave * QT * 4);
    };
    const int steps = tiles * a.group;
    if (steps > 0) stage(0);

    v8s k[2][D / 16], v[DV / 16];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
            k[i][c] = row_operand(head_of<T>(a.k, s.batch, s.k0 + key, 2 * hk + i), valid, c, a.d, a.vec, lane);
#pragma unroll
    for (int c = 0; c < DV / 16; ++c)
        if (DK) v[c] = row_operand(head_of<T>(a.v, s.batch, s.k0 + key, hk), valid, c, a.dv, a.vec, lane);
    v16f dk[2][D / 32], dv[DV / 32];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int x = 0; x < D / 32; ++x) dk[i][x] = v16f{};
#pragma unroll
    for (int x = 0; x < DV / 32; ++x) dv[x] = v16f{};

    float lam = 0.f;
    for (int n = 0; n < steps; ++n) {
        if (n % tiles == 0) lam = weight_of(a.weight, hk * a.group + n / tiles, lane).lam;
        arrive();
        if (n + 1 < steps) stage(n + 1);
        const uint32_t qt = lds + (n & 1) * STAGE, gt = qt + 2 * QTile::BYTES;
#pragma unroll 1
        for (int qb = 0; qb < QT; qb += 32) {
            const int r0 = t0 + (n % tiles) * QT + qb;
            if (r0 >= s.nq || key0 >= s.nk || r0 > wave_high || r0 + 31 < wave_low) continue;
            v16f z[2], dp = v16f{};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                z[i] = v16f{};
#pragma unroll
                for (int c = 0; c < D / 16; ++c)
                    z[i] = Mfma<T>::mul(QTile::rows(qt + i * QTile::BYTES, qb, c, lane), k[i][c], z[i]);
            }
#pragma unroll
            for (int c = 0; c < DV / 16; ++c)
                if (DK) dp = Mfma<T>::mul(GTile::rows(gt, qb, c, lane), v[c], dp);
            // (rows behind the last are zero in q and do: they add nothing)
            if (r0 < full_low || r0 + 31 > full_high) {
                const int64_t from = (int64_t)key - off - a.right, to = (int64_t)key - off + a.left;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int t = r0 + 8 * (e / 4) + 4 * (lane >> 5) + e % 4;
                    const bool seen = t >= from && t <= to;
                    z[0][e] = seen ? z[0][e] : -__builtin_inff();
                    z[1][e] = seen ? z[1][e] : -__builtin_inff();
                }
            }
            float both[16], ds1[16], ds2[16];
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
                const uint32_t at = qt + TILES + (qb + 8 * e4 + 4 * (lane >> 5)) * 4;
                const v4f l1 = lds_load<v4f>(at), l2 = lds_load<v4f>(at + QT * 4);
                const v4f d1 = lds_load<v4f>(at + 2 * QT * 4), d2 = lds_load<v4f>(at + 3 * QT * 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int e = 4 * e4 + j;
                    const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[0][e], a.scale2, -l1[j]));
                    const float p2 = lam * __builtin_amdgcn_exp2f(__builtin_fmaf(z[1][e], a.scale2, -l2[j]));
                    both[e] = p1 - p2;
                    ds1[e] = p1 * (dp[e] - d1[j]);
                    ds2[e] = p2 * (d2[j] - dp[e]);
                }
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const v8s b0 = pack<T>(both, c), b1 = pack<T>(ds1, c), b2 = pack<T>(ds2, c);
#pragma unroll
                for (int x = 0; x < DV / 32; ++x)
                    if (DV_) dv[x] = Mfma<T>::mul(GTile::turned(gt, qb + 16 * c, x, lane), b0, dv[x]);
#pragma unroll
                for (int x = 0; x < D / 32; ++x) {
                    if (!DK) break;
                    dk[0][x] = Mfma<T>::mul(QTile::turned(qt, qb + 16 * c, x, lane), b1, dk[0][x]);
                    dk[1][x] = Mfma<T>::mul(QTile::turned(qt + QTile::BYTES, qb + 16 * c, x, lane), b2, dk[1][x]);
                }
            }
        }
    }
    if (!valid) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (!DK) break;
        T *out = head_of<T>(a.dk, s.batch, s.k0 + key, 2 * hk + i);
#pragma unroll
        for (int x = 0; x < D / 32; ++x)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                store4(out, 32 * x + 2 * e + 4 * (lane >> 5), a.d, a.vec_out, dk[i][x][e] * a.scale,
                       dk[i][x][e + 1] * a.scale, dk[i][x][e + 2] * a.scale, dk[i][x][e + 3] * a.scale);
    }
    if (!DV_) return;
    T *out = head_of<T>(a.dv_, s.batch, s.k0 + key, hk);
#pragma unroll
    for (int x = 0; x < DV / 32; ++x)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
            store4(out, 32 * x + 2 * e + 4 * (lane >> 5), a.dv, a.vec_out, dv[x][e], dv[x][e + 1], dv[x][e + 2],
                   dv[x][e + 3]);
}

// The widest class's sums of both do not fit the registers: a workgroup for dk and one for dv, each
// with the scores.  The last workgroup of the launch makes the learned weights' gradients.
template <class T, int D, int DV>
__global__ __launch_bounds__(256, 1) void k_diff_grad_k(AttnArgs a) {
    __shared__ __attribute__((aligned(1024))) char shared[2 * KeySteps<T, D, DV>::STAGE];
    const uint32_t lds = lds_start(shared);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (blockIdx.x == gridDim.x - 1) {
        weight_grads(a, lane, wave);
        return;
    }
    const int id = near_block(blockIdx.x, gridDim.x - 1);
    if constexpr (DV <= 128)
        key_grads<T, D, DV, true, true>(a, lds, id, lane, wave);
    else if (id & 1)
        key_grads<T, D, DV, false, true>(a, lds, id >> 1, lane, wave);
    else
        key_grads<T, D, DV, true, false>(a, lds, id >> 1, lane, wave);
}

template <class T>
int grad_q(int cls, const AttnArgs &a, hipStream_t s) {
    const dim3 grid((unsigned)((int64_t)a.batch * a.Hk * a.row_tiles)), block(256);
    if (cls == 0)
        hipLaunchKernelGGL((k_diff_grad_q<T, 32, 64>), grid, block, 0, s, a);
    else if (cls == 1)
        hipLaunchKernelGGL((k_diff_grad_q<T, 64, 128>), grid, block, 0, s, a);
    else
        hipLaunchKernelGGL((k_diff_grad_q<T, 128, 256>), grid, block, 0, s, a);
    return (int)hipGetLastError();
}
template <class T>
int grad_k(int cls, const AttnArgs &a, hipStream_t s) {
    const dim3 grid((unsigned)((int64_t)a.batch * a.Hk * a.key_tiles * (cls == 2 ? 2 : 1) + 1)), block(256);
    if (cls == 0)
        hipLaunchKernelGGL((k_diff_grad_k<T, 32, 64>), grid, block, 0, s, a);
    else if (cls == 1)
        hipLaunchKernelGGL((k_diff_grad_k<T, 64, 128>), grid, block, 0, s, a);
    else
        hipLaunchKernelGGL((k_diff_grad_k<T, 128, 256>), grid, block, 0, s, a);
    return (int)hipGetLastError();
}

}  // namespace

int launch_diff_grad_q(int type, int cls, const AttnArgs &a, void *stream) {
    return type == NM_TYPE_F16 ? grad_q<half_t>(cls, a, (hipStream_t)stream) : grad_q<bf16_t>(cls, a, (hipStream_t)stream);
}
int launch_diff_grad_k(int type, int cls, const AttnArgs &a, void *stream) {
    return type == NM_TYPE_F16 ? grad_k<half_t>(cls, a, (hipStream_t)stream) : grad_k<bf16_t>(cls, a, (hipStream_t)stream);
}

}  // namespace nmspmm
