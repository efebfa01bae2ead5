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
    constexpr int KT = kGradKeyTile;
    using KTile = Tile<T, D / 8, KT, 4>;
    using VTile = Tile<T, DV / 8, KT, 4>;
    using KFeed = Feed<T, D / 8, KT, 4, 2>;
    using VFeed = Feed<T, DV / 8, KT, 4, 1>;
    constexpr int STAGE = 2 * KTile::BYTES + VTile::BYTES;
    __shared__ __attribute__((aligned(1024))) char shared[2 * STAGE];
    const uint32_t lds = lds_start(shared);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const RowTile r = row_tile<kGradRows>(a, near_block(blockIdx.x, gridDim.x), lane, wave);
    const Sequence &s = r.s;
    float *lam_part = a.dlam_parts + (int64_t)r.hk * a.group * a.dlam_count + ((int64_t)r.b * a.row_tiles + r.tile) * 4 + wave;
    if (r.rows <= 0) {
        for (int k = lane; k < a.group; k += 64) lam_part[(int64_t)k * a.dlam_count] = 0.f;
        return;
    }
    const int tile0 = r.low / KT, tiles = r.high >= r.low ? r.high / KT + 1 - tile0 : 0;
    const int64_t key0 = s.k0 + (int64_t)tile0 * KT;
    const int left = s.nk - tile0 * KT;
    KFeed keys(head_of<T>(a.k, s.batch, key0, 2 * r.hk), a.k.token, a.k.head, left, a.d, a.vec, wave, lane);
    VFeed values(head_of<T>(a.v, s.batch, key0, r.hk), a.v.token, 0, left, a.dv, a.vec, wave, lane);
    auto stage = [&](int n) {      // the next tile
        keys.load(lds + (n & 1) * STAGE, wave, lane);
        values.load(lds + (n & 1) * STAGE + 2 * KTile::BYTES, wave, lane);
    };
    if (tiles > 0) stage(0);

    v8s q[2][D / 16], grad[DV / 16];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
            q[i][c] = row_operand(head_of<T>(a.q, s.batch, s.q0 + r.t, 2 * r.head + i), r.valid, c, a.d, a.vec, lane);
    const float lam = row_weight(a, r, lane);
    float d[2], lse[2];
    {
        typedef T v8 __attribute__((ext_vector_type(8)));
        const T *gp = head_of<T>(a.grad, s.batch, s.q0 + r.t, r.head);
        const int16_t *kept = a.kept + ((s.row0 + r.t) * a.H + r.head) * 2 * a.dv;
        float sums[2][(DV + kScaleWidth - 1) / kScaleWidth] = {};
#pragma unroll
        for (int c = 0; c < DV / 16; ++c) {
            grad[c] = row_operand(gp, r.valid, c, a.dv, a.vec, lane);
            const v8 x = __builtin_bit_cast(v8, grad[c]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const v8s y = row_operand(kept + i * a.dv, r.valid, c, a.dv, a.dv % 8 == 0, lane);
#pragma unroll
                for (int e = 0; e < 8; ++e) sums[i][c * 16 / kScaleWidth] += (float)x[e] * (float)y[e];
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t at = (2 * (int64_t)r.head + i) * a.stat_rows * a.rows + s.row0 + r.t;
            lse[i] = a.stats[at];
            d[i] = 0.f;
#pragma unroll
            for (int c = 0; c < (DV + kScaleWidth - 1) / kScaleWidth; ++c)
                if (c * kScaleWidth < a.dv) d[i] += half_sum(sums[i][c]) * a.stats[at + (1 + c) * a.rows];
            if (r.valid && lane < 32) a.delta[(2 * (int64_t)r.head + i) * a.rows + s.row0 + r.t] = d[i];
        }
    }
    v16f dq[2][D / 32];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int x = 0; x < D / 32; ++x) dq[i][x] = v16f{};
    float second = 0.f;   // sum of p2 dp over this lane's keys

    const uint32_t k_at = lds + KTile::rows_lane(lane), k_turned = lds + KTile::turned_lane(lane);
    const uint32_t v_at = lds + 2 * KTile::BYTES + VTile::rows_lane(lane);
    for (int n = 0; n < tiles; ++n) {
        arrive();
        if (n + 1 < tiles) stage(n + 1);
        const uint32_t slot = (n & 1) * STAGE;
#pragma unroll
        for (int kb = 0; kb < KT; kb += 32) {
            const int j0 = (tile0 + n) * KT + kb;
            if (j0 > r.block_high || j0 + 31 < r.block_low) continue;
            v16f z[2] = {v16f{}, v16f{}}, dp = v16f{};
#pragma unroll
            for (int c = 0; c < D / 16; ++c)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    z[i] = Mfma<T>::mul(KTile::rows(k_at + slot + i * KTile::BYTES, kb, c), q[i][c], z[i]);
#pragma unroll
            for (int c = 0; c < DV / 16; ++c) dp = Mfma<T>::mul(VTile::rows(v_at + slot, kb, c), grad[c], dp);
            if (j0 + 31 > r.block_end || j0 < r.block_full) hide(r, j0, lane, z);
            float part = 0.f;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float ds1[8], ds2[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[0][8 * c + e], a.scale2, -lse[0]));
                    const float p2 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[1][8 * c + e], a.scale2, -lse[1]));
                    part = __builtin_fmaf(p2, dp[8 * c + e], part);
                    ds1[e] = p1 * (dp[8 * c + e] - d[0]);
                    ds2[e] = p2 * (dp[8 * c + e] - d[1]);
                }
                const v8s b1 = pack<T>(ds1), b2 = pack<T>(ds2);
#pragma unroll
                for (int x = 0; x < D / 32; ++x) {
                    dq[0][x] = Mfma<T>::mul(KTile::turned(k_turned + slot, kb + 16 * c, x), b1, dq[0][x]);
                    dq[1][x] = Mfma<T>::mul(KTile::turned(k_turned + slot + KTile::BYTES, kb + 16 * c, x), b2, dq[1][x]);
                }
            }
            second += part;
        }
    }
    if (!r.valid) second = 0.f;
    for (int k = 0; k < a.group; ++k) {
        const float w = wave_sum(r.g == k ? second : 0.f);
        if (lane == 0) lam_part[(int64_t)k * a.dlam_count] = w;
    }
    if (!r.valid) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        T *out = head_of<T>(a.dq, s.batch, s.q0 + r.t, 2 * r.head + i);
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
    static constexpr int QT = 32;
    using QTile = Tile<T, D / 8, QT, 4>;
    using GTile = Tile<T, DV / 8, QT, 4>;
    using VTile = Tile<T, DV / 8, kGradKeys, 4>;
    using QFeed = Feed<T, D / 8, QT, 4, 2>;
    using GFeed = Feed<T, DV / 8, QT, 4, 1>;
    using VFeed = Feed<T, DV / 8, kGradKeys, 4, 1>;
    static constexpr int TILES = 2 * QTile::BYTES + GTile::BYTES, STAGE = TILES + 1024;
    static constexpr int BYTES = VTile::BYTES + 2 * STAGE;
};
template <class T, int D, int DV, bool DK, bool DV_>
__device__ __forceinline__ void key_grads(const AttnArgs &a, uint32_t lds, int id, int lane, int wave) {
    using S = KeySteps<T, D, DV>;
    using QTile = typename S::QTile;
    using GTile = typename S::GTile;
    using VTile = typename S::VTile;
    constexpr int QT = S::QT, TILES = S::TILES, STAGE = S::STAGE;
    const int tile = id % a.key_tiles;
    id /= a.key_tiles;
    const int hk = id % a.Hk, b = id / a.Hk;
    const Sequence s = sequence(a, b);
    const int begin = tile * kGradKeys;
    if (begin >= s.nk) return;
    const int key0 = begin + wave * 32, key = key0 + (lane & 31);
    const bool valid = key < s.nk;
    const int off = s.nk - s.nq;
    // rows that see any of the workgroup's keys; any of the wave's, and all of them
    const int end = s.nk - 1 < begin + kGradKeys - 1 ? s.nk - 1 : begin + kGradKeys - 1;
    const int low = begin - off - a.right, high = end - off + a.left;
    auto clip = [&](int t) { return t < 0 ? 0 : t < s.nq ? t : s.nq - 1; };
    const int t0 = clip(low) / QT * QT;
    const int tiles = s.nq > 0 && high >= 0 && low < s.nq ? (clip(high) - t0) / QT + 1 : 0;
    const int from = key - off - a.right;                       // rows that see this lane's key
    const uint32_t span = (uint32_t)a.right + (uint32_t)a.left;
    const int wave_low = key0 - off - a.right, wave_high = key0 < s.nk ? key0 + 31 - off + a.left : -1;
    const int full_low = wave_low + 31, full_high = key0 - off + a.left;

    const uint32_t steps_at = lds + VTile::BYTES;
    auto queries_of = [&](int head) {
        return typename S::QFeed(head_of<T>(a.q, s.batch, s.q0 + t0, 2 * head), a.q.token, a.q.head, s.nq - t0, a.d, a.vec, wave,
                                 lane);
    };
    auto grads_of = [&](int head) {
        return typename S::GFeed(head_of<T>(a.grad, s.batch, s.q0 + t0, head), a.grad.token, 0, s.nq - t0, a.dv, a.vec, wave,
                                 lane);
    };
    auto queries = queries_of(hk * a.group);
    auto grads = grads_of(hk * a.group);
    auto stage = [&](int n, int head, int t) {
        const uint32_t to = steps_at + (n & 1) * STAGE;
        queries.load(to, wave, lane);
        grads.load(to + 2 * QTile::BYTES, wave, lane);
        // a wave each: logarithms of both maps' sums, D1 and D2 (a load is of 64 lanes: zeros behind the 32 rows)
        const int left = s.nq - t;
        const int64_t map = 2 * (int64_t)head + (wave & 1);
        const float *stat = (wave < 2 ? a.stats + map * a.stat_rows * a.rows : a.delta + map * a.rows) + s.row0 + t;
        dma4(buffer_of(stat, (left < QT ? left : QT) * 4), lane * 4, to + TILES + wave * 256);
    };
    const int steps = tiles * a.group;
    if (steps > 0) {
        if (DK)
            typename S::VFeed(head_of<T>(a.v, s.batch, s.k0 + begin, hk), a.v.token, 0, s.nk - begin, a.dv, a.vec, wave, lane)
                .load(lds, wave, lane);
        stage(0, hk * a.group, t0);
    }

    v8s k[2][D / 16];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
            k[i][c] = row_operand(head_of<T>(a.k, s.batch, s.k0 + key, 2 * hk + i), valid, c, a.d, a.vec, lane);
    v16f dk[2][D / 32], dv[DV / 32];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int x = 0; x < D / 32; ++x) dk[i][x] = v16f{};
#pragma unroll
    for (int x = 0; x < DV / 32; ++x) dv[x] = v16f{};

    const uint32_t q_at = steps_at + QTile::rows_lane(lane), q_turned = steps_at + QTile::turned_lane(lane);
    const uint32_t g_at = steps_at + 2 * QTile::BYTES + GTile::rows_lane(lane);
    const uint32_t g_turned = steps_at + 2 * QTile::BYTES + GTile::turned_lane(lane);
    const uint32_t v_at = lds + VTile::rows_lane(lane) + VTile::place_of(wave * 32);
    const uint32_t stat_at = steps_at + TILES + (lane >> 5) * 16;
    float lam = 0.f;
    int head = hk * a.group, at = 0;       // this step's head and tile of rows
    for (int n = 0; n < steps; ++n) {
        if (at == 0) lam = weight_of(a.weight, head, lane).lam;
        arrive();
        const int r0 = t0 + at * QT;
        const bool next = at + 1 == tiles;
        at = next ? 0 : at + 1;
        if (next && ++head < (hk + 1) * a.group) {
            queries = queries_of(head);
            grads = grads_of(head);
        }
        if (n + 1 < steps) stage(n + 1, head, t0 + at * QT);
        if (r0 > wave_high || r0 + 31 < wave_low) continue;
        const uint32_t slot = (n & 1) * STAGE;
        v16f z[2] = {v16f{}, v16f{}}, dp = v16f{};
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                z[i] = Mfma<T>::mul(QTile::rows(q_at + slot + i * QTile::BYTES, 0, c), k[i][c], z[i]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c = 0; c < DV / 16; ++c)
            if (DK) dp = Mfma<T>::mul(GTile::rows(g_at + slot, 0, c), VTile::rows(v_at, 0, c), dp);
        __builtin_amdgcn_sched_barrier(0);
        // (rows behind the last are zero in q and do: they add nothing)
        if (r0 < full_low || r0 + 31 > full_high) {
            const int first = r0 + 4 * (lane >> 5) - from;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const bool seen = (uint32_t)(first + 8 * (e / 4) + e % 4) <= span;
                z[0][e] = seen ? z[0][e] : -__builtin_inff();
                z[1][e] = seen ? z[1][e] : -__builtin_inff();
            }
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float both[8], ds1[8], ds2[8];
#pragma unroll
            for (int e4 = 0; e4 < 2; ++e4) {
                const uint32_t stat = stat_at + slot + 64 * c + 32 * e4;
                const v4f l1 = lds_load<v4f>(stat), l2 = lds_load<v4f>(stat + 256);
                const v4f d1 = lds_load<v4f>(stat + 512), d2 = lds_load<v4f>(stat + 768);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int e = 4 * e4 + j, from = 8 * c + e;
                    const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[0][from], a.scale2, -l1[j]));
                    const float p2 = lam * __builtin_amdgcn_exp2f(__builtin_fmaf(z[1][from], a.scale2, -l2[j]));
                    both[e] = p1 - p2;
                    ds1[e] = p1 * (dp[from] - d1[j]);
                    ds2[e] = p2 * (d2[j] - dp[from]);
                }
            }
            const v8s b0 = pack<T>(both), b1 = pack<T>(ds1), b2 = pack<T>(ds2);
            __builtin_amdgcn_sched_barrier(0);      // (the second half's statistics would not fit the registers)
#pragma unroll
            for (int x = 0; x < DV / 32; ++x)
                if (DV_) dv[x] = Mfma<T>::mul(GTile::turned(g_turned + slot, 16 * c, x), b0, dv[x]);
#pragma unroll
            for (int x = 0; x < D / 32; ++x) {
                if (!DK) break;
                dk[0][x] = Mfma<T>::mul(QTile::turned(q_turned + slot, 16 * c, x), b1, dk[0][x]);
                dk[1][x] = Mfma<T>::mul(QTile::turned(q_turned + slot + QTile::BYTES, 16 * c, x), b2, dk[1][x]);
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
__global__ __launch_bounds__(256, DV <= 128 ? 2 : 1) void k_diff_grad_k(AttnArgs a) {
    __shared__ __attribute__((aligned(1024))) char shared[KeySteps<T, D, DV>::BYTES];
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
