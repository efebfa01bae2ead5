// Differential attention's backward pass, from do (dp = do v^T, D_i = sum over keys of p_i dp):
//   dv   = (p1 - lam p2)^T do
//   ds1  = p1 (dp - D1),  ds2 = -lam p2 (dp - D2)
//   dq_i = scale ds_i k_i,  dk_i = scale ds_i^T q_i,  dlam = -sum over rows of D2
// The maps are made again from the scores and the forward pass's logarithms of their sums.
// D1 and D2 enter ds as do . (p_i v), of the codes that the forward pass kept: 16 bits with a
// scale for each row, 2^-16 of its largest value.  (Products rounded to the type, and the output among
// them, put dq and dk at up to 2.5 times the error of a form in 32 bits.)  dlam takes the sums of p2 dp
// themselves, in 32 bits.
// ds and p1 - lam p2 are rounded to 16 bits once, for the matrix instructions.  In binary16 both are scaled
// by powers of two before that and their sums are scaled back: the maps by |p1 - lam p2| <= 1 + |lam|, ds
// by |dp - D| <= 2 |do| |v|, the largest norm of
// the keys' v in tiles of 128 made by a kernel of its own: for dq a row by itself, for dk all rows that a workgroup's
// keys see.  (Unscaled, do of 1e-4 over 4096 keys lost 14 % of ds, do of 1e3 had infinities, and dv over 9000 keys was up
// to 9 times its bound off.  With a running
// maximum of |dp| in place of the norms the kernel of dq spilled at 128 channels: 2 x 2048 rows of 4 heads, 128 + 256, 297 us
// against 245.)
//
// Two kernels, each with its sums in registers in a fixed order: one over keys for the
// rows of q (which also makes D1, D2 and the parts of dlam), one over rows for the
// keys.  The second makes scores and dp again: 512 of 1792 operations a pair at width
// 64 + 128, against sums of dq in memory by atomics, whose order would change results.
// Where the keys make too few workgroups, the rows are split too, and a third kernel joins their sums.
#include "nmspmm_attn.h"

namespace nmspmm {
namespace {

// The largest |v|^2 of 128 keys (of those that are finite: a row that sees another is not finite whatever its scale), a
// workgroup a tile, 16 lanes a key.  Bound by the latency of its launch, loads and sums: 8 MB, 2 x 2048 keys of 4 heads with
// 256 channels or 32 x 197 of 6 with 128, 5 us.
__global__ __launch_bounds__(256) void k_diff_norms(AttnArgs a) {
    __shared__ float largest[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int tile = blockIdx.x % a.key_tiles, outer = blockIdx.x / a.key_tiles, hk = outer % a.Hk, b = outer / a.Hk;
    const Sequence s = sequence(a, b);
    typedef half_t v8 __attribute__((ext_vector_type(8)));
    constexpr int KEYS = kGradKeys / 16;         // of a thread: its loads are under way together
    const int key0 = tile * kGradKeys + threadIdx.x / 16;
    float sum[KEYS] = {}, most = 0.f;
    for (int c = lane % 16 * 8; c < a.dv; c += 128) {
        const int over = piece_over(c, a.dv);
        v8s y[KEYS];
#pragma unroll
        for (int n = 0; n < KEYS; ++n) {
            y[n] = v8s{};
            if (key0 + 16 * n < s.nk) y[n] = row_piece(head_of<half_t>(a.v, s.batch, s.k0 + key0 + 16 * n, hk), c, a.dv, over);
        }
#pragma unroll
        for (int n = 0; n < KEYS; ++n) {
            const v8 x = __builtin_bit_cast(v8, over > 0 ? moved(y[n], over) : y[n]);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[n] += (float)x[e] * (float)x[e];
        }
    }
#pragma unroll
    for (int n = 0; n < KEYS; ++n) {             // over the 16 lanes of a key
        float x = sum[n];
        x += dpp<0xB1>(0.f, x);
        x += dpp<0x4E>(0.f, x);
        x += dpp<0x141>(0.f, x);
        x += dpp<0x140>(0.f, x);
        most = fmaxf(most, x < __builtin_inff() ? x : 0.f);
    }
    most = wave_largest(most);
    if (lane == 0) largest[wave] = most;
    __syncthreads();
    if (threadIdx.x == 0)
        a.norms[blockIdx.x] = fmaxf(fmaxf(largest[0], largest[1]), fmaxf(largest[2], largest[3]));
}

// dq, D1, D2 and the parts of dlam: rows as in the forward pass, scores transposed, so a
// lane's keys are of one row and ds is the operand of dq as it lies.  128 rows a workgroup share tiles of 64 keys in a ring
// of two.  Bound by matrix instructions (8 d + 2 dv operations a pair) and the exponentials and products beside
// them: 2 x 4096 causal rows of 8 heads, 4 key heads, 64 + 128, 154 us, 670 TFLOP/s (binary16 158).
template <class T, int D, int DV, bool PIECES>
__global__ __launch_bounds__(256, D <= 64 ? 2 : 1) void k_diff_grad_q(AttnArgs a) {
    constexpr int KT = kGradKeyTile;
    using KTile = Tile<T, D / 8, KT, 4>;
    using VTile = Tile<T, DV / 8, KT, 4>;
    using KFeed = Feed<T, D / 8, KT, 4, 2, PIECES>;
    using VFeed = Feed<T, DV / 8, KT, 4, 1, PIECES>;
    constexpr int STAGE = 2 * KTile::BYTES + VTile::BYTES;
    __shared__ __attribute__((aligned(1024))) char shared[2 * STAGE];
    const uint32_t lds = lds_start(shared);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const RowTile r = row_tile<kGradRows>(a, near_block(blockIdx.x, gridDim.x), lane, wave);
    const Sequence &s = r.s;
    float *lam_part = a.dlam_parts + (int64_t)r.hk * a.group * a.dlam_count + ((int64_t)r.b * a.row_tiles + r.tile) * 4 + wave;
    float *top_part = a.tops + (((int64_t)r.b * a.Hk + r.hk) * a.row_tiles + r.tile) * 4 + wave;
    if (r.rows <= 0) {
        for (int k = lane; k < a.group; k += 64) lam_part[(int64_t)k * a.dlam_count] = 0.f;
        if (lane == 0) *top_part = 0.f;
        return;
    }
    const int tile0 = r.low / KT, tiles = r.high >= r.low ? r.high / KT + 1 - tile0 : 0;
    const int64_t key0 = s.k0 + (int64_t)tile0 * KT;
    const int left = s.nk - tile0 * KT;
    KFeed keys(head_of<T>(a.k, s.batch, key0, 2 * r.hk), a.k.token, a.k.head, left, a.d, wave, lane);
    VFeed values(head_of<T>(a.v, s.batch, key0, r.hk), a.v.token, 0, left, a.dv, wave, lane);
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
            q[i][c] = row_operand<PIECES>(head_of<T>(a.q, s.batch, s.q0 + r.t, 2 * r.head + i), r.valid, c, a.d, lane);
    const float lam = row_weight(a, r, lane);
    float d[2], lse[2];
    constexpr bool kScaled = kFewExponents<T>;
    float square = 0.f;   // of this lane's part of do
    {
        typedef T v8 __attribute__((ext_vector_type(8)));
        const T *gp = head_of<T>(a.grad, s.batch, s.q0 + r.t, r.head);
        const int16_t *kept = a.kept + ((s.row0 + r.t) * a.H + r.head) * 2 * a.dv;
        float sums[2][(DV + kScaleWidth - 1) / kScaleWidth] = {};
#pragma unroll
        for (int c = 0; c < DV / 16; ++c) {
            grad[c] = row_operand<PIECES>(gp, r.valid, c, a.dv, lane);
            const v8 x = __builtin_bit_cast(v8, grad[c]);
            if (kScaled)
#pragma unroll
                for (int e = 0; e < 8; ++e) square += (float)x[e] * (float)x[e];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const v8s y = row_operand<PIECES>(kept + i * a.dv, r.valid, c, a.dv, lane);
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
    // binary16: the power of two of this row's ds (and of d from here on).  2^13 <= up |do| |v| < 2^14, so |ds| is
    // at most 2^15.  (|do|^2 |v|^2 is below 2^80; at kMostSquare it is not finite.)
    constexpr int kLeastSquare = -100, kMostSquare = 90;
    float up = 1.f;
    if (kScaled) {
        const float *norms = a.norms + ((int64_t)r.b * a.Hk + r.hk) * a.key_tiles;
        float most = 0.f;
        if (r.high >= r.low)
            for (int i = r.low / kGradKeys + lane; i <= r.high / kGradKeys; i += 64) most = fmaxf(most, norms[i]);
        up = power(14 - half_up(exponent(half_sum(square) * wave_largest(most), kLeastSquare, kMostSquare)));
        d[0] *= up;
        d[1] *= up;
    }
    // A row that sees one key has ds = 0: the codes would leave 2^-16 of dp.  Its D1 and D2 are dp itself, which the
    // kernel of the keys makes by the same instructions.
    const bool one = r.first == r.last, any_one = __any(one);
    float only = 0.f;

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
            // scores of both maps and dp, operands read a few instructions ahead
            constexpr int AHEAD = 3, QK = 2 * (D / 16), ALL = QK + DV / 16, N = D / 32;
            v16f z[2], dp;
            v8s f[ALL + AHEAD];
            auto operand = [&](int m) {
                return m < QK ? KTile::rows(k_at + slot + m % 2 * KTile::BYTES, kb, m / 2) : VTile::rows(v_at + slot, kb, m - QK);
            };
#pragma unroll
            for (int m = 0; m < AHEAD; ++m) f[m] = operand(m);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int m = 0; m < ALL; ++m) {
                if (m + AHEAD < ALL) f[m + AHEAD] = operand(m + AHEAD);
                __builtin_amdgcn_sched_barrier(0);
                if (m < QK)
                    z[m % 2] = Mfma<T>::mul(f[m], q[m % 2][m / 2], m < 2 ? v16f{} : z[m % 2]);
                else
                    dp = Mfma<T>::mul(f[m], grad[m - QK], m == QK ? v16f{} : dp);
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_setprio(0);
            if (j0 + 31 > r.block_end || j0 < r.block_full) {
                hide(r, j0, lane, z);
                if (any_one) {
                    const int at = r.first - j0 - 4 * (lane >> 5);
#pragma unroll
                    for (int e = 0; e < 16; ++e) only = at == 8 * (e / 4) + e % 4 ? dp[e] : only;
                }
            }
            // ds of values 8 c .. 8 c + 7, two of them at a time (part k of 4)
            typedef T v2 __attribute__((ext_vector_type(2)));
            v4i ds[2][2];
            float part = 0.f;
            auto some = [&](int c, int k) {
                float d1[2], d2[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int at = 8 * c + 2 * k + e;
                    const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[0][at], a.scale2, -lse[0]));
                    const float p2 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[1][at], a.scale2, -lse[1]));
                    part = __builtin_fmaf(p2, dp[at], part);
                    d1[e] = p1 * (kScaled ? __builtin_fmaf(dp[at], up, -d[0]) : dp[at] - d[0]);
                    d2[e] = p2 * (kScaled ? __builtin_fmaf(dp[at], up, -d[1]) : dp[at] - d[1]);
                }
                ds[c][0][k] = __builtin_bit_cast(int, v2{(T)d1[0], (T)d1[1]});
                ds[c][1][k] = __builtin_bit_cast(int, v2{(T)d2[0], (T)d2[1]});
            };
            // the first half's products with k beside the second half's values
            v8s w[4 * N + 2];
            auto turned = [&](int m) {
                return KTile::turned(k_turned + slot + m % 2 * KTile::BYTES, kb + m / (2 * N) * 16, m / 2 % N);
            };
            w[0] = turned(0);
#pragma unroll
            for (int k = 0; k < 4; ++k) some(0, k);
            w[1] = turned(1);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int m = 0; m < 4 * N; ++m) {
                if (m + 2 < 4 * N) w[m + 2] = turned(m + 2);
                __builtin_amdgcn_sched_barrier(0);
                v16f &to = dq[m % 2][m / 2 % N];
                to = Mfma<T>::mul(w[m], __builtin_bit_cast(v8s, ds[m / (2 * N)][m % 2]), to);
                if (m < 2 * N)
#pragma unroll
                    for (int k = m * 4 / (2 * N); k < (m + 1) * 4 / (2 * N); ++k) some(1, k);
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_setprio(0);
            second += part;
        }
    }
    if (!r.valid) second = 0.f;
    for (int k = 0; k < a.group; ++k) {
        const float w = wave_sum(r.g == k ? second : 0.f);
        if (lane == 0) lam_part[(int64_t)k * a.dlam_count] = w;
    }
    only = half_sum(only);
    if (kScaled) {        // (rows that are not finite leave no bound: what they add is not finite at any scale)
        const float bound = inverse(up) * 0x1p14f * fmaxf(1.f, __builtin_fabsf(lam));
        const bool counts = r.valid && !one && up > power(14 - half_up(kMostSquare)) && bound < __builtin_inff();
        const float most = wave_largest(counts ? bound : 0.f);
        if (lane == 0) *top_part = most;
    }
    if (!r.valid) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (one && lane < 32) a.delta[(2 * (int64_t)r.head + i) * a.rows + s.row0 + r.t] = only;
        T *out = head_of<T>(a.dq, s.batch, s.q0 + r.t, 2 * r.head + i);
        const float f = one ? 0.f : (i ? -lam * a.scale : a.scale) * (kScaled ? inverse(up) : 1.f);
#pragma unroll
        for (int x = 0; x < D / 32; ++x)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                store4(out, 32 * x + 2 * e + 4 * (lane >> 5), a.d, dq[i][x][e] * f, dq[i][x][e + 1] * f, dq[i][x][e + 2] * f,
                       dq[i][x][e + 3] * f);
    }
}

// dlam and the learned vectors' gradients from the parts, by one workgroup.
__device__ __forceinline__ void weight_grads(const AttnArgs &a, int lane, int wave, int waves) {
    __shared__ float totals[8];
    float total = 0.f;
    for (int h = wave; h < a.H; h += waves) {
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
    total = 0.f;
    for (int n = 0; n < waves; ++n) total += totals[n];
    const Weight w = weight_of(a.weight, 0, lane);
    for (int i = threadIdx.x; i < a.weight.n; i += 64 * waves) {
        a.dq1[i] = total * w.e1 * a.weight.k1[i];
        a.dk1[i] = total * w.e1 * a.weight.q1[i];
        a.dq2[i] = -total * w.e2 * a.weight.k2[i];
        a.dk2[i] = -total * w.e2 * a.weight.q2[i];
    }
}

// dk and dv: 128 keys a workgroup, over the rows of all heads that share them.  Scores as rows x keys, so a
// lane's rows are of one key and the maps are the operands of dv and dk as they lie.
// PAIR 2: two waves for each 32 keys take every other block of 32 rows, and their sums meet at the end;
// k and v are read from LDS as q and do are, which leaves the registers to the sums (256 of them hold both
// maps' operands too, but not without spilling, and a wait for a spilled register waits for the next
// tile's loads as well: 4 x 4096 rows of 8 heads, width 64 + 128, 760 us and 672).
// PAIR 1, for keys of 128 channels, which with v would fill LDS: a wave each, k in registers.
// Bound as the kernel above (8 d + 4 dv operations a pair): 227 us there, 600 TFLOP/s; binary16, with two products more for
// each value, 247.
template <class T, int D, int DV, bool PIECES>
struct KeySteps {
    static constexpr int PAIR = D <= 64 ? 2 : 1, WAVES = 4 * PAIR, QT = 32 * PAIR;
    using QTile = Tile<T, D / 8, QT, WAVES>;
    using GTile = Tile<T, DV / 8, QT, WAVES>;
    using KTile = Tile<T, D / 8, kGradKeys, WAVES>;
    using VTile = Tile<T, DV / 8, kGradKeys, WAVES>;
    using QFeed = Feed<T, D / 8, QT, WAVES, 2, PIECES>;
    using GFeed = Feed<T, DV / 8, QT, WAVES, 1, PIECES>;
    using KFeed = Feed<T, D / 8, kGradKeys, WAVES, 2, PIECES>;
    using VFeed = Feed<T, DV / 8, kGradKeys, WAVES, 1, PIECES>;
    static constexpr int TILES = 2 * QTile::BYTES + GTile::BYTES, STAGE = TILES + 1024;
    static constexpr int KEYS = PAIR == 2 ? 2 * KTile::BYTES : 0, FIXED = KEYS + VTile::BYTES;
    static constexpr int HAND = PAIR == 2 ? 4 * 64 * (2 * D + DV) * 2 : 0;      // the second waves' sums
    static constexpr int BYTES = FIXED + 2 * STAGE > HAND ? FIXED + 2 * STAGE : HAND;
};
// DK, DV_: which of the two a workgroup makes.
template <class T, int D, int DV, bool PIECES, bool DK, bool DV_>
__device__ __forceinline__ void key_grads(const AttnArgs &a, uint32_t lds, int id, int lane, int wave) {
    using S = KeySteps<T, D, DV, PIECES>;
    using QTile = typename S::QTile;
    using GTile = typename S::GTile;
    using KTile = typename S::KTile;
    using VTile = typename S::VTile;
    constexpr int PAIR = S::PAIR, QT = S::QT, TILES = S::TILES, STAGE = S::STAGE;
    const int block = wave / PAIR, sub = wave % PAIR;             // the wave's 32 keys, and which blocks of rows
    const int split = id % a.key_splits;
    id /= a.key_splits;
    const int tile = id % a.key_tiles;
    id /= a.key_tiles;
    const int hk = id % a.Hk, b = id / a.Hk;
    const Sequence s = sequence(a, b);
    const int begin = tile * kGradKeys;
    if (begin >= s.nk) return;
    const int key0 = begin + block * 32, key = key0 + (lane & 31);
    const bool valid = key < s.nk;
    const int off = s.nk - s.nq;
    // rows that see any of the workgroup's keys, and all of the wave's
    const int end = s.nk - 1 < begin + kGradKeys - 1 ? s.nk - 1 : begin + kGradKeys - 1;
    const int low = begin - off - a.right, high = end - off + a.left;
    auto clip = [&](int t) { return t < 0 ? 0 : t < s.nq ? t : s.nq - 1; };
    const int t0 = clip(low) / QT * QT;
    const int tiles = s.nq > 0 && high >= 0 && low < s.nq ? (clip(high) - t0) / QT + 1 : 0;
    const int from = key - off - a.right;                       // rows that see this lane's key
    const uint32_t span = (uint32_t)a.right + (uint32_t)a.left;
    const int full_low = key0 + 31 - off - a.right, full_high = key0 - off + a.left;

    // steps: the tiles of rows of one head after the other; this split's part of them
    const int all = tiles * a.group, step0 = a.key_splits > 1 ? (int)((int64_t)all * split / a.key_splits) : 0;
    const int steps = (a.key_splits > 1 ? (int)((int64_t)all * (split + 1) / a.key_splits) : all) - step0;
    int head = hk * a.group, at = 0;       // this step's head and tile of rows
    if (step0 > 0) {
        head += step0 / tiles;
        at = step0 % tiles;
    }
    const uint32_t steps_at = lds + S::FIXED;
    auto queries_of = [&](int head, int t) {
        return typename S::QFeed(head_of<T>(a.q, s.batch, s.q0 + t, 2 * head), a.q.token, a.q.head, s.nq - t, a.d, wave, lane);
    };
    auto grads_of = [&](int head, int t) {
        return typename S::GFeed(head_of<T>(a.grad, s.batch, s.q0 + t, head), a.grad.token, 0, s.nq - t, a.dv, wave, lane);
    };
    auto queries = queries_of(head, t0 + at * QT);
    auto grads = grads_of(head, t0 + at * QT);
    auto stage = [&](int n, int head, int t) {
        const uint32_t to = steps_at + (n & 1) * STAGE;
        queries.load(to, wave, lane);
        grads.load(to + 2 * QTile::BYTES, wave, lane);
        // a wave each: logarithms of both maps' sums, D1 and D2 (a load is of 64 lanes: zeros behind the last row)
        if (wave < 4) {
            const int left = s.nq - t;
            const int64_t map = 2 * (int64_t)head + (wave & 1);
            const float *stat = (wave < 2 ? a.stats + map * a.stat_rows * a.rows : a.delta + map * a.rows) + s.row0 + t;
            dma4(lane < (left < QT ? left : QT) ? stat + lane : (const float *)zeros, to + TILES + wave * 256);
        }
    };
    if (steps > 0) {
        if (PAIR == 2) {
            typename S::KFeed keys(head_of<T>(a.k, s.batch, s.k0 + begin, 2 * hk), a.k.token, a.k.head, s.nk - begin, a.d,
                                   wave, lane);
            keys.load(lds, wave, lane);
        }
        if (DK) {
            typename S::VFeed values(head_of<T>(a.v, s.batch, s.k0 + begin, hk), a.v.token, 0, s.nk - begin, a.dv, wave, lane);
            values.load(lds + S::KEYS, wave, lane);
        }
        stage(0, head, t0 + at * QT);
    }

    v8s k[2][D / 16];
    if constexpr (PAIR == 1)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int c = 0; c < D / 16; ++c)
                k[i][c] = row_operand<PIECES>(head_of<T>(a.k, s.batch, s.k0 + key, 2 * hk + i), valid, c, a.d, lane);
    v16f dk[2][D / 32], dv[DV / 32];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int x = 0; x < D / 32; ++x) dk[i][x] = v16f{};
#pragma unroll
    for (int x = 0; x < DV / 32; ++x) dv[x] = v16f{};

    const uint32_t rows_at = steps_at + QTile::place_of(sub * 32);
    const uint32_t g_rows_at = steps_at + 2 * QTile::BYTES + GTile::place_of(sub * 32);
    const uint32_t q_at = rows_at + QTile::rows_lane(lane), q_turned = rows_at + QTile::turned_lane(lane);
    const uint32_t g_at = g_rows_at + GTile::rows_lane(lane), g_turned = g_rows_at + GTile::turned_lane(lane);
    const uint32_t k_at = lds + KTile::rows_lane(lane) + KTile::place_of(block * 32);
    const uint32_t v_at = lds + S::KEYS + VTile::rows_lane(lane) + VTile::place_of(block * 32);
    const uint32_t stat_at = steps_at + TILES + sub * 128 + (lane >> 5) * 16;
    // binary16: powers of two of the maps for dv (`maps_up` max(|p1 - lam p2|) <= 2^15 of all heads that share it) and of ds for
    // dk (at most 2^15 by the bounds of the rows from t0 on, which have numbers t * group + g, 32 a bound)
    constexpr bool kScaled = kFewExponents<T>;
    float maps_up = 1.f, up = 1.f;
    if (kScaled && DV_) {
        float most = 0.f;
        for (int g = 0; g < a.group; ++g) {
            const float w = __builtin_fabsf(weight_of(a.weight, hk * a.group + g, lane).lam);
            most = fmaxf(most, w < __builtin_inff() ? w : 0.f);
        }
        maps_up = power(15 - exponent(1.f + most, 1, 30));
    }
    if (kScaled && DK && steps > 0) {
        const float *tops = a.tops + ((int64_t)b * a.Hk + hk) * a.row_tiles * 4;
        const int to = ((clip(high) + 1) * a.group - 1) / 32;
        float most = 0.f;
        for (int i = t0 * a.group / 32 + lane; i <= to; i += 64) most = fmaxf(most, tops[i]);
        up = power(14 - exponent(wave_largest(most), -40, 100));
    }
    const float beside = up * inverse(maps_up);          // of dp - D, beside the maps' own
    float lam = 0.f;
    for (int n = 0; n < steps; ++n) {
        if (n == 0 || at == 0) lam = weight_of(a.weight, head, lane).lam * maps_up;       // (as p2 is used)
        arrive();
        const int r0 = t0 + at * QT + sub * 32;
        const bool next = at + 1 == tiles;
        at = next ? 0 : at + 1;
        if (next && ++head < (hk + 1) * a.group) {
            queries = queries_of(head, t0);
            grads = grads_of(head, t0);
        }
        if (n + 1 < steps) stage(n + 1, head, t0 + at * QT);
        // (Rows behind the last are zero in q and do and add nothing, and neither do rows that see none of the wave's
        // keys.  They are few, and a branch around the step would cost copies of all sums.)
        const uint32_t slot = (n & 1) * STAGE;
        constexpr int AHEAD = 2, QK = 2 * (D / 16), ALL = QK + (DK ? DV / 16 : 0);
        v16f z[2], dp = v16f{};
        v8s f[ALL + AHEAD], g[ALL + AHEAD];        // operands, read a few instructions ahead
        auto operands = [&](int m) {
            if (m < QK) {
                f[m] = QTile::rows(q_at + slot + m % 2 * QTile::BYTES, 0, m / 2);
                if constexpr (PAIR == 2) g[m] = KTile::rows(k_at + m % 2 * KTile::BYTES, 0, m / 2);
            } else {
                f[m] = GTile::rows(g_at + slot, 0, m - QK);
                g[m] = VTile::rows(v_at, 0, m - QK);
            }
        };
#pragma unroll
        for (int m = 0; m < AHEAD; ++m) operands(m);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int m = 0; m < ALL; ++m) {
            if (m + AHEAD < ALL) operands(m + AHEAD);
            __builtin_amdgcn_sched_barrier(0);
            if (m < QK)
                z[m % 2] = Mfma<T>::mul(f[m], PAIR == 2 ? g[m] : k[m % 2][m / 2], m < 2 ? v16f{} : z[m % 2]);
            else
                dp = Mfma<T>::mul(f[m], g[m], dp);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        if (r0 < full_low || r0 + 31 > full_high) {
            const int first = r0 + 4 * (lane >> 5) - from;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const bool seen = (uint32_t)(first + 8 * (e / 4) + e % 4) <= span;
                z[0][e] = seen ? z[0][e] : -__builtin_inff();
                z[1][e] = seen ? z[1][e] : -__builtin_inff();
            }
        }
        // p1 - lam p2 and ds of values 8 c .. 8 c + 7, four of them at a time (part h of 2)
        typedef T v4 __attribute__((ext_vector_type(4)));
        typedef int v2i __attribute__((ext_vector_type(2)));
        v4i made[2][3];
        auto some = [&](int c, int h) {
            const uint32_t stat = stat_at + slot + 64 * c + 32 * h;
            const v4f l1 = lds_load<v4f>(stat), l2 = lds_load<v4f>(stat + 256);
            v4f d1 = {}, d2 = {};
            if (DK) {
                d1 = lds_load<v4f>(stat + 512);
                d2 = lds_load<v4f>(stat + 768);
            }
            v4 r0, r1, r2;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int v = 8 * c + 4 * h + e;
                float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[0][v], a.scale2, -l1[e]));
                if (kScaled && DV_) p1 *= maps_up;
                const float p2 = lam * __builtin_amdgcn_exp2f(__builtin_fmaf(z[1][v], a.scale2, -l2[e]));
                r0[e] = (T)(p1 - p2);
                if (kScaled && DK) {
                    const float x = dp[v] * beside;
                    r1[e] = (T)(p1 * __builtin_fmaf(-d1[e], beside, x));
                    r2[e] = (T)(p2 * __builtin_fmaf(d2[e], beside, -x));
                } else {
                    r1[e] = (T)(p1 * (dp[v] - d1[e]));
                    r2[e] = (T)(p2 * (d2[e] - dp[v]));
                }
            }
            const v2i i0 = __builtin_bit_cast(v2i, r0), i1 = __builtin_bit_cast(v2i, r1), i2 = __builtin_bit_cast(v2i, r2);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                made[c][0][2 * h + e] = i0[e];
                made[c][1][2 * h + e] = i1[e];
                made[c][2][2 * h + e] = i2[e];
            }
        };
        // the first half's products beside the second half's values
        constexpr int NV = DV_ ? DV / 32 : 0, NK = DK ? 2 * (D / 32) : 0, NALL = NV + NK;
        v8s w[2 * NALL + 2];
        auto turned = [&](int m) {
            const int c = m / NALL, x = m % NALL;
            return x < NV ? GTile::turned(g_turned + slot, 16 * c, x)
                          : QTile::turned(q_turned + slot + (x - NV) % 2 * QTile::BYTES, 16 * c, (x - NV) / 2);
        };
        some(0, 0);
        some(0, 1);
        w[0] = turned(0);
        w[1] = turned(1);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int m = 0; m < 2 * NALL; ++m) {
            if (m + 2 < 2 * NALL) w[m + 2] = turned(m + 2);
            __builtin_amdgcn_sched_barrier(0);
            const int c = m / NALL, x = m % NALL;
            v16f &to = x < NV ? dv[x] : dk[(x - NV) % 2][(x - NV) / 2];
            to = Mfma<T>::mul(w[m], __builtin_bit_cast(v8s, made[c][x < NV ? 0 : 1 + (x - NV) % 2]), to);
            if (m < NALL && m % (NALL / 2) == 0) some(1, m / (NALL / 2));
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
    }
    if constexpr (PAIR == 2) {             // the second waves hand their sums to the first
        constexpr int N = 2 * (D / 32) + DV / 32;
        const uint32_t hand = lds + block * 64 * (2 * D + DV) * 2 + lane * 16;
        auto sums = [&](int n) -> v16f & { return n < DV / 32 ? dv[n] : dk[(n - DV / 32) % 2][(n - DV / 32) / 2]; };
        arrive();
        if (sub) {
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                    *(__attribute__((address_space(3))) v4f *)(uintptr_t)(hand + (4 * n + e / 4) * 1024) =
                        v4f{sums(n)[e], sums(n)[e + 1], sums(n)[e + 2], sums(n)[e + 3]};
        }
        arrive();
        if (sub) return;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const v4f y = lds_load<v4f>(hand + (4 * n + e / 4) * 1024);
#pragma unroll
                for (int j = 0; j < 4; ++j) sums(n)[e + j] += y[j];
            }
    }
    if (!valid) return;
    const float down = inverse(up), maps_down = inverse(maps_up);
    if (a.key_splits > 1) {                // sums in 32 bits, dk's before its scale: 2 d and dv of a key
        float *part = a.key_parts + ((((int64_t)b * a.Hk + hk) * a.key_splits + split) * a.tk + key) * (2 * a.d + a.dv);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int x = 0; x < D / 32; ++x)
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                    if (DK)
                        store4(part + i * a.d, 32 * x + 2 * e + 4 * (lane >> 5), a.d, dk[i][x][e] * down, dk[i][x][e + 1] * down,
                               dk[i][x][e + 2] * down, dk[i][x][e + 3] * down);
#pragma unroll
        for (int x = 0; x < DV / 32; ++x)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                if (DV_)
                    store4(part + 2 * a.d, 32 * x + 2 * e + 4 * (lane >> 5), a.dv, dv[x][e] * maps_down,
                           dv[x][e + 1] * maps_down, dv[x][e + 2] * maps_down, dv[x][e + 3] * maps_down);
        return;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (!DK) break;
        const float f = a.scale * down;
        T *out = head_of<T>(a.dk, s.batch, s.k0 + key, 2 * hk + i);
#pragma unroll
        for (int x = 0; x < D / 32; ++x)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                store4(out, 32 * x + 2 * e + 4 * (lane >> 5), a.d, dk[i][x][e] * f, dk[i][x][e + 1] * f, dk[i][x][e + 2] * f,
                       dk[i][x][e + 3] * f);
    }
    if (!DV_) return;
    T *out = head_of<T>(a.dv_, s.batch, s.k0 + key, hk);
#pragma unroll
    for (int x = 0; x < DV / 32; ++x)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
            store4(out, 32 * x + 2 * e + 4 * (lane >> 5), a.dv, dv[x][e] * maps_down, dv[x][e + 1] * maps_down,
                   dv[x][e + 2] * maps_down, dv[x][e + 3] * maps_down);
}

// The widest class's sums of both do not fit the registers: a workgroup for dk and one for dv, each
// with the scores.  The last workgroup of the launch makes the learned weights' gradients.
template <class T, int D, int DV, bool PIECES>
__global__ __launch_bounds__((KeySteps<T, D, DV, PIECES>::WAVES * 64), (D <= 64 ? 2 : 1)) void k_diff_grad_k(AttnArgs a) {
    __shared__ __attribute__((aligned(1024))) char shared[KeySteps<T, D, DV, PIECES>::BYTES];
    const uint32_t lds = lds_start(shared);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (blockIdx.x == gridDim.x - 1) {
        weight_grads(a, lane, wave, KeySteps<T, D, DV, PIECES>::WAVES);
        return;
    }
    const int id = near_block(blockIdx.x, gridDim.x - 1);
    if constexpr (DV <= 128)
        key_grads<T, D, DV, PIECES, true, true>(a, lds, id, lane, wave);
    else if (id & 1)
        key_grads<T, D, DV, PIECES, false, true>(a, lds, id >> 1, lane, wave);
    else
        key_grads<T, D, DV, PIECES, true, false>(a, lds, id >> 1, lane, wave);
}

// The splits' sums of a key: a wave each, in the splits' order.  Bound by memory: two splits there, 84 MB in 20 us.
template <class T>
__global__ __launch_bounds__(256) void k_diff_join_keys(AttnArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= (int64_t)a.batch * a.Hk * a.tk) return;
    const int key = (int)(row % a.tk);
    const int64_t outer = row / a.tk;
    const int hk = (int)(outer % a.Hk), b = (int)(outer / a.Hk), width = 2 * a.d + a.dv;
    const Sequence s = sequence(a, b);
    if (key >= s.nk) return;
    const float *p = a.key_parts + (outer * a.key_splits * a.tk + key) * width;
    const int64_t next = (int64_t)a.tk * width;
    T *dk = head_of<T>(a.dk, s.batch, s.k0 + key, 2 * hk), *dv = head_of<T>(a.dv_, s.batch, s.k0 + key, hk);
    for (int c = lane; c < width; c += 64) {
        float sum = 0.f;
        for (int n = 0; n < a.key_splits; ++n) sum += p[n * next + c];
        if (c < a.d)
            dk[c] = (T)(sum * a.scale);
        else if (c < 2 * a.d)
            dk[a.dk.head + c - a.d] = (T)(sum * a.scale);
        else
            dv[c - 2 * a.d] = (T)sum;
    }
}

template <class T, bool PIECES>
int grad_q(int cls, const AttnArgs &a, hipStream_t s) {
    const dim3 grid((unsigned)((int64_t)a.batch * a.Hk * a.row_tiles)), block(256);
    if (cls == 0)
        hipLaunchKernelGGL((k_diff_grad_q<T, 32, 64, PIECES>), grid, block, 0, s, a);
    else if (cls == 1)
        hipLaunchKernelGGL((k_diff_grad_q<T, 64, 128, PIECES>), grid, block, 0, s, a);
    else if (cls == 2)
        hipLaunchKernelGGL((k_diff_grad_q<T, 128, 128, PIECES>), grid, block, 0, s, a);
    else
        hipLaunchKernelGGL((k_diff_grad_q<T, 128, 256, PIECES>), grid, block, 0, s, a);
    return (int)hipGetLastError();
}
template <class T, int D, int DV, bool PIECES>
int grad_k(const AttnArgs &a, hipStream_t s) {
    const int64_t groups = (int64_t)a.batch * a.Hk * a.key_tiles * a.key_splits * (DV <= 128 ? 1 : 2) + 1;
    hipLaunchKernelGGL((k_diff_grad_k<T, D, DV, PIECES>), dim3((unsigned)groups), dim3(KeySteps<T, D, DV, PIECES>::WAVES * 64), 0,
                       s, a);
    return (int)hipGetLastError();
}
template <class T, bool PIECES>
int grad_k(int cls, const AttnArgs &a, hipStream_t s) {
    return cls == 0   ? grad_k<T, 32, 64, PIECES>(a, s)
           : cls == 1 ? grad_k<T, 64, 128, PIECES>(a, s)
           : cls == 2 ? grad_k<T, 128, 128, PIECES>(a, s)
                      : grad_k<T, 128, 256, PIECES>(a, s);
}
template <class T>
int join_keys(const AttnArgs &a, hipStream_t s) {
    const int64_t rows = (int64_t)a.batch * a.Hk * a.tk;
    hipLaunchKernelGGL(k_diff_join_keys<T>, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, a);
    return (int)hipGetLastError();
}

}  // namespace

int launch_diff_norms(const AttnArgs &a, void *stream) {
    const dim3 grid((unsigned)((int64_t)a.batch * a.Hk * a.key_tiles));
    hipLaunchKernelGGL(k_diff_norms, grid, dim3(256), 0, (hipStream_t)stream, a);
    return (int)hipGetLastError();
}
int launch_diff_grad_q(int type, int cls, const AttnArgs &a, void *stream) {
    const hipStream_t s = (hipStream_t)stream;
    if (type == NM_TYPE_F16) return a.pieces ? grad_q<half_t, true>(cls, a, s) : grad_q<half_t, false>(cls, a, s);
    return a.pieces ? grad_q<bf16_t, true>(cls, a, s) : grad_q<bf16_t, false>(cls, a, s);
}
int launch_diff_grad_k(int type, int cls, const AttnArgs &a, void *stream) {
    const hipStream_t s = (hipStream_t)stream;
    if (type == NM_TYPE_F16) return a.pieces ? grad_k<half_t, true>(cls, a, s) : grad_k<half_t, false>(cls, a, s);
    return a.pieces ? grad_k<bf16_t, true>(cls, a, s) : grad_k<bf16_t, false>(cls, a, s);
}
int launch_diff_join_keys(int type, const AttnArgs &a, void *stream) {
    return type == NM_TYPE_F16 ? join_keys<half_t>(a, (hipStream_t)stream) : join_keys<bf16_t>(a, (hipStream_t)stream);
}

}  // namespace nmspmm
