// Differential attention, forward: per head two softmax maps over the keys that a
// row sees, o = (p1 - lam p2) v.
//
// One pass over the keys.  The ratio of the maps' sums is not known before the last
// key, so each map has its own running maximum, sum and product with v.  Scores are made
// transposed (keys x rows): a lane holds keys of one row of q, so maximum and sum are a
// lane's own but for one exchange of halves, and the maps go into the product with v as
// they lie (nmspmm_attn.h).
// The maps' values are rounded to 16 bits before that product (the matrix instructions
// take no more): half an ulp of each value, the same size as the output's own rounding.  Binary16 holds them times
// 2^7: its ulps end at 2^-24, which keys of little weight reach (as they are, a row lost keys of 2^-25 of the
// largest altogether); now at 2^-31 of the largest, the maximum's lag (below) included.
// Sums, maxima and products are in 32 bits.
//
// The rows of a workgroup are those of all heads that share a key head: row (token
// t, head g of the group) is number t * group + g, so shared keys are read once.
#include "nmspmm_attn.h"

namespace nmspmm {
namespace {

// What the runs of keys of one block of rows have made, joined:  M = max of m_s,
// o_i = sum of 2^(m_s - M) O_s / sum of 2^(m_s - M) l_s, each wave for some of the channels.
template <class T, int DV, int RUNS, int REGION>
__device__ __forceinline__ void join_runs(const AttnArgs &a, const RowTile &r, uint32_t lds, int split, float lam,
                                          float (&top)[2], float (&sum)[2], v16f (&o)[2][DV / 32], int lane, int run) {
    constexpr int N = DV / 32;
    static_assert(N <= RUNS, "a wave for each 32 channels");
    __shared__ v4f ends[RUNS][32];
    __shared__ float largest[N][2][32];
    const int row = lane & 31;
    const bool joins = run < N;                     // this wave makes the channels from 32 run
    const uint32_t mine = lds + run * REGION + lane * 16;
    if (lane < 32) ends[run][row] = v4f{top[0], sum[0], top[1], sum[1]};
    v16f y[2] = {v16f{}, v16f{}};
    float most[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        arrive();                                   // the tiles, or the other map's products, have been read
#pragma unroll
        for (int x = 0; x < N; ++x)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *(__attribute__((address_space(3))) v4f *)(uintptr_t)(mine + (x * 4 + e / 4) * 1024) =
                    v4f{o[i][x][e], o[i][x][e + 1], o[i][x][e + 2], o[i][x][e + 3]};
        arrive();
        float m = -__builtin_inff(), l = 0.f, f[RUNS];
#pragma unroll
        for (int n = 0; n < RUNS; ++n) m = fmaxf(m, ends[n][row][2 * i]);
#pragma unroll
        for (int n = 0; n < RUNS; ++n) {            // (a run that saw no key has no products)
            f[n] = ends[n][row][2 * i + 1] == 0.f ? 0.f : __builtin_amdgcn_exp2f(ends[n][row][2 * i] - m);
            l += f[n] * ends[n][row][2 * i + 1];
        }
        top[i] = m;
        sum[i] = l;
        if (!joins) continue;
        const float over = a.splits > 1 ? 1.f : l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int n = 0; n < RUNS; ++n)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const v4f p = lds_load<v4f>(lds + n * REGION + lane * 16 + (run * 4 + e / 4) * 1024);
#pragma unroll
                for (int j = 0; j < 4; ++j) y[i][e + j] += f[n] * over * p[j];
            }
#pragma unroll
        for (int e = 0; e < 16; ++e) most[i] = larger(most[i], magnitude(y[i][e]));
    }
    if (a.splits > 1) {
        if (!r.valid) return;
        const int64_t part =
            (((int64_t)r.b * a.Hk + r.hk) * a.splits + split) * ((int64_t)a.tq * a.group) + r.t * a.group + r.g;
        float *ml = a.parts + part * 4, *sums = a.parts + (int64_t)a.batch * a.Hk * a.splits * a.tq * a.group * 4;
        if (run == 0 && lane < 32) *(v4f *)ml = v4f{top[0], sum[0], top[1], sum[1]};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                if (joins)
                    store4(sums + (part * 2 + i) * a.dv, 32 * run + 2 * e + 4 * (lane >> 5), a.dv, y[i][e], y[i][e + 1],
                           y[i][e + 2], y[i][e + 3]);
        return;
    }
    if (r.valid && joins) {
        T *op = head_of<T>(a.o, r.s.batch, r.s.q0 + r.t, r.head);
#pragma unroll
        for (int e = 0; e < 16; e += 4)
            store4(op, 32 * run + 2 * e + 4 * (lane >> 5), a.dv, y[0][e] - lam * y[1][e], y[0][e + 1] - lam * y[1][e + 1],
                   y[0][e + 2] - lam * y[1][e + 2], y[0][e + 3] - lam * y[1][e + 3]);
    }
    if (!a.kept) return;
    static_assert(DV <= kScaleWidth, "one scale a row and map");
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        most[i] = larger(most[i], __shfl_xor(most[i], 32));
        if (joins && lane < 32) largest[run][i][row] = most[i];
    }
    arrive();
    if (!r.valid || !joins) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float m = largest[0][i][row];
#pragma unroll
        for (int n = 1; n < N; ++n) m = larger(m, largest[n][i][row]);
        const KeptScale k = kept_scale(m);
        if (run == 0 && lane < 32) {
            float *at = a.stats + (2 * (int64_t)r.head + i) * a.stat_rows * a.rows + r.s.row0 + r.t;
            at[0] = sum[i] == 0.f ? __builtin_inff() : top[i] - kMapsUp<T> + __builtin_amdgcn_logf(sum[i]);
            at[a.rows] = k.scale;
        }
        int16_t *kept = a.kept + (((r.s.row0 + r.t) * a.H + r.head) * 2 + i) * a.dv;
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            store4(kept, 32 * run + 2 * e + 4 * (lane >> 5), a.dv, kept_code(y[i][e], k.inv), kept_code(y[i][e + 1], k.inv),
                   kept_code(y[i][e + 2], k.inv), kept_code(y[i][e + 3], k.inv));
        }
    }
}

// BLOCKS blocks of 32 rows share tiles of KT keys in a ring of two.  MAPS 2: a wave makes both
// maps of its block, whose products share v's operands; MAPS 1: two waves a block make one each and
// meet at the end.  Both maps' sums of 256 channels do not fit a wave's registers, and of 128 they do: (64, 128)
// runs 4 x 4096 rows of 8 heads in 0.47 ms with MAPS 2 and 0.61 with MAPS 1 (more reads of LDS and scalar instructions),
// (128, 256) 2 x 4096 rows in 0.44 ms with MAPS 1 and 0.75 with the scores made for 128 channels at a time.
// RUNS: runs of keys of one block of rows, a wave and a ring each, that meet at the end (few rows): the smallest calls
// need no second kernel.  Bound by memory where the cache is long: 16 x 1 rows over 16384 keys (4 key heads of
// 64 + 128, 537 MB) 110 us; where it is short, by a fixed 6 us (the launch, q, the weight, joining the runs: 1 row of 8 heads
// over 32 to 128 keys 7.7 us) and 1.5 us for each tile that a wave has after its first: over 577 keys, five tiles, 14 us.
// (Eight waves with a tile each, one at its loads beside another that computes: 117 and 14.0 us.)
template <class T, int D, int DV, int BLOCKS, int MAPS, int KT, int RUNS, bool PIECES>
__global__ __launch_bounds__(64 * BLOCKS * (3 - MAPS) * RUNS, BLOCKS > 1 ? 2 : 1) void k_diff_forward(AttnArgs a) {
    static_assert(RUNS == 1 || (BLOCKS == 1 && MAPS == 2), "runs of one block");
    constexpr int WAVES = BLOCKS * (3 - MAPS);     // that share a ring
    using KTile = Tile<T, D / 8, KT, WAVES>;
    using VTile = Tile<T, DV / 8, KT, WAVES>;
    using KFeed = Feed<T, D / 8, KT, WAVES, 2, PIECES>;
    using VFeed = Feed<T, DV / 8, KT, WAVES, 1, PIECES>;
    constexpr int STAGE = 2 * KTile::BYTES + VTile::BYTES;
    constexpr int SLOTS = 2;
    static_assert(MAPS == 2 || BLOCKS * 64 * DV * 2 <= SLOTS * STAGE, "room for the second maps' products");
    static_assert(RUNS == 1 || 64 * DV * 2 <= SLOTS * STAGE, "room for one map's products of a run");
    __shared__ __attribute__((aligned(1024))) char shared[RUNS * SLOTS * STAGE];
    const int lane = threadIdx.x & 63, all = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int run = RUNS > 1 ? all : 0, wave = RUNS > 1 ? 0 : all;
    const uint32_t lds = lds_start(shared) + run * SLOTS * STAGE;
    const int block = MAPS == 2 ? wave : wave >> 1, map = MAPS == 2 ? 0 : wave & 1;   // the wave's first map

    // (the parts of a cache share nothing: those of a long one go to all XCDs)
    int id = RUNS > 1 ? (int)blockIdx.x : near_block(blockIdx.x, gridDim.x);
    const int split = id % a.splits;
    id /= a.splits;
    const RowTile r = row_tile<32 * BLOCKS>(a, id, lane, block);
    if (r.rows <= 0) return;
    const Sequence &s = r.s;
    int tile0 = r.low / KT, tiles = r.high >= r.low ? r.high / KT + 1 - tile0 : 0;
    if (a.splits > 1) {   // this split's part of them
        const int from = (int)((int64_t)tiles * split / a.splits), to = (int)((int64_t)tiles * (split + 1) / a.splits);
        tile0 += from;
        tiles = to - from;
    }
    if (RUNS > 1) {
        const int from = tiles * run / RUNS, to = tiles * (run + 1) / RUNS;
        tile0 += from;
        tiles = to - from;
    }

    const int64_t key0 = s.k0 + (int64_t)tile0 * KT;
    const int left = s.nk - tile0 * KT;
    KFeed keys(head_of<T>(a.k, s.batch, key0, 2 * r.hk), a.k.token, a.k.head, left, a.d, wave, lane);
    VFeed values(head_of<T>(a.v, s.batch, key0, r.hk), a.v.token, 0, left, a.dv, wave, lane);
    auto stage = [&](int n) {      // the next tile
        keys.load(lds + n % SLOTS * STAGE, wave, lane);
        values.load(lds + n % SLOTS * STAGE + 2 * KTile::BYTES, wave, lane);
    };
    if (tiles > 0) stage(0);

    v8s q[MAPS][D / 16];
#pragma unroll
    for (int i = 0; i < MAPS; ++i)
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
            q[i][c] = row_operand<PIECES>(head_of<T>(a.q, s.batch, s.q0 + r.t, 2 * r.head + map + i), r.valid, c, a.d, lane);
    const float lam = a.splits > 1 ? 0.f : row_weight(a, r, lane);

    v16f o[MAPS][DV / 32];
    float top[MAPS], sum[MAPS];
#pragma unroll
    for (int i = 0; i < MAPS; ++i) {
        top[i] = -__builtin_inff();
        sum[i] = 0.f;
#pragma unroll
        for (int x = 0; x < DV / 32; ++x) o[i][x] = v16f{};
    }

    const uint32_t k_at = lds + map * KTile::BYTES + KTile::rows_lane(lane);
    const uint32_t v_at = lds + 2 * KTile::BYTES + VTile::turned_lane(lane);
    for (int n = 0; n < tiles; ++n) {
        if (RUNS > 1)
            arrive_alone();
        else
            arrive();
        if (n + 1 < tiles) stage(n + 1);
        const uint32_t kt = k_at + n % SLOTS * STAGE, vt = v_at + n % SLOTS * STAGE;
#pragma unroll
        for (int kb = 0; kb < KT; kb += 32) {
            const int j0 = (tile0 + n) * KT + kb;
            if (j0 > r.block_high || j0 + 31 < r.block_low) continue;
            // Operands are read from LDS a few matrix instructions before their own; the compiler would
            // put each read right before its use.
            constexpr int AHEAD = 3, QK = MAPS * (D / 16), N = DV / 32;
            v16f z[MAPS];
            v8s f[QK + AHEAD];
            auto key_operand = [&](int m) { return KTile::rows(kt + m % MAPS * KTile::BYTES, kb, m / MAPS); };
#pragma unroll
            for (int m = 0; m < AHEAD && m < QK; ++m) f[m] = key_operand(m);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int m = 0; m < QK; ++m) {
                if (m + AHEAD < QK) f[m + AHEAD] = key_operand(m + AHEAD);
                __builtin_amdgcn_sched_barrier(0);
                z[m % MAPS] = Mfma<T>::mul(f[m], q[m % MAPS][m / MAPS], m < MAPS ? v16f{} : z[m % MAPS]);
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_setprio(0);
            if (j0 + 31 > r.block_end || j0 < r.block_full) hide(r, j0, lane, z);
            // The maximum that the exponents are taken from follows the true one only when that has
            // grown by more than 2^8: a value is then at most 2^8 (2^15 in binary16), which 16 bits and the sums hold.  Each
            // row by itself: its bits do not depend on the rows beside it.
            float now[MAPS], from[MAPS];
            bool grown[MAPS], any = false;
#pragma unroll
            for (int i = 0; i < MAPS; ++i) {
                float m = z[i][0];
#pragma unroll
                for (int e = 1; e < 16; ++e) m = fmaxf(m, z[i][e]);
                now[i] = half_max(m) * a.scale2;
                grown[i] = now[i] > top[i] + 8.f;
                any = any || grown[i];
            }
            if (__any(any)) {
#pragma unroll
                for (int i = 0; i < MAPS; ++i) {
                    const float by = grown[i] ? __builtin_amdgcn_exp2f(top[i] - now[i]) : 1.f;
                    top[i] = grown[i] ? now[i] : top[i];
                    sum[i] *= by;
#pragma unroll
                    for (int x = 0; x < N; ++x) o[i][x] *= by;
                }
            }
#pragma unroll
            for (int i = 0; i < MAPS; ++i) from[i] = top[i] == -__builtin_inff() ? 0.f : top[i] - kMapsUp<T>;
            // values 8 c .. 8 c + 7 of the maps, two of them at a time (part k of PARTS)
            constexpr int PARTS = MAPS * 4;
            typedef T v2 __attribute__((ext_vector_type(2)));
            v4i p[2][MAPS];
            auto some = [&](int c, int k) {
                const int i = k / 4, e = 8 * c + k % 4 * 2;
                const float f0 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[i][e], a.scale2, -from[i]));
                const float f1 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[i][e + 1], a.scale2, -from[i]));
                sum[i] += f0 + f1;
                p[c][i][k % 4] = __builtin_bit_cast(int, v2{(T)f0, (T)f1});
            };
            // the product of the first half with v beside the second half's exponentials
            v8s w[2 * N + 2];
            w[0] = VTile::turned(vt, kb, 0);
#pragma unroll
            for (int k = 0; k < PARTS; ++k) some(0, k);
            w[1] = VTile::turned(vt, kb, 1 % N);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int m = 0; m < 2 * N; ++m) {
                if (m + 2 < 2 * N) w[m + 2] = VTile::turned(vt, kb + (m + 2) / N * 16, (m + 2) % N);
#pragma unroll
                for (int i = 0; i < MAPS; ++i) {
                    __builtin_amdgcn_sched_barrier(0);
                    o[i][m % N] = Mfma<T>::mul(w[m], __builtin_bit_cast(v8s, p[m / N][i]), o[i][m % N]);
                    if (m < N)
#pragma unroll
                        for (int k = (MAPS * m + i) * PARTS / (MAPS * N); k < (MAPS * m + i + 1) * PARTS / (MAPS * N); ++k)
                            some(1, k);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            __builtin_amdgcn_s_setprio(0);
        }
    }
#pragma unroll
    for (int i = 0; i < MAPS; ++i) sum[i] = half_sum(sum[i]);

    if constexpr (RUNS > 1) {
        join_runs<T, DV, RUNS, SLOTS * STAGE>(a, r, lds_start(shared), split, lam, top, sum, o, lane, run);
        return;
    }
    if (a.splits > 1) {
        if (!r.valid) return;
        // rows of a part: [sequence][key head][split][number]
        const int64_t part =
            (((int64_t)r.b * a.Hk + r.hk) * a.splits + split) * ((int64_t)a.tq * a.group) + r.t * a.group + r.g;
        float *ml = a.parts + part * 4 + 2 * map, *sums = a.parts + (int64_t)a.batch * a.Hk * a.splits * a.tq * a.group * 4;
#pragma unroll
        for (int i = 0; i < MAPS; ++i) {
            if (lane < 32) {
                ml[2 * i] = top[i];
                ml[2 * i + 1] = sum[i];
            }
#pragma unroll
            for (int x = 0; x < DV / 32; ++x)
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                    store4(sums + (part * 2 + map + i) * a.dv, 32 * x + 2 * e + 4 * (lane >> 5), a.dv, o[i][x][e],
                           o[i][x][e + 1], o[i][x][e + 2], o[i][x][e + 3]);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < MAPS; ++i) {
        const float over = sum[i] == 0.f ? 0.f : 1.f / sum[i];
#pragma unroll
        for (int x = 0; x < DV / 32; ++x) o[i][x] *= over;
    }
    const uint32_t hand = lds + block * 64 * DV * 2 + lane * 16;
    if constexpr (MAPS == 1) {   // the second map's wave hands its product to the first one's
        arrive();
        if (map) {
#pragma unroll
            for (int x = 0; x < DV / 32; ++x)
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                    *(__attribute__((address_space(3))) v4f *)(uintptr_t)(hand + (x * 4 + e / 4) * 1024) =
                        v4f{o[0][x][e], o[0][x][e + 1], o[0][x][e + 2], o[0][x][e + 3]};
        }
        arrive();
    }
    if (!r.valid) return;
    if (map == 0) {
        T *op = head_of<T>(a.o, s.batch, s.q0 + r.t, r.head);
#pragma unroll
        for (int x = 0; x < DV / 32; ++x)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                v4f y;
                if constexpr (MAPS == 1)
                    y = lds_load<v4f>(hand + (x * 4 + e / 4) * 1024);
                else
                    y = v4f{o[MAPS - 1][x][e], o[MAPS - 1][x][e + 1], o[MAPS - 1][x][e + 2], o[MAPS - 1][x][e + 3]};
                store4(op, 32 * x + 2 * e + 4 * (lane >> 5), a.dv, o[0][x][e] - lam * y[0], o[0][x][e + 1] - lam * y[1],
                       o[0][x][e + 2] - lam * y[2], o[0][x][e + 3] - lam * y[3]);
            }
    }
    if (!a.kept) return;
#pragma unroll
    for (int i = 0; i < MAPS; ++i) {
        float *at = a.stats + (2 * (int64_t)r.head + map + i) * a.stat_rows * a.rows + s.row0 + r.t;
        if (lane < 32) at[0] = sum[i] == 0.f ? __builtin_inff() : top[i] - kMapsUp<T> + __builtin_amdgcn_logf(sum[i]);
        int16_t *kept = a.kept + (((s.row0 + r.t) * a.H + r.head) * 2 + map + i) * a.dv;
#pragma unroll
        for (int w = 0; w < (DV + kScaleWidth - 1) / kScaleWidth; ++w) {
            if (w * kScaleWidth >= a.dv) break;
            float most = 0.f;
#pragma unroll
            for (int x = w * 4; x < w * 4 + 4 && x < DV / 32; ++x)
#pragma unroll
                for (int e = 0; e < 16; ++e) most = larger(most, magnitude(o[i][x][e]));
            most = larger(most, __shfl_xor(most, 32));
            const KeptScale k = kept_scale(most);
            if (lane < 32) at[(1 + w) * a.rows] = k.scale;
#pragma unroll
            for (int x = w * 4; x < w * 4 + 4 && x < DV / 32; ++x)
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const int c = 32 * x + 2 * e + 4 * (lane >> 5);
                    store4(kept, c, a.dv, kept_code(o[i][x][e], k.inv), kept_code(o[i][x][e + 1], k.inv),
                           kept_code(o[i][x][e + 2], k.inv), kept_code(o[i][x][e + 3], k.inv));
                }
        }
    }
}

// The splits' sums of one row and head, a workgroup each:  M = max of m_s,
// o_i = sum of 2^(m_s - M) O_s / sum of 2^(m_s - M) l_s.
// A thread makes the factors of one split (of up to 256), then 4 channels of both maps over every
// `turns`-th split; the turns meet in LDS.  The order of the sums is fixed.  Bound by the latency of its three dependent
// steps: 16 x 1 rows of 16 heads with 8 splits 5.3 us (a wave for a row and head, one split after another: 26 us).
template <class T>
__global__ __launch_bounds__(256) void k_diff_join(AttnArgs a) {
    __shared__ float factor[2][kMaxSplits], low[4][4];
    __shared__ v4f sums[2][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t wide = (int64_t)a.tq * a.group, all = (int64_t)a.batch * a.Hk * wide;
    const int64_t row = blockIdx.x, number = row % wide, outer = row / wide;
    const int hk = (int)(outer % a.Hk), b = (int)(outer / a.Hk);
    const int t = token_of(a, (int)number), head = hk * a.group + (int)number - t * a.group;
    const Sequence s = sequence(a, b);
    if (t >= s.nq) return;
    const int64_t part = outer * a.splits * wide + number;
    const float *ml = a.parts + part * 4, *products = a.parts + all * a.splits * 4;
    const int n = threadIdx.x;
    v4f mine = {-__builtin_inff(), 0.f, -__builtin_inff(), 0.f};
    if (n < a.splits) mine = *(const v4f *)(ml + n * wide * 4);
    const float lam = weight_of(a.weight, head, lane).lam;
    float top[2], sum[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float m = mine[2 * i];
#pragma unroll
        for (int step = 1; step < 64; step <<= 1) m = fmaxf(m, __shfl_xor(m, step));
        if (lane == 0) low[i][wave] = m;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        top[i] = fmaxf(fmaxf(low[i][0], low[i][1]), fmaxf(low[i][2], low[i][3]));
        // (a split that saw no key has no products)
        const float f = mine[2 * i + 1] == 0.f ? 0.f : __builtin_amdgcn_exp2f(mine[2 * i] - top[i]);
        if (n < a.splits) factor[i][n] = f;
        const float part_sum = wave_sum(f * mine[2 * i + 1]);
        if (lane == 0) low[2 + i][wave] = part_sum;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) sum[i] = (low[2 + i][0] + low[2 + i][1]) + (low[2 + i][2] + low[2 + i][3]);
    // channels: pieces of 4, `turns` threads each
    const int pieces = (a.dv + 3) / 4, turns = 256 / pieces < a.splits ? 256 / pieces : a.splits;
    const int c = n % pieces * 4, turn = n / pieces;
    v4f y[2] = {v4f{0.f, 0.f, 0.f, 0.f}, v4f{0.f, 0.f, 0.f, 0.f}};
    if (turn < turns) {
        typedef float v4any __attribute__((ext_vector_type(4), aligned(4)));
        for (int k = turn; k < a.splits; k += turns) {
            const float *p = products + (part + k * wide) * 2 * a.dv + c;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float f = factor[i][k];
                if (f == 0.f) continue;
                if (c + 4 <= a.dv)
                    y[i] += f * *(const v4any *)(p + i * a.dv);
                else
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (c + j < a.dv) y[i][j] += f * p[i * a.dv + j];
            }
        }
    }
    sums[0][n] = y[0];
    sums[1][n] = y[1];
    __syncthreads();
    if (wave) return;                 // pieces: at most 64
    const bool live = lane < pieces;
    if (live)
        for (int k = 1; k < turns; ++k) {
            y[0] += sums[0][k * pieces + lane];
            y[1] += sums[1][k * pieces + lane];
        }
    else
        y[0] = y[1] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 2; ++i) y[i] *= sum[i] == 0.f ? 0.f : 1.f / sum[i];
    if (live) {
        const v4f out = y[0] - lam * y[1];
        store4(head_of<T>(a.o, s.batch, s.q0 + t, head), lane * 4, a.dv, out[0], out[1], out[2], out[3]);
    }
    if (!a.kept) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float *at = a.stats + (2 * (int64_t)head + i) * a.stat_rows * a.rows + s.row0 + t;
        if (lane == 0) at[0] = sum[i] == 0.f ? __builtin_inff() : top[i] - kMapsUp<T> + __builtin_amdgcn_logf(sum[i]);
        int16_t *to = a.kept + (((s.row0 + t) * a.H + head) * 2 + i) * a.dv;
        const float most = larger(larger(magnitude(y[i][0]), magnitude(y[i][1])), larger(magnitude(y[i][2]), magnitude(y[i][3])));
#pragma unroll
        for (int w = 0; w < kMaxValueWidth / kScaleWidth; ++w) {
            if (w * kScaleWidth >= a.dv) break;
            const bool in = lane * 4 / kScaleWidth == w;
            const KeptScale k = kept_scale(wave_largest(in ? most : 0.f));
            if (lane == 0) at[(1 + w) * a.rows] = k.scale;
            if (in)
                store4(to, lane * 4, a.dv, kept_code(y[i][0], k.inv), kept_code(y[i][1], k.inv), kept_code(y[i][2], k.inv),
                       kept_code(y[i][3], k.inv));
        }
    }
}

template <class T, bool WIDE, bool PIECES>
int forward(int cls, const AttnArgs &a, hipStream_t s) {
    const dim3 grid((unsigned)((int64_t)a.batch * a.Hk * a.row_tiles * a.splits)), block(cls < 2 || WIDE ? 256 : 128);
    constexpr int BLOCKS = WIDE ? 4 : 1, KT = WIDE ? 64 : 32, RUNS = WIDE ? 1 : 4;
    if (cls == 0)
        hipLaunchKernelGGL((k_diff_forward<T, 32, 64, BLOCKS, 2, KT, RUNS, PIECES>), grid, block, 0, s, a);
    else if (cls == 1)
        hipLaunchKernelGGL((k_diff_forward<T, 64, 128, BLOCKS, 2, KT, RUNS, PIECES>), grid, block, 0, s, a);
    else if (cls == 2)
        hipLaunchKernelGGL((k_diff_forward<T, 128, 128, WIDE ? 2 : 1, 1, 32, 1, PIECES>), grid, block, 0, s, a);
    else
        hipLaunchKernelGGL((k_diff_forward<T, 128, 256, WIDE ? 2 : 1, 1, 32, 1, PIECES>), grid, block, 0, s, a);
    return (int)hipGetLastError();
}
template <class T>
int forward(int cls, bool wide, const AttnArgs &a, hipStream_t s) {
    if (a.pieces) return wide ? forward<T, true, true>(cls, a, s) : forward<T, false, true>(cls, a, s);
    return wide ? forward<T, true, false>(cls, a, s) : forward<T, false, false>(cls, a, s);
}

}  // namespace

int launch_diff_forward(int type, int cls, bool wide, const AttnArgs &a, void *stream) {
    const hipStream_t s = (hipStream_t)stream;
    return type == NM_TYPE_F16 ? forward<half_t>(cls, wide, a, s) : forward<bf16_t>(cls, wide, a, s);
}

int launch_diff_join(int type, const AttnArgs &a, void *stream) {
    const dim3 grid((unsigned)((int64_t)a.batch * a.Hk * a.tq * a.group));
    if (type == NM_TYPE_F16)
        hipLaunchKernelGGL(k_diff_join<half_t>, grid, dim3(256), 0, (hipStream_t)stream, a);
    else
        hipLaunchKernelGGL(k_diff_join<bf16_t>, grid, dim3(256), 0, (hipStream_t)stream, a);
    return (int)hipGetLastError();
}

}  // namespace nmspmm
