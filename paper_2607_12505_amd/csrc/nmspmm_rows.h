// A k-loop for int8 products whose operands are both plain rows (a dense weight) and
// whose epilogue is long: tiles of 256 x 160 on 8 waves whose ring of three 64-byte
// k-steps takes half of a compute unit's LDS, so two workgroups share it and one
// multiplies while the other starts, waits at its barrier or runs its epilogue.  At
// 64 bytes of each row a k-step, a wave has 4 + 5 operand pieces for 20 matrix
// instructions; the loads to LDS bring 41 bytes a cycle of them (128 x 128 tiles
// would need 64, all that the path gives).  Measured at 18464 x 4096 -> 1024 with the loads
// left out 67 us, with the matrix instructions left out 85, whole 88: the wait for the
// operands, not the stores, is what the second workgroup does not cover, and
// plain products are as fast or faster on the tiles of nmspmm_gemm.h.
#pragma once

#include "nmspmm_gemm.h"

namespace nmspmm {
namespace {

template <int WN_, int WM_, int FN_, int FM_>
struct RowGeometry {
    static constexpr int WN = WN_, WM = WM_, FN = FN_, FM = FM_, NW = WN * WM, R = 3;
    static constexpr int BN = WN * FN * 16, BM = WM * FM * 16;
    static constexpr int XC = BM / 16, NC = (BN + BM) / 16;      // loads of 1024 bytes (16 rows) a k-step
    static constexpr int SLOT = NC * 1024;
    static constexpr int ND = (NC + NW - 1) / NW, EXTRA = NC % NW;   // a wave's: ND, or (past EXTRA) one less
    static constexpr int FEW = EXTRA ? ND - 1 : ND;
    static constexpr int CPR = FN * 4, RPI = 64 / CPR;
    static constexpr int stage_rows(int eb) { return 16 * FN * eb >= 64 ? 16 : 1024 / (16 * FN * eb); }
    static constexpr int stage_bytes(int eb) { return stage_rows(eb) * (FN * 16 * eb + 16); }
    static constexpr int STG = stage_bytes(4) > stage_bytes(1) ? stage_bytes(4) : stage_bytes(1);
    static constexpr int LDSB = R * SLOT;
    static_assert(NW * STG <= LDSB && 2 * LDSB <= 160 * 1024 && 64 % CPR == 0, "two workgroups a compute unit");
};

template <int WN, int WM, int FN, int FM, class EPI, class ARGS>
__device__ __forceinline__ void gemm_rows(const ARGS &a, int8_t *lds) {
    using G = RowGeometry<WN, WM, FN, FM>;
    constexpr int BN = G::BN, BM = G::BM, NW = G::NW, R = G::R;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) int8_t *)lds;

    const int lid = map_block(blockIdx.x, gridDim.x);
    int tn, tm;
    tile_order(lid, a.tiles_n, a.tiles_m, a.group_rows, &tn, &tm);
    const int tid = threadIdx.x, lane = tid & 63, lg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wn = wave % WN, wm = wave / WN;
    const int tok0 = tm * BM, ch0 = tn * BN;
    const int nsteps = (a.k + 63) >> 6;
    const int ragged = a.k & 63;                                         // bytes of the last k-step, if it is short
    const int t_tail = ragged ? nsteps - 1 : -1;

    // --- loads.  Instruction q of a k-step: 16 rows, lane L row L / 4 and, at
    // place L % 4, the row's chunk (L % 4) ^ ((row / 2) % 4): eight consecutive rows
    // of an operand read lie in distinct banks (by row / 4 half of the LDS cycles were
    // conflicts).  Rows past the end read the last one.
    const int place = ((lane & 3) ^ ((lane >> 3) & 3)) * 16;
    uint32_t off[G::ND];
#pragma unroll
    for (int c = 0; c < G::ND; ++c) {
        const int q = NW * c + wave, r = lane >> 2;
        const int row = q < G::XC ? tok0 + 16 * q + r : ch0 + 16 * (q - G::XC) + r;
        const int last = (q < G::XC ? a.m : a.n) - 1;
        off[c] = (uint32_t)(row < last ? row : last) * (uint32_t)a.k + (uint32_t)place;
    }
    const int8_t *xp = a.X, *wp = a.A;
    asm("" : "+s"(xp), "+s"(wp));
    auto load = [&](int t, int st, int live) {
#pragma unroll
        for (int c = 0; c < G::ND; ++c) {
            const int q = NW * c + wave;
            const bool x = NW * c + NW <= G::XC || (NW * c < G::XC && q < G::XC);
            const int l = NW * c + NW <= G::NC || q < G::NC ? live : 0;
            dma16o_if((x ? xp : wp) + (uint64_t)t * 64, off[c], lds0 + st * G::SLOT + q * 1024,
                      __builtin_amdgcn_readfirstlane(l));
        }
    };
    // before the short last k-step: chunks past k read the row's last chunk (the weight's are masked)
    auto clamp_tail = [&](int t) {
        if (t == t_tail) {
            const uint32_t back = place >= ragged ? (uint32_t)(place - (ragged - 16)) : 0u;
#pragma unroll
            for (int c = 0; c < G::ND; ++c) off[c] -= back;
        }
    };
    // this wave's loads of the k-step before the last one issued have landed
    auto landed = [&](bool later) {
        if (!later) {
            wait_only<0>();
        } else if (G::EXTRA && wave < G::EXTRA) {
            wait_only<G::ND>();
        } else {
            wait_only<G::FEW>();
        }
        wait_then_barrier<63>();
    };

    v4i acc[FN][FM];
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) acc[i][j] = v4i{0, 0, 0, 0};

    const int sw = (lg ^ ((lane >> 1) & 3)) << 4;                        // the lane's chunk of its row
    const int8_t *xrow = lds + (wm * FM * 16 + (lane & 15)) * 64 + sw;
    const int8_t *wrow = lds + G::XC * 1024 + (wn * FN * 16 + (lane & 15)) * 64 + sw;

    clamp_tail(0);
    load(0, 0, nsteps);
    if (nsteps > 1) clamp_tail(1);
    load(1, 1, nsteps - 1);
    int st = 0;
    for (int t = 0; t < nsteps; ++t) {
        landed(t + 1 < nsteps);        // k-step t is in LDS, and nobody reads slot t - 1 any more
        const int next = st == 0 ? R - 1 : st - 1;
        clamp_tail(t + 2);
        load(t + 2, next, nsteps - 2 - t);
        v4i w[FN], x[FM];
#pragma unroll
        for (int i = 0; i < FN; ++i) w[i] = *(const v4i *)(wrow + st * G::SLOT + i * 1024);
#pragma unroll
        for (int j = 0; j < FM; ++j) x[j] = *(const v4i *)(xrow + st * G::SLOT + j * 1024);
        if (t == t_tail && 16 * lg >= ragged) {
#pragma unroll
            for (int i = 0; i < FN; ++i) w[i] = v4i{0, 0, 0, 0};
        }
#pragma unroll
        for (int j = 0; j < FM; ++j)
#pragma unroll
            for (int i = 0; i < FN; ++i) acc[i][j] = mfma_rows<NM_KIND_DENSE>(w[i], x[j], acc[i][j]);
        st = st + 1 == R ? 0 : st + 1;
    }
    wait_only<0>();
    __syncthreads();                   // every wave is done with the ring
    // multipliers straight from memory: the other workgroup covers their latency
    const float *first = EPI::first(a), *second = EPI::second(a);
    const int c0 = ch0 + wn * FN * 16 + 4 * lg;
    auto multiplier = [&](int h, int i) {
        const int ch = c0 + i * 16;
        return *(const v4f *)((h ? second : first) + (ch < a.n ? ch : 0));
    };
    EPI::template finish<G>(a, TileAt{tok0 + wm * FM * 16, ch0 + wn * FN * 16, 0, tm, tn, lane}, acc,
                            lds + wave * G::STG, multiplier, nullptr);
}

}  // namespace
}  // namespace nmspmm
