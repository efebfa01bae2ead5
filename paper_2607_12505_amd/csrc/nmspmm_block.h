// Internal declarations of the transformer-block operators: kernel arguments
// and launch functions shared by their host file and their kernels.
#pragma once

#include "nmspmm_internal.h"

namespace nmspmm {

struct NormArgs {
    const void *y, *r;        // rows of ldy and ldr values; either may be null
    const float *gate;        // [groups x d] or null (1)
    nm_norm post, pre;
    void *res, *z;            // [m x d] or null
    int8_t *zq;               // [m x ldq] or null
    float *zs;                // [m], with zq
    int64_t ldy, ldr, ldq;
    int m, d, groups, per_group;
    float alpha;
};

struct NormGradArgs {
    const void *y, *res, *dz, *dres;
    const float *gate;
    nm_norm post, pre;
    void *dy, *dr;
    float *dgate, *dpre_weight, *dpre_bias, *dpost_weight, *dpost_bias;
    float *parts;             // [5][workgroups][d]
    float *gate_parts;        // [runs][2][d]: gate groups that several runs share
    int64_t ldy, ldr, lddz, lddres;
    int m, d, groups, per_group;
    int runs, turns;          // teams with rows (team t: rows t m / runs to (t + 1) m / runs), the most rows of one
    float alpha;
};
// Teams that take rows, the most rows of one, workgroups; of the form for pieces (vec) and for a norm after the block.
struct NormGradShape {
    int runs, turns, workgroups;
};
NormGradShape norm_grad_shape(int m, int d, bool vec, bool post);

struct QuantArgs {
    const void *x;
    int8_t *q;                // [m x ldq], ldq = k rounded up to 16
    float *scale;             // [m]
    int64_t ldx, ldq;
    int64_t m;
    int k;
};

// Rows of q as 16-byte pieces of rows of ldq bytes, zeros from k on.
struct PadArgs {
    const int8_t *q;
    int8_t *out;              // [m x ldo], ldo = k rounded up to 16
    int64_t ldq, ldo;
    int64_t m;
    int k;
};
int launch_pad_codes(const PadArgs &a, void *stream);

constexpr int kMaxNormWidth = 16384;
constexpr int64_t kMaxRows = 1 << 30;

inline int round16(int k) { return (k + 15) & ~15; }

// vec: rows are whole 16-byte pieces at 16-byte boundaries.
int launch_norm_residual(int type, bool vec, const NormArgs &a, void *stream);
int launch_norm_residual_backward(int type, bool vec, const NormGradArgs &a, int workgroups, void *stream);
int launch_quantize_rows(int type, bool vec, const QuantArgs &a, void *stream);

// ---------------------------------------------------------------- products

// GemmArgs plus what the epilogues of the block's products need.  `scale` and
// `qscale` hold the channels' scales and biases (qscale null: none).
struct BlockArgs : GemmArgs {
    const float *row_scale = nullptr;   // [m]
    void *out = nullptr;                // rows of ldo values, n_out of them wanted
    int64_t ldo = 0;
    int n_out = 0;
    int type = 0;                       // NM_TYPE_* of out (and of dh)
    int act = 0;                        // NM_ACT_*
    // few tokens: activations as values instead of codes (rows of ldx, kx of them)
    const void *x = nullptr;
    int64_t ldx = 0;
    int xtype = 0, kx = 0;
    // gradients of the gated block
    const void *dh = nullptr;           // [m] rows of lddh values
    int64_t lddh = 0;
    void *da = nullptr, *dat = nullptr; // [m x n], [n x ldt]
    int64_t ldt = 0;
    float *bias_parts = nullptr;        // [rows of waves x n] or null: a row for each wave's tokens of a tile
    void *out2 = nullptr;               // second half of interleaved rows
    int interleaved = 0;
};

constexpr int kDeepTile = 13;    // of kTiles: 128 ch x 64 tok, 4-slot ring
// Tiles that the products are built for, by what they write.
constexpr uint32_t scaled_tiles(int kind) {
    return 1u << 1 | 1u << 3 | 1u << 6 | 1u << 7 | 1u << 8 | 1u << 9 | 1u << 10 | 1u << 12 | 1u << 15 |
           (tile_built(kind, kDeepTile) ? 1u << kDeepTile : 0u);
}
constexpr uint32_t kGradTiles = 1u << 1 | 1u << 3 | 1u << 6;   // whole 64-token groups: the transposed rows' padding is written too
constexpr uint32_t kCastTiles = 1u << 1 | 1u << 3 | 1u << 6 | 1u << 12 | 1u << 4;

// The kernel of few tokens: the most that it is built for, and whether it takes them as values.
constexpr int kFewTokens = 32;
bool few_takes_values(int m, int k);
// The tile of nmspmm_rows.h, numbered after kTiles.
struct RowTile {
    int wn, wm, fn, fm;
    constexpr int tile_n() const { return wn * fn * kFragRows; }
    constexpr int tile_m() const { return wm * fm * 16; }
};
constexpr int kRowTile = kNumSchedules;
constexpr RowTile kRowTileShape = {4, 2, 4, 5};
constexpr int tile_n_of(int tile) { return tile == kRowTile ? kRowTileShape.tile_n() : kTiles[tile].tile_n(); }
constexpr int tile_m_of(int tile) { return tile == kRowTile ? kRowTileShape.tile_m() : kTiles[tile].tile_m(); }
int launch_few(int kind, bool gated, const BlockArgs &a, void *stream);
int launch_scaled(int kind, int tile, const BlockArgs &a, int grid, void *stream);
int launch_gated(int kind, int tile, const BlockArgs &a, int grid, void *stream);
int launch_gated_grad(int tile, const BlockArgs &a, int grid, void *stream);
// C = A B^T of 16-bit rows (a.k counts bytes), to `type`: one or two of them on the same tile in one launch (their
// gemm_grid: workgroups, 0 for none).
struct CastPair {
    BlockArgs part[2];
};
int launch_cast(int type, int tile, const CastPair &a, void *stream);

// Codes [rows x ld] with a scale each -> their transpose [cols x ldt] in 16 bits, each code times the power of two
// of its row's scale (exact); zeros from `rows` to ldt.
struct TransposeArgs {
    const int8_t *q;
    const float *scale;
    void *out;
    int64_t ld, ldt;
    int rows, cols;
};
// Two such (rows 0: none) and `counters` (or null) set to zero, in one launch.
int launch_transpose_codes(int type, const TransposeArgs &a, const TransposeArgs &b, int *counters, int count,
                           void *stream);
// dst[c] = sum over rows of parts[rows x n] for the channels of interleaved rows.
int launch_bias_sums(const float *parts, int rows, int n, int n_out, float *gate, float *up, void *stream);

}  // namespace nmspmm
