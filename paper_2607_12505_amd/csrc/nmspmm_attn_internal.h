// Internal declarations of rotary positions and differential attention: kernel
// arguments and launch functions shared by their host file and their kernels.
#pragma once

#include "nmspmm_internal.h"

namespace nmspmm {

// ---------------------------------------------------------------- rotary positions

struct RotaryPart {
    const void *x;
    void *out;
    int64_t x_token, x_head, out_token, out_head;   // in values
    int heads;
};
struct RotaryArgs {
    RotaryPart part[2];       // the second without heads: absent
    const void *pos;          // [axes] rows of ld_pos positions, int32 or binary32
    int64_t ld_pos;
    const double *freq;       // [pairs]
    const int32_t *axis;      // [pairs]
    int64_t tokens;
    int pos_float, pairs, d, interleaved, axes;
    float sign;               // of the angle
};
constexpr int kMaxRotaryWidth = 1024;
int launch_rotary(int type, const RotaryArgs &a, void *stream);

// ---------------------------------------------------------------- differential attention

constexpr int kMaxHeadWidth = 128, kMaxValueWidth = 256;
constexpr int64_t kMaxAttnTokens = 1 << 28;   // of a sequence: sums of positions and windows stay in 32 bits
constexpr int64_t kMaxTokenStride = 1 << 22;  // a tile's rows lie within 2^31 bytes

// A tensor of heads; strides in values.
struct Heads {
    char *p;
    int64_t batch, token, head;
};

struct AttnArgs {
    Heads q, k, v, o;
    int16_t *kept;            // [rows][H][2][dv]: codes of both maps' products with v (or null)
    float *stats;             // [2 H][stat_rows][rows]: base-2 logarithms of the maps' sums, scales of the codes (or null)
    int stat_rows;
    const int32_t *q_offsets, *k_offsets, *q_lens, *k_lens;
    int64_t total_q, total_k; // rows of packed tensors
    int64_t rows;             // rows of q in all: batch * tq, or total_q
    int batch, tq, tk, H, Hk, group, d, dv, left, right;
    float scale, scale2;      // and in base 2
    nm_diff_weight weight;
    int pieces;               // q, k, v (and do) are whole 16-byte pieces at their boundaries
    int row_tiles, splits;
    float *parts;             // [batch * Hk * splits * tq * group] x 4: m1, l1, m2, l2, then the same x 2 dv values
    // backward
    Heads grad, dq, dk, dv_;  // do and the gradients
    float *delta;             // [2 H][rows]: do . o1, do . o2
    float *dlam_parts;        // [H][batch * row_tiles * 4]
    int dlam_count;           // batch * row_tiles * 4
    float *tops;              // [batch * Hk][row_tiles * 4]: of 32 rows, at least their largest |do| |v| max(1, |lam|)
    float *norms;             // [batch * Hk][key_tiles]: the largest |v|^2 of a tile's keys
    float *dlam, *dq1, *dk1, *dq2, *dk2;
    int key_tiles, key_splits;
    float *key_parts;         // [batch * Hk * key_splits * tk][2 d + dv] (key_splits > 1)
};

// Width classes that the kernels are built for: (32, 64), (64, 128), (128, 128), (128, 256).
inline int width_class(int d, int dv) { return d <= 32 && dv <= 64 ? 0 : d <= 64 && dv <= 128 ? 1 : dv <= 128 ? 2 : 3; }
constexpr int kScaleWidth = 128;              // channels of a scale of `kept`
inline int stat_rows_of(int dv) { return 1 + (dv + kScaleWidth - 1) / kScaleWidth; }
// Rows of a workgroup of the forward pass: many, and few whose keys may be split.
inline int wide_rows(int cls) { return cls >= 2 ? 64 : 128; }
constexpr int kFewRows = 32, kFewRowsKeys = 32, kMaxSplits = 256;
inline int key_runs(int cls) { return cls >= 2 ? 1 : 4; }    // of a workgroup of few rows
// Of the backward pass: rows and keys of a workgroup, keys of a tile.
constexpr int kGradRows = 128, kGradKeys = 128, kGradKeyTile = 64;

int launch_diff_forward(int type, int cls, bool wide, const AttnArgs &a, void *stream);
int launch_diff_join(int type, const AttnArgs &a, void *stream);
int launch_diff_norms(const AttnArgs &a, void *stream);
int launch_diff_grad_q(int type, int cls, const AttnArgs &a, void *stream);
int launch_diff_grad_k(int type, int cls, const AttnArgs &a, void *stream);
int launch_diff_join_keys(int type, const AttnArgs &a, void *stream);

}  // namespace nmspmm
