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
    float *gate_parts;        // [teams][2][d]: gate groups that several runs share
    int64_t ldy, ldr, lddz, lddres;
    int m, d, groups, per_group;
    int run;                  // rows of one team
    float alpha;
};
// Teams of waves that share a workgroup, rows that one team takes, workgroups.
struct NormGradShape {
    int teams, run, workgroups;
};
NormGradShape norm_grad_shape(int m, int d);

struct QuantArgs {
    const void *x;
    int8_t *q;                // [m x ldq], ldq = k rounded up to 16
    float *scale;             // [m]
    int64_t ldx, ldq;
    int64_t m;
    int k;
};

constexpr int kMaxNormWidth = 16384;
constexpr int64_t kMaxRows = 1 << 30;

inline int round16(int k) { return (k + 15) & ~15; }

// vec: rows are whole 16-byte pieces at 16-byte boundaries.
int launch_norm_residual(int type, bool vec, const NormArgs &a, void *stream);
int launch_norm_residual_backward(int type, bool vec, const NormGradArgs &a, int workgroups, void *stream);
int launch_quantize_rows(int type, bool vec, const QuantArgs &a, void *stream);

}  // namespace nmspmm
