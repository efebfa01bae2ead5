// C entry points of the transformer-block operators: argument checks,
// workspaces and dispatch (host only).
#include "nmspmm_block.h"

using namespace nmspmm;

namespace {

bool valid_type(int t) { return t >= NM_TYPE_F16 && t <= NM_TYPE_F32; }
int type_bytes(int t) { return t == NM_TYPE_F32 ? 4 : 2; }
bool aligned(const void *p, int to) { return ((uintptr_t)p & (uintptr_t)(to - 1)) == 0; }

// Whether rows of `width` values with this stride are whole 16-byte pieces at
// 16-byte boundaries (8 values of a 16-bit type at once, 4 + 4 of binary32).
bool pieces(const void *p, int64_t ld, int width, int type) {
    return !p || (aligned(p, 16) && ld % 8 == 0 && width % 8 == 0);
}

bool valid_norm(const nm_norm &n) {
    if (n.kind == NM_NORM_NONE) return true;
    return (n.kind == NM_NORM_RMS || n.kind == NM_NORM_LAYER) && n.eps > 0.f && aligned(n.weight, 4) &&
           aligned(n.bias, 4);
}
nm_norm as_read(nm_norm n) {
    if (n.kind == NM_NORM_NONE) n.weight = n.bias = nullptr;
    return n;
}

nm_status check_rows(int type, int m, int d, int groups) {
    if (!valid_type(type)) return NM_ERR_ARG;
    if (m < 0 || m >= kMaxRows || d < 1 || d > kMaxNormWidth || groups < 1) return NM_ERR_SHAPE;
    return m % groups == 0 ? NM_OK : NM_ERR_SHAPE;
}

size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace

extern "C" nm_status nm_quantize_rows(const void *x, int64_t ldx, int type, int m, int k, int8_t *xq, float *scale,
                                      void *stream) {
    if (!valid_type(type)) return NM_ERR_ARG;
    if (m < 0 || m >= kMaxRows || k < 1 || k >= (1 << 30) || ldx < k) return NM_ERR_SHAPE;
    if (m == 0) return NM_OK;
    if (!x || !xq || !scale || !aligned(x, type_bytes(type)) || !aligned(xq, 16) || !aligned(scale, 4))
        return NM_ERR_ARG;
    QuantArgs a;
    a.x = x;
    a.q = xq;
    a.scale = scale;
    a.ldx = ldx;
    a.ldq = round16(k);
    a.m = m;
    a.k = k;
    return launch_quantize_rows(type, pieces(x, ldx, k, type), a, stream) == 0 ? NM_OK : NM_ERR_HIP;
}

extern "C" nm_status nm_norm_residual(const nm_norm_args *args, void *stream) {
    if (!args) return NM_ERR_ARG;
    const nm_norm_args &g = *args;
    nm_status st = check_rows(g.type, g.m, g.d, g.groups);
    if (st != NM_OK) return st;
    if ((!g.y && !g.r) || (!g.res && !g.z && !g.zq) || (g.zq && !g.zs) || (!g.gate && g.groups != 1))
        return g.m == 0 ? NM_OK : NM_ERR_ARG;
    if (!valid_norm(g.post) || !valid_norm(g.pre)) return NM_ERR_ARG;
    if ((g.y && g.ldy < g.d) || (g.r && g.ldr < g.d)) return NM_ERR_SHAPE;
    if (g.m == 0) return NM_OK;
    const int eb = type_bytes(g.type);
    for (const void *p : {g.y, g.r, (const void *)g.res, (const void *)g.z})
        if (!aligned(p, eb)) return NM_ERR_ARG;
    if (!aligned(g.gate, 4) || !aligned(g.zs, 4) || !aligned(g.zq, 16)) return NM_ERR_ARG;
    NormArgs a;
    a.y = g.y;
    a.r = g.r;
    a.gate = g.gate;
    a.post = as_read(g.post);
    a.pre = as_read(g.pre);
    a.res = g.res;
    a.z = g.z;
    a.zq = g.zq;
    a.zs = g.zs;
    a.ldy = g.ldy;
    a.ldr = g.ldr;
    a.ldq = round16(g.d);
    a.m = g.m;
    a.d = g.d;
    a.groups = g.groups;
    a.per_group = g.m / g.groups;
    a.alpha = g.alpha;
    const bool vec = pieces(g.y, g.ldy, g.d, g.type) && pieces(g.r, g.ldr, g.d, g.type) &&
                     pieces(g.res, g.d, g.d, g.type) && pieces(g.z, g.d, g.d, g.type) && g.d % 8 == 0;
    return launch_norm_residual(g.type, vec, a, stream) == 0 ? NM_OK : NM_ERR_HIP;
}

extern "C" nm_status nm_norm_residual_backward_workspace(int m, int d, int groups, size_t *bytes) {
    if (!bytes) return NM_ERR_ARG;
    nm_status st = check_rows(NM_TYPE_F32, m, d, groups);
    if (st != NM_OK) return st;
    *bytes = 0;
    if (m == 0) return NM_OK;
    const NormGradShape s = norm_grad_shape(m, d);
    *bytes = round256((size_t)5 * s.workgroups * d * 4);
    if (groups > 1) *bytes += (size_t)s.workgroups * s.teams * 2 * d * 4;
    return NM_OK;
}

extern "C" nm_status nm_norm_residual_backward(const nm_norm_grad_args *args, void *ws, size_t ws_bytes,
                                               void *stream) {
    if (!args) return NM_ERR_ARG;
    const nm_norm_grad_args &g = *args;
    nm_status st = check_rows(g.type, g.m, g.d, g.groups);
    if (st != NM_OK) return st;
    if (!valid_norm(g.post) || !valid_norm(g.pre)) return NM_ERR_ARG;
    float *sums[] = {g.dgate, g.dpre_weight, g.dpre_bias, g.dpost_weight, g.dpost_bias};
    for (const float *p : sums)
        if (!aligned(p, 4)) return NM_ERR_ARG;
    if (g.m == 0) {
        for (float *p : sums) {
            const size_t rows = p == g.dgate ? (size_t)g.groups : 1;
            if (p && launch_zero(p, rows * g.d * 4, stream) != 0) return NM_ERR_HIP;
        }
        return NM_OK;
    }
    const bool to_block = g.dy || g.dgate || g.dpost_weight || g.dpost_bias;
    if (!g.dr && !to_block && !g.dpre_weight && !g.dpre_bias) return NM_ERR_ARG;
    if ((!g.dz && !g.dres) || (to_block && !g.y) || (g.pre.kind != NM_NORM_NONE && !g.res) ||
        (!g.gate && g.groups != 1))
        return NM_ERR_ARG;
    if (((g.dpre_weight || g.dpre_bias) && g.pre.kind == NM_NORM_NONE) ||
        ((g.dpost_weight || g.dpost_bias) && g.post.kind == NM_NORM_NONE))
        return NM_ERR_ARG;
    if ((g.y && g.ldy < g.d) || (g.res && g.ldres < g.d) || (g.dz && g.lddz < g.d) || (g.dres && g.lddres < g.d))
        return NM_ERR_SHAPE;
    const int eb = type_bytes(g.type);
    for (const void *p : {g.y, g.res, g.dz, g.dres, (const void *)g.dy, (const void *)g.dr})
        if (!aligned(p, eb)) return NM_ERR_ARG;
    if (!aligned(g.gate, 4)) return NM_ERR_ARG;
    size_t need = 0;
    st = nm_norm_residual_backward_workspace(g.m, g.d, g.groups, &need);
    if (st != NM_OK) return st;
    if (!ws || ws_bytes < need || !aligned(ws, 16)) return NM_ERR_WORKSPACE;
    const NormGradShape s = norm_grad_shape(g.m, g.d);
    NormGradArgs a;
    a.y = to_block ? g.y : nullptr;
    a.res = g.res;
    a.dz = g.dz;
    a.dres = g.dres;
    a.gate = g.gate;
    a.post = as_read(g.post);
    a.pre = as_read(g.pre);
    a.dy = g.dy;
    a.dr = g.dr;
    a.dgate = g.dgate;
    a.dpre_weight = g.dpre_weight;
    a.dpre_bias = g.dpre_bias;
    a.dpost_weight = g.dpost_weight;
    a.dpost_bias = g.dpost_bias;
    a.parts = (float *)ws;
    a.gate_parts = (float *)((char *)ws + round256((size_t)5 * s.workgroups * g.d * 4));
    a.ldy = g.ldy;
    a.ldr = g.ldres;
    a.lddz = g.lddz;
    a.lddres = g.lddres;
    a.m = g.m;
    a.d = g.d;
    a.groups = g.groups;
    a.per_group = g.m / g.groups;
    a.run = s.run;
    a.alpha = g.alpha;
    const bool vec = pieces(a.y, g.ldy, g.d, g.type) && pieces(g.res, g.ldres, g.d, g.type) &&
                     pieces(g.dz, g.lddz, g.d, g.type) && pieces(g.dres, g.lddres, g.d, g.type) &&
                     pieces(g.dy, g.d, g.d, g.type) && pieces(g.dr, g.d, g.d, g.type) && g.d % 8 == 0;
    return launch_norm_residual_backward(g.type, vec, a, s.workgroups, stream) == 0 ? NM_OK : NM_ERR_HIP;
}
