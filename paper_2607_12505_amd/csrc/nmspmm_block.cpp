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
bool pieces(const void *p, int64_t ld, int width) {
    return !p || (aligned(p, 16) && ld % 8 == 0 && width % 8 == 0);
}

bool valid_norm(const nm_norm &n) {
    if (n.kind == NM_NORM_NONE) return true;
    return (n.kind == NM_NORM_RMS || n.kind == NM_NORM_LAYER) && n.eps > 0.f && aligned(n.weight, 4) &&
           aligned(n.bias, 4);
}
constexpr nm_norm kNoNorm = {NM_NORM_NONE, 0.f, nullptr, nullptr};
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
    if (m < 0 || m >= kMaxRows || k < 1 || k >= (1 << 28) || ldx < k) return NM_ERR_SHAPE;
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
    return launch_quantize_rows(type, pieces(x, ldx, k), a, stream) == 0 ? NM_OK : NM_ERR_HIP;
}

extern "C" nm_status nm_pad_codes(const int8_t *q, int64_t ldq, int m, int k, int8_t *out, void *stream) {
    if (m < 0 || m >= kMaxRows || k < 1 || k >= (1 << 28) || ldq < k) return NM_ERR_SHAPE;
    if (m == 0) return NM_OK;
    if (!q || !out || !aligned(out, 16)) return NM_ERR_ARG;
    const PadArgs a = {q, out, ldq, round16(k), m, k};
    return launch_pad_codes(a, stream) == 0 ? NM_OK : NM_ERR_HIP;
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
    // an absent term is absent whole: a norm's bias, a gate or alpha times nothing adds nothing, whatever they hold
    NormArgs a;
    a.y = g.y;
    a.r = g.r;
    a.gate = g.y ? g.gate : nullptr;
    a.post = g.y ? as_read(g.post) : kNoNorm;
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
    a.groups = g.y ? g.groups : 1;
    a.per_group = g.m / a.groups;
    a.alpha = g.r ? g.alpha : 0.f;
    const bool vec = pieces(g.y, g.ldy, g.d) && pieces(g.r, g.ldr, g.d) &&
                     pieces(g.res, g.d, g.d) && pieces(g.z, g.d, g.d) && g.d % 8 == 0;
    return launch_norm_residual(g.type, vec, a, stream) == 0 ? NM_OK : NM_ERR_HIP;
}

extern "C" nm_status nm_norm_residual_backward_workspace(int m, int d, int groups, size_t *bytes) {
    if (!bytes) return NM_ERR_ARG;
    nm_status st = check_rows(NM_TYPE_F32, m, d, groups);
    if (st != NM_OK) return st;
    *bytes = 0;
    if (m == 0) return NM_OK;
    // the most of what the forms of the kernel need
    size_t parts = 0, runs = 0;
    for (int form = 0; form < 4; ++form) {
        const NormGradShape s = norm_grad_shape(m, d, form & 1, form & 2);
        if ((size_t)s.workgroups > parts) parts = s.workgroups;
        if ((size_t)s.runs > runs) runs = s.runs;
    }
    *bytes = round256(5 * parts * d * 4);
    if (groups > 1) *bytes += runs * 2 * d * 4;
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
    NormGradArgs a;
    a.y = to_block ? g.y : nullptr;
    a.res = g.res;
    a.dz = g.dz;
    a.dres = g.dres;
    a.gate = g.gate;
    a.post = as_read(g.post);
    a.pre = g.dz ? as_read(g.pre) : kNoNorm;     // without dz nothing comes through it, whatever res holds
    a.dy = g.dy;
    a.dr = g.dr;
    a.dgate = g.dgate;
    a.dpre_weight = g.dpre_weight;
    a.dpre_bias = g.dpre_bias;
    a.dpost_weight = g.dpost_weight;
    a.dpost_bias = g.dpost_bias;
    a.parts = (float *)ws;
    a.ldy = g.ldy;
    a.ldr = g.ldres;
    a.lddz = g.lddz;
    a.lddres = g.lddres;
    a.m = g.m;
    a.d = g.d;
    a.groups = g.groups;
    a.per_group = g.m / g.groups;
    a.alpha = g.alpha;
    const bool vec = pieces(a.y, g.ldy, g.d) && pieces(g.res, g.ldres, g.d) &&
                     pieces(g.dz, g.lddz, g.d) && pieces(g.dres, g.lddres, g.d) &&
                     pieces(g.dy, g.d, g.d) && pieces(g.dr, g.d, g.d) && g.d % 8 == 0;
    const NormGradShape s = norm_grad_shape(g.m, g.d, vec, a.post.kind != NM_NORM_NONE && a.y);
    a.runs = s.runs;
    a.turns = s.turns;
    a.gate_parts = (float *)((char *)ws + round256((size_t)5 * s.workgroups * g.d * 4));
    return launch_norm_residual_backward(g.type, vec, a, s.workgroups, stream) == 0 ? NM_OK : NM_ERR_HIP;
}

// ---------------------------------------------------------------- products

namespace {

constexpr int64_t kMaxReduction = 1 << 17;   // 127 * 127 * 2^17 < 2^31

nm_status check_weight(const nm_scaled_weight *w, bool gated) {
    if (!w) return NM_ERR_ARG;
    nm_status st = check_desc(w->desc);
    if (st != NM_OK) return st;
    const nm_desc &d = *w->desc;
    if (w->n < 1 || w->k < 1 || w->k > d.k || d.k % 16 != 0 || d.k - w->k >= 16 || d.n % 4 != 0) return NM_ERR_ARG;
    if (gated ? d.n != 2 * ((w->n + 31) / 32 * 32) : w->n > d.n) return NM_ERR_ARG;
    if (d.k >= kMaxReduction) return NM_ERR_SHAPE;
    if (d.vals_bytes + d.meta_bytes >= kWeightLimit) return NM_ERR_SHAPE;
    if (!w->vals || (d.meta_bytes && !w->meta) || !w->scale || !aligned(w->vals, 16) || !aligned(w->meta, 16) ||
        !aligned(w->scale, 16) || !aligned(w->bias, 16))
        return NM_ERR_ARG;
    return NM_OK;
}

// Whether codes of m tokens take the kernel of few tokens (n: rows of the weight).  It
// repeats the codes for every 16 channels, so it loses where they outweigh its start,
// and with long dense rows of both projections of a gated block.  Times against the tiles'
// in us, weights from memory, on a grid of k 256 to 16384, n 512 to 32768 (gated: k 512 to 4096) and m to 32:
//   dense 1024 -> 4096 with 1 token 3.3 to 4.2, with 32 4.1 to 4.6; 4096 -> 4096 with 16 7.2 to 7.2;
//     2048 -> 6144 with 4 5.6 to 5.4, with 16 6.5 to 5.5; 1024 -> 16384 with 8 5.9 to 6.1, with 16 6.6 to 6.2;
//     4096 -> 11008 with 16 15.1 to 12.3
//   gated dense 1024 -> 2 x 4096 with 16 4.7 to 5.0; 2048 -> 2 x 1024 with 4 4.7 to 4.6, with 16 5.1 to 4.6;
//     4096 -> 2 x 2048 with 1 7.8 to 7.3; 1024 -> 2 x 2048 with 32 4.5 to 4.1, 512 -> 2 x 4096 3.8 to 4.0
//   2:4 4096 -> 4096 with 16 5.8 to 6.2; 2048 -> 8192 with 8 5.0 to 5.2, with 16 5.6 to 5.3
//   4:8 (weights of 3:8 to 5:8 cost the tiles more, which expand a block for every token tile) 4096 ->
//     4096 with 16 5.8 to 9.8, with 32 7.5 to 9.7; 4096 -> 16384 with 16 15.3 to 13.9; 1024 -> 8192 with 32
//     5.1 to 5.2, 1024 -> 16384 7.9 to 6.7, 2048 -> 6144 7.4 to 6.8
// Within the rule the grid's worst are 1.12 (dense 256 -> 32768 with 16, 5.8 to 5.2) and 1.10 (4:8 4096 -> 16384 with 16).
bool takes_few(int kind, bool gated, int64_t m, int64_t n, int64_t k) {
    const bool dense = kind == NM_KIND_DENSE;
    if (m > kFewTokens) return false;
    if (layout_mask_values(kind) > 0)
        return m <= 16 || (n * k <= 1 << 24 && (n <= 4096 || (n <= 8192 && k <= 1024)));
    if (m > 16) return n * k <= 1 << 22 && n <= 8192 && k <= (dense && gated ? 512 : 1024);
    if (n * k > 1 << 24) return false;
    if (dense && gated) return k <= 1024 || (k <= 2048 && m <= 4);
    return n <= 4096 || (m * n * k <= 1 << 27 && (!dense || k <= 1024));
}

// Whether a compact weight is expanded once for the call, and the bytes of that.
int64_t expansion(const nm_desc &d, int m) {
    nm_plan plan;
    if (!kind_is_compact(d.kind) || takes_few(d.kind, false, m, d.n, d.k) ||   // (a compact kind: gated or not)
        make_plan(d.kind, m, d.n, d.k, NM_OUT_F16, &plan) != NM_OK)
        return 0;
    return plan.expand ? plan.expand_bytes : 0;
}

// The codes of x and their scales at the start of the workspace.
size_t codes_bytes(int m, int k) { return round256((size_t)m * k) + round256((size_t)m * 4); }

void fill_product(BlockArgs &a, int m, const nm_scaled_weight &w) {
    const nm_desc &d = *w.desc;
    a.Y = nullptr;
    a.Yh = nullptr;
    a.Yq = nullptr;
    a.scale = w.scale;
    a.qscale = w.bias;
    a.counters = nullptr;
    a.partials = nullptr;
    a.m = m;
    a.n = d.n;
    a.k = d.k;
    a.k_steps = d.k_steps;
    a.n_frags = d.n_frags;
    a.split_k = 1;
    a.n_out = w.n;
}

int place_tiles(BlockArgs &a, int tile) {
    const int tn = tile_n_of(tile), tm = tile_m_of(tile);
    a.tiles_n = (a.n + tn - 1) / tn;
    a.tiles_m = (a.m + tm - 1) / tm;
    a.group_rows = group_rows_for(a.tiles_m, tm);
    a.gemm_grid = a.tiles_n * a.tiles_m * a.split_k;
    return a.gemm_grid;
}

// What the estimate of a GEMM's time is given as output: the bytes written for each weight row.
int out_mode_for(int type, bool gated) {
    return gated ? (type == NM_TYPE_F32 ? NM_OUT_F16 : NM_OUT_I8) : type == NM_TYPE_F32 ? NM_OUT_I32 : NM_OUT_F16;
}

// The tile of a product.  Dense gated blocks with many tiles and a short reduction
// take the tile of which two share a compute unit: one's epilogue (an exponential a
// value) runs beside the other's products.  Of 42 gated shapes with 0.5 to 12 tiles a unit, the
// 15 within the rule took 0.80 to 1.03 of the time of the estimate's tile (0.92 on
// average; 18464 x 1024 -> 2736: 120.5 us against 128.1).  Outside it (28 shapes, before the
// activation was decided once for four values) 0.91 to 1.35; 32 plain products 0.83 to 1.29,
// 1.07 on average.
//   A 4:2 operand and a long reduction take the 4-slot ring where its tiles fit the
// device at once, two a compute unit: the deeper ring covers the load latency that few
// workgroups leave bare.  Of 11 random shapes within the rule, operands out of L2, 10 took
// 0.79 to 0.95 of the estimate's tile and one 0.98 (1906 x 1200 -> 1504 10.5 us against 11.7);
// 13 of k 320 to 900 at that many tiles 0.97 to 1.10; past two a unit 31 shapes 1.12 to 1.47.
int product_tile(int kind, bool gated, int m, int n, int k, int out_mode) {
    const int tn = tile_n_of(kRowTile), tm = tile_m_of(kRowTile);
    const int64_t tiles = (int64_t)((n + tn - 1) / tn) * ((m + tm - 1) / tm);
    if (gated && kind == NM_KIND_DENSE && k <= 1536 && 2 * tiles >= 5 * device_cu_count()) return kRowTile;
    if (kind == NM_KIND_SP42 && k >= 1024) {
        const TileCfg &t = kTiles[kDeepTile];
        const int64_t deep = (int64_t)((n + t.tile_n() - 1) / t.tile_n()) * ((m + t.tile_m() - 1) / t.tile_m());
        if (deep > device_cu_count() && deep <= 2 * device_cu_count()) return kDeepTile;
    }
    return schedule_among(kind, m, n, k, out_mode, scaled_tiles(kind));
}

struct Product {
    const int8_t *xq;
    const float *sx;
    int m;
    const nm_scaled_weight *w;
    void *out;
    int64_t ldo;
    int type;
    bool gated;
    int act;
    const void *x = nullptr;    // values in place of codes (few tokens)
    int64_t ldx = 0;
    int xtype = 0;
};

// Whether the kernel of few tokens makes the codes of these rows itself.
bool takes_values(const void *x, int64_t ldx, int m, int k) {
    return few_takes_values(m, k) && ldx % 8 == 0 && aligned(x, 16);
}

// Whether m rows of `wide_a` bytes every `step_a` from a and m of b share a byte.  Rows of
// one stride that lie side by side do not.
bool rows_meet(const void *a, int64_t step_a, int64_t wide_a, const void *b, int64_t step_b, int64_t wide_b, int m) {
    const int64_t off = (int64_t)((uintptr_t)b - (uintptr_t)a);
    if (off >= (m - 1) * step_a + wide_a || -off >= (m - 1) * step_b + wide_b) return false;
    const int64_t side = ((off % step_a) + step_a) % step_a;
    return step_a != step_b || side < wide_a || side + wide_b > step_a;
}

// ws: room for the expanded weight where there is one.
nm_status run_product(const Product &p, char *ws, void *stream) {
    const nm_desc &d = *p.w->desc;
    int kind = d.kind;
    const int8_t *vals = p.w->vals;
    const uint8_t *meta = p.w->meta;
    if (p.x || takes_few(kind, p.gated, p.m, d.n, d.k)) {
        BlockArgs a;
        fill_product(a, p.m, *p.w);
        a.X = p.xq;
        a.A = vals;
        a.meta = meta;
        a.row_scale = p.sx;
        a.x = p.x;
        a.ldx = p.ldx;
        a.xtype = p.xtype;
        a.kx = p.w->k;
        a.out = p.out;
        a.ldo = p.ldo;
        a.type = p.type;
        a.act = p.act;
        return launch_few(kind, p.gated, a, stream) == 0 ? NM_OK : NM_ERR_HIP;
    }
    if (expansion(d, p.m)) {
        int8_t *out = (int8_t *)ws;
        if (launch_expand(kind, vals, meta, d.n, d.k, out, stream) != 0) return NM_ERR_HIP;
        kind = expanded_kind(kind);
        vals = out;
        meta = kind == NM_KIND_SP42 ? (const uint8_t *)(out + (int64_t)d.n_frags * d.k_steps * kVBlock) : nullptr;
    }
    // the kernels address X with 32-bit byte offsets: a longer batch goes in parts
    const int64_t fits = ((((int64_t)1 << 32) - 1) / d.k) / 1280 * 1280;
    const int eb = type_bytes(p.type);
    for (int64_t row = 0; row < p.m; row += fits) {
        const int m = (int)(p.m - row < fits ? p.m - row : fits);
        BlockArgs a;
        fill_product(a, m, *p.w);
        a.X = p.xq + row * d.k;
        a.A = vals;
        a.meta = meta;
        a.row_scale = p.sx + row;
        a.out = (char *)p.out + row * p.ldo * eb;
        a.ldo = p.ldo;
        a.type = p.type;
        a.act = p.act;
        a.stream_out = aligned(p.out, 128) ? stream_out_for(m, (int)(p.ldo < (1 << 30) ? p.ldo : 1), d.k) : 0;
        const int tile = product_tile(kind, p.gated, m, d.n, d.k, out_mode_for(p.type, p.gated));
        const int grid = place_tiles(a, tile);
        const int err = p.gated ? launch_gated(kind, tile, a, grid, stream) : launch_scaled(kind, tile, a, grid, stream);
        if (err != 0) return NM_ERR_HIP;
    }
    return NM_OK;
}

nm_status check_product(int m, const nm_scaled_weight *w, bool gated, int act, const void *out, int64_t ldo, int type) {
    if (m < 0 || m >= kMaxRows) return NM_ERR_SHAPE;
    nm_status st = check_weight(w, gated);
    if (st != NM_OK) return st;
    if (!valid_type(type) || (gated && (act < NM_ACT_SILU || act > NM_ACT_SIGMOID))) return NM_ERR_ARG;
    if (ldo < w->n) return NM_ERR_SHAPE;
    if (m > 0 && (!out || !aligned(out, type_bytes(type)))) return NM_ERR_ARG;
    return NM_OK;
}

nm_status product_of_codes(const int8_t *xq, const float *sx, int m, const nm_scaled_weight *w, bool gated, int act,
                           void *out, int64_t ldo, int type, void *ws, size_t ws_bytes, void *stream) {
    nm_status st = check_product(m, w, gated, act, out, ldo, type);
    if (st != NM_OK || m == 0) return st;
    if (!xq || !sx || !aligned(xq, 16) || !aligned(sx, 4)) return NM_ERR_ARG;
    const size_t need = (size_t)expansion(*w->desc, m);
    if (need && (!ws || ws_bytes < need || !aligned(ws, 256))) return NM_ERR_WORKSPACE;
    return run_product({xq, sx, m, w, out, ldo, type, gated, act}, (char *)ws, stream);
}

nm_status product_of_rows(const void *x, int64_t ldx, int xtype, int m, const nm_scaled_weight *w, bool gated, int act,
                          void *out, int64_t ldo, int type, void *ws, size_t ws_bytes, void *stream) {
    nm_status st = check_product(m, w, gated, act, out, ldo, type);
    if (st != NM_OK) return st;
    if (!valid_type(xtype)) return NM_ERR_ARG;
    if (ldx < w->k) return NM_ERR_SHAPE;
    if (m == 0) return NM_OK;
    if (!x || !aligned(x, type_bytes(xtype))) return NM_ERR_ARG;
    // (a workgroup of that kernel reads x while others have written their outputs: where the two share
    // memory the codes are made first)
    const int xb = type_bytes(xtype), ob = type_bytes(type);
    if (takes_values(x, ldx, m, w->k) &&
        !rows_meet(x, ldx * xb, (int64_t)w->k * xb, out, ldo * ob, (int64_t)w->n * ob, m)) {
        Product p = {nullptr, nullptr, m, w, out, ldo, type, gated, act};
        p.x = x;
        p.ldx = ldx;
        p.xtype = xtype;
        return run_product(p, nullptr, stream);
    }
    const nm_desc &d = *w->desc;
    const size_t codes = codes_bytes(m, d.k), need = codes + (size_t)expansion(d, m);
    if (!ws || ws_bytes < need || !aligned(ws, 256)) return NM_ERR_WORKSPACE;
    int8_t *xq = (int8_t *)ws;
    float *sx = (float *)((char *)ws + round256((size_t)m * d.k));
    st = nm_quantize_rows(x, ldx, xtype, m, w->k, xq, sx, stream);
    if (st != NM_OK) return st;
    return run_product({xq, sx, m, w, out, ldo, type, gated, act}, (char *)ws + codes, stream);
}

// ---------------------------------------------------------------- gated backward

// A product of 16-bit operands, [m x n] outputs over k_bytes of each row: the
// tile and split of the reduction with the least estimated time (us).  The estimate
// is linear in ten terms, among them rounds of one workgroup and of as many as a
// unit holds, fitted per tile (non-negative least squares on relative errors, near-best
// rows weighted most) to timings of every (tile, split) on 191 shapes, m 64..20000, n to
// 4096, 128..20000 values of k.  Fitted to 108 of them, its choice on the other 83 took 1.7 %
// longer than the best on average, for one in ten 3.7 % or more, 39 % at most.
struct CastCost {
    int tile, per_cu;
    float launch, chain, round_steps, mean_steps, full_steps, rounds, out_mb, x_mb, split, part_mb;
};
constexpr CastCost kCastCost[] = {
    {1, 3, 2.8f, 0.117f, 0.0f, 0.21f, 0.217f, 0.639f, 0.0f, 0.0f, 4.94f, 0.942f},
    {3, 5, 2.68f, 0.147f, 0.0f, 0.141f, 0.118f, 0.412f, 0.0f, 0.0f, 2.78f, 1.45f},
    {4, 1, 1.84f, 0.0f, 0.0f, 0.429f, 1.03f, 5.61f, 0.0427f, 0.00878f, 15.6f, 0.367f},
    {6, 2, 1.88f, 0.0405f, 0.0f, 0.258f, 0.395f, 1.66f, 0.0f, 0.000901f, 5.12f, 0.67f},
    {12, 1, 0.92f, 0.0f, 0.812f, 0.189f, 0.0f, 4.91f, 0.043f, 0.00755f, 11.2f, 0.38f},
};
// The best split of a product on one tile, and its estimate.
struct CastChoice {
    int split = 1;
    float us = 0.f;
};
CastChoice cast_choice(const CastCost &c, int64_t m, int64_t n, int64_t k_bytes) {
    const int64_t k_steps = k_bytes / kKStep, cus = device_cu_count();
    const float out_mb = (float)(m * n) * 2e-6f, x_mb = (float)(m * k_bytes) * 1e-6f;
    const TileCfg &t = kTiles[c.tile];
    const int64_t tiles = ((m + t.tile_m() - 1) / t.tile_m()) * ((n + t.tile_n() - 1) / t.tile_n());
    CastChoice best;
    for (int s = 1; s <= 8; s *= 2) {
        if (s > 1 && (k_steps / s < 4 || tiles > kMaxSplitTiles || s * m * n * 4 >= ((int64_t)1 << 31))) break;
        const float steps = (float)k_steps / (float)s, mean = (float)(tiles * s) / (float)cus;
        const float rounds = (float)((tiles * s + cus - 1) / cus);
        const float full = (float)((tiles * s + c.per_cu * cus - 1) / (c.per_cu * cus));
        float us = c.launch + steps * (c.chain + c.round_steps * rounds + c.mean_steps * mean + c.full_steps * full) +
                   c.rounds * rounds + c.out_mb * out_mb + c.x_mb * x_mb;
        if (s > 1) us += c.split + c.part_mb * 2.f * (float)s * out_mb;
        if (s == 1 || us < best.us) {
            best.us = us;
            best.split = s;
        }
    }
    return best;
}
// Pieces of the workspace, in their order.
struct GradPlan {
    int64_t rows_w, cols, ldt;     // 2 n', k rounded up to 16, tokens rounded up to 64
    int grad_tile, parts_rows, cast_tile = 0, dx_split = 1, dw_split = 1;
    size_t at_da, at_dat, at_xt, at_wt, at_parts, at_dx_split, at_dw_split, bytes;

    GradPlan(const nm_scaled_weight &w, int m)
        : rows_w(w.desc->n), cols(w.desc->k), ldt((int64_t)(m + 63) / 64 * 64) {
        grad_tile = schedule_among(NM_KIND_DENSE, m, w.desc->n, w.desc->k, NM_OUT_I32, kGradTiles);
        const TileCfg &g = kTiles[grad_tile];
        parts_rows = (m + g.tile_m() - 1) / g.tile_m() * g.wm;
        // dx and the weights' gradients run in one launch, on the tile that is best for both
        float least = 0.f;
        for (const CastCost &c : kCastCost) {
            const CastChoice dx = cast_choice(c, m, cols, 2 * rows_w), dw = cast_choice(c, rows_w, cols, 2 * ldt);
            if (cast_tile == 0 || dx.us + dw.us < least) {
                least = dx.us + dw.us;
                cast_tile = c.tile;
                dx_split = dx.split;
                dw_split = dw.split;
            }
        }
        size_t at = 0;
        auto take = [&](int64_t n) {
            const size_t here = at;
            at += round256((size_t)n);
            return here;
        };
        at_da = take((int64_t)m * rows_w * 2);
        at_dat = take(rows_w * ldt * 2);
        at_xt = take(cols * ldt * 2);
        at_wt = take(cols * rows_w * 2);
        at_parts = take((int64_t)parts_rows * rows_w * 4);
        // (split products: counters, then partial sums; the two counter blocks lie one after the other)
        at_dx_split = take(2 * kCounterBytes + (dx_split > 1 ? dx_split * (int64_t)m * cols * 4 : 0));
        at_dw_split = take(dw_split > 1 ? dw_split * rows_w * cols * 4 : 0);
        bytes = at;
    }
};

nm_status check_grad(const nm_scaled_weight *w, int m) {
    nm_status st = check_weight(w, true);
    if (st != NM_OK) return st;
    if (w->desc->layout != NM_LAYOUT_DENSE) return NM_ERR_UNSUPPORTED;
    if (m < 0 || m >= kMaxRows) return NM_ERR_SHAPE;
    const int64_t tokens = ((int64_t)m + 63) / 64 * 64, wide = w->desc->n > w->desc->k ? w->desc->n : w->desc->k;
    if (tokens * ((wide + 63) / 64 * 64) >= ((int64_t)1 << 31)) return NM_ERR_SHAPE;
    if ((int64_t)w->desc->n * w->desc->k >= ((int64_t)1 << 29)) return NM_ERR_SHAPE;
    return NM_OK;
}

}  // namespace

extern "C" nm_status nm_linear_workspace(const nm_scaled_weight *w, int m, int xtype, size_t *bytes) {
    if (!bytes || !w || (xtype != 0 && !valid_type(xtype))) return NM_ERR_ARG;
    nm_status st = check_desc(w->desc);
    if (st != NM_OK) return st;
    if (m < 0 || m >= kMaxRows) return NM_ERR_SHAPE;
    *bytes = m == 0 ? 0 : (xtype ? codes_bytes(m, w->desc->k) : 0) + (size_t)expansion(*w->desc, m);
    return NM_OK;
}

extern "C" nm_status nm_gemm_i8_scaled(const int8_t *xq, const float *sx, int m, const nm_scaled_weight *w, void *y,
                                       int64_t ldy, int type, void *ws, size_t ws_bytes, void *stream) {
    return product_of_codes(xq, sx, m, w, false, 0, y, ldy, type, ws, ws_bytes, stream);
}

extern "C" nm_status nm_linear_i8(const void *x, int64_t ldx, int xtype, int m, const nm_scaled_weight *w, void *y,
                                  int64_t ldy, int type, void *ws, size_t ws_bytes, void *stream) {
    return product_of_rows(x, ldx, xtype, m, w, false, 0, y, ldy, type, ws, ws_bytes, stream);
}

extern "C" nm_status nm_gated_i8(const int8_t *xq, const float *sx, int m, const nm_scaled_weight *w, int act, void *h,
                                 int64_t ldh, int type, void *ws, size_t ws_bytes, void *stream) {
    return product_of_codes(xq, sx, m, w, true, act, h, ldh, type, ws, ws_bytes, stream);
}

extern "C" nm_status nm_gated(const void *x, int64_t ldx, int xtype, int m, const nm_scaled_weight *w, int act, void *h,
                              int64_t ldh, int type, void *ws, size_t ws_bytes, void *stream) {
    return product_of_rows(x, ldx, xtype, m, w, true, act, h, ldh, type, ws, ws_bytes, stream);
}

extern "C" nm_status nm_gated_backward_workspace(const nm_scaled_weight *w, int m, size_t *bytes) {
    if (!bytes) return NM_ERR_ARG;
    nm_status st = check_grad(w, m);
    if (st != NM_OK) return st;
    *bytes = m == 0 ? 0 : GradPlan(*w, m).bytes;
    return NM_OK;
}

extern "C" nm_status nm_gated_backward(const nm_gated_grad_args *args, const nm_scaled_weight *w, void *ws,
                                       size_t ws_bytes, void *stream) {
    if (!args) return NM_ERR_ARG;
    const nm_gated_grad_args &g = *args;
    nm_status st = check_grad(w, g.m);
    if (st != NM_OK) return st;
    if ((g.type != NM_TYPE_F16 && g.type != NM_TYPE_BF16) || g.act < NM_ACT_SILU || g.act > NM_ACT_SIGMOID)
        return NM_ERR_ARG;
    for (const void *p : {(const void *)g.dx, (const void *)g.dw_gate, (const void *)g.dw_up})
        if (!aligned(p, 2)) return NM_ERR_ARG;
    if (!aligned(g.dbias_gate, 4) || !aligned(g.dbias_up, 4)) return NM_ERR_ARG;
    if ((!g.dw_gate) != (!g.dw_up)) return NM_ERR_ARG;
    const nm_desc &d = *w->desc;
    if (g.m == 0) {
        const size_t each = (size_t)w->n * w->k * 2;
        if ((g.dw_gate && (launch_zero(g.dw_gate, each, stream) != 0 || launch_zero(g.dw_up, each, stream) != 0)) ||
            (g.dbias_gate && launch_zero(g.dbias_gate, (size_t)w->n * 4, stream) != 0) ||
            (g.dbias_up && launch_zero(g.dbias_up, (size_t)w->n * 4, stream) != 0))
            return NM_ERR_HIP;
        return NM_OK;
    }
    if (g.lddh < w->n) return NM_ERR_SHAPE;
    if (!g.xq || !g.sx || !g.dh || !aligned(g.xq, 16) || !aligned(g.sx, 4) || !aligned(g.dh, 2)) return NM_ERR_ARG;
    const GradPlan p(*w, g.m);
    if (!ws || ws_bytes < p.bytes || !aligned(ws, 256)) return NM_ERR_WORKSPACE;
    char *base = (char *)ws;

    // dg and du
    BlockArgs a;
    fill_product(a, g.m, *w);
    a.X = g.xq;
    a.A = w->vals;
    a.meta = nullptr;
    a.row_scale = g.sx;
    a.type = g.type;
    a.act = g.act;
    a.dh = g.dh;
    a.lddh = g.lddh;
    a.da = base + p.at_da;
    a.dat = base + p.at_dat;
    a.ldt = p.ldt;
    a.bias_parts = g.dbias_gate || g.dbias_up ? (float *)(base + p.at_parts) : nullptr;
    int grid = place_tiles(a, p.grad_tile);
    if (launch_gated_grad(p.grad_tile, a, grid, stream) != 0) return NM_ERR_HIP;
    if (a.bias_parts && launch_bias_sums(a.bias_parts, p.parts_rows, d.n, w->n, g.dbias_gate, g.dbias_up, stream) != 0)
        return NM_ERR_HIP;

    if (!g.dx && !g.dw_gate) return NM_OK;
    const TransposeArgs wt = {w->vals, w->scale, base + p.at_wt, d.k, p.rows_w, g.dx ? d.n : 0, d.k};
    const TransposeArgs xt = {g.xq, g.sx, base + p.at_xt, d.k, p.ldt, g.dw_gate ? g.m : 0, d.k};
    int *counters = (int *)(base + p.at_dx_split);
    if (launch_transpose_codes(g.type, wt, xt, p.dx_split > 1 || p.dw_split > 1 ? counters : nullptr,
                               (int)(2 * kCounterBytes / 4), stream) != 0)
        return NM_ERR_HIP;
    CastPair pair;
    for (BlockArgs &c : pair.part) {
        fill_product(c, g.m, *w);
        c.scale = nullptr;
        c.qscale = nullptr;
        c.meta = nullptr;
        c.n = d.k;
        c.n_out = w->k;
        c.ldo = w->k;
        c.n_frags = (d.k + kFragRows - 1) / kFragRows;
        c.gemm_grid = 0;
    }
    // the weights' gradients first: their reductions are the longer ones where the device is hard to fill
    if (g.dw_gate) {
        BlockArgs &c = pair.part[0];
        c.X = (const int8_t *)(base + p.at_dat);
        c.A = (const int8_t *)(base + p.at_xt);
        c.m = d.n;
        c.k = (int)(2 * p.ldt);
        c.k_steps = c.k / kKStep;
        c.out = g.dw_gate;
        c.out2 = g.dw_up;
        c.interleaved = w->n;
        c.split_k = p.dw_split;
        c.counters = counters + kCounterBytes / 4;
        c.partials = (int32_t *)(base + p.at_dw_split);
        c.stream_out = 0;
        place_tiles(c, p.cast_tile);
    }
    if (g.dx) {
        BlockArgs &c = pair.part[1];
        c.X = (const int8_t *)(base + p.at_da);
        c.A = (const int8_t *)(base + p.at_wt);
        c.k = (int)(2 * p.rows_w);
        c.k_steps = c.k / kKStep;
        c.out = g.dx;
        c.split_k = p.dx_split;
        c.counters = counters;
        c.partials = (int32_t *)(base + p.at_dx_split + 2 * kCounterBytes);
        c.stream_out = aligned(g.dx, 128) ? stream_out_for(g.m, w->k, c.k) : 0;
        place_tiles(c, p.cast_tile);
    }
    if (launch_cast(g.type, p.cast_tile, pair, stream) != 0) return NM_ERR_HIP;
    return NM_OK;
}
