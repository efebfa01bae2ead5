// C entry points of rotary positions and differential attention: argument checks,
// workspaces and dispatch (host only).
#include <cmath>

#include "nmspmm_attn_internal.h"

using namespace nmspmm;

namespace {

bool aligned(const void *p, int to) { return ((uintptr_t)p & (uintptr_t)(to - 1)) == 0; }
size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

// Whether heads of `width` 16-bit values are whole 16-byte pieces at their boundaries.
bool pieces(const nm_heads &t, int width) {
    return aligned(t.p, 16) && t.token % 8 == 0 && t.head % 8 == 0 && t.batch % 8 == 0 && width % 8 == 0;
}

// A tensor with strides that do not matter, along dimensions of one, put out of the way.
nm_heads extent(nm_heads t, const nm_tokens &tokens, bool keys, int heads, int width) {
    const int64_t n = keys ? (tokens.k_offsets ? tokens.total_k : tokens.tk) : tokens.q_offsets ? tokens.total_q : tokens.tq;
    if (tokens.batch <= 1 || tokens.q_offsets) t.batch = 0;
    if (n <= 1) t.token = (width + 7) & ~7;
    if (heads <= 1) t.head = 0;
    return t;
}

nm_status check_tokens(const nm_tokens &t) {
    if (t.batch < 0 || t.tq < 0 || t.tk < 0 || t.batch >= (1 << 24) || t.tq >= kMaxAttnTokens ||
        t.tk >= kMaxAttnTokens)
        return NM_ERR_SHAPE;
    if (!t.q_offsets != !t.k_offsets) return NM_ERR_ARG;
    if (t.q_offsets) {
        if (t.q_lens || t.k_lens) return NM_ERR_ARG;
        if (t.total_q < 0 || t.total_k < 0 || t.total_q >= (1ll << 31) || t.total_k >= (1ll << 31)) return NM_ERR_SHAPE;
    }
    for (const int32_t *p : {t.q_offsets, t.k_offsets, t.q_lens, t.k_lens})
        if (!aligned(p, 4)) return NM_ERR_ARG;
    return NM_OK;
}

nm_status check_heads(int type, int H, int Hk, int d, int dv, float scale) {
    if (type != NM_TYPE_F16 && type != NM_TYPE_BF16) return NM_ERR_ARG;
    if (H < 1 || Hk < 1 || H % Hk != 0 || H >= (1 << 16) || d < 1 || d > kMaxHeadWidth || dv < 1 || dv > kMaxValueWidth)
        return NM_ERR_SHAPE;
    return scale > 0.f && std::isfinite(scale) ? NM_OK : NM_ERR_ARG;
}

nm_status check_weight(const nm_diff_weight &w) {
    if (w.value) return aligned(w.value, 4) ? NM_OK : NM_ERR_ARG;
    if (w.n < 1 || w.n >= (1 << 20)) return NM_ERR_SHAPE;
    for (const float *p : {w.q1, w.k1, w.q2, w.k2})
        if (!p || !aligned(p, 4)) return NM_ERR_ARG;
    return NM_OK;
}

// A tensor's strides; its pointer where it has rows.
nm_status check_tensor(const nm_heads &t, bool rows) {
    if (t.token < 0 || t.head < 0 || t.batch < 0 || t.token >= kMaxTokenStride) return NM_ERR_SHAPE;
    return (!rows || t.p) && aligned(t.p, 2) ? NM_OK : NM_ERR_ARG;
}

Heads heads_of(const nm_heads &t) { return {(char *)t.p, t.batch, t.token, t.head}; }

int64_t rows_of(const nm_tokens &t) { return t.q_offsets ? t.total_q : (int64_t)t.batch * t.tq; }
int64_t keys_of(const nm_tokens &t) { return t.k_offsets ? t.total_k : (int64_t)t.batch * t.tk; }

void fill(AttnArgs &a, const nm_tokens &t, const nm_diff_weight &w, int H, int Hk, int d, int dv, float scale) {
    a = AttnArgs{};
    a.q_offsets = t.q_offsets;
    a.k_offsets = t.k_offsets;
    a.q_lens = t.q_lens;
    a.k_lens = t.k_lens;
    a.total_q = t.total_q;
    a.total_k = t.total_k;
    a.rows = rows_of(t);
    a.batch = t.batch;
    a.tq = t.tq;
    a.tk = t.tk;
    a.H = H;
    a.Hk = Hk;
    a.group = H / Hk;
    a.d = d;
    a.dv = dv;
    // no bound is one that no pair of positions reaches; larger ones say the same
    const int most = 1 << 29;
    a.left = t.left < 0 || t.left > most ? most : t.left;
    a.right = t.right < 0 || t.right > most ? most : t.right;
    a.scale = scale;
    a.stat_rows = stat_rows_of(dv);
    a.scale2 = scale * 1.4426950408889634f;
    a.weight = w;
}

// How the forward pass is cut: workgroups of many rows that share their tiles of keys, or of few rows, whose
// keys go to the runs of a workgroup and in `splits` parts to several, which a second kernel joins.
//   Few rows: up to 64, and more where workgroups of many would leave too much of the device without work (468 shapes of 65 to
//   1024 causal rows over 256 to 8192 keys; the rule is within 1 % of the better variant on average).  Many and few:
//     32 + 64:   4 x 512 rows of 8 heads over 1024 keys (128 workgroups of many) 27.5 and 22.5 us, 4 x 1024 (256) 27 and 36
//     64 + 128:  4 x 200 over 2048 (64) 62 and 44, 4 x 512 over 1024 (128) 34 and 44
//     128 + 256: 4 x 256 over 512 (128) 23 and 41, over 8192 238 and 208, 4 x 512 over 8192 (256) 246 and 335
//   Splits: a workgroup a compute unit, of four tiles a wave at least (1 row of 8 heads over 577 keys
//   in one 14.3 us, in three and a second kernel 13.3; over 8192 in eight 20.0).  Sequences of unequal length: twice as
//   many where those are few and long (16 x 1 rows over up to 16384 keys, 4 key heads, 69 to 61 us; 8 over 32768, 8
//   key heads, 162 to 129; 4 over 16384 would go 31 to 34 us, 64 over 4096 67 to 71).
struct Cut {
    bool wide;
    int row_tiles, splits;
};
Cut cut_of(const nm_tokens &t, int H, int Hk, int cls) {
    const int64_t rows = (int64_t)t.tq * (H / Hk), heads = (int64_t)t.batch * Hk;
    const int cus = device_cu_count();
    const int64_t wide_groups = heads * ((rows + wide_rows(cls) - 1) / wide_rows(cls));
    Cut c;
    c.wide = rows > 64 && (cls == 0   ? 4 * wide_groups >= 3 * cus
                           : cls == 1 ? 8 * wide_groups >= 3 * cus
                                      : wide_groups >= cus || 16 * wide_groups >= t.tk);
    const int tile = c.wide ? wide_rows(cls) : kFewRows;
    c.row_tiles = (int)((rows + tile - 1) / tile);
    c.splits = 1;
    if (!c.wide) {
        const int64_t groups = heads * c.row_tiles, key_tiles = (t.tk + kFewRowsKeys - 1) / kFewRowsKeys;
        int64_t splits = groups ? (cls >= 2 ? 2 : 1) * cus / groups : 1;
        if ((t.k_lens || t.k_offsets) && 4 * groups <= cus && key_tiles >= 128 * splits) splits *= 2;
        const int64_t most = key_tiles / (4 * key_runs(cls));
        if (splits > most) splits = most;
        if (splits > kMaxSplits) splits = kMaxSplits;
        c.splits = splits > 1 ? (int)splits : 1;
    }
    return c;
}
size_t parts_bytes(const nm_tokens &t, int H, int dv, int splits) {
    return splits > 1 ? (size_t)t.batch * H * t.tq * splits * (2 * dv + 4) * 4 : 0;
}
bool grid_fits(int64_t n) { return n < (1ll << 24); }   // a launch's threads are counted in 32 bits

}  // namespace

// ---------------------------------------------------------------- rotary positions

extern "C" nm_status nm_rotary(const nm_rotary_args *args, void *stream) {
    if (!args) return NM_ERR_ARG;
    const nm_rotary_args &g = *args;
    if (g.type < NM_TYPE_F16 || g.type > NM_TYPE_F32) return NM_ERR_ARG;
    if (g.tokens < 0 || g.tokens >= (1ll << 31) || g.pairs < 1 || g.d < 2 * (int64_t)g.pairs || g.d > kMaxRotaryWidth ||
        g.axes < 1 || g.ld_pos < 0)
        return NM_ERR_SHAPE;
    const int eb = g.type == NM_TYPE_F32 ? 4 : 2;
    int64_t heads = 0;
    for (const nm_rotary_part &p : g.part) {
        if (p.heads < 0 || p.x_token < 0 || p.x_head < 0 || p.out_token < 0 || p.out_head < 0) return NM_ERR_SHAPE;
        heads += p.heads;
        if (p.heads == 0 || g.tokens == 0) continue;
        if (!p.x || !p.out || !aligned(p.x, eb) || !aligned(p.out, eb)) return NM_ERR_ARG;
    }
    if (heads >= (1 << 16)) return NM_ERR_SHAPE;
    if (heads == 0) return NM_ERR_ARG;
    if (g.tokens == 0) return NM_OK;
    if (!g.pos || !g.freq || !g.axis || !aligned(g.pos, 4) || !aligned(g.freq, 8) || !aligned(g.axis, 4))
        return NM_ERR_ARG;
    RotaryArgs a;
    for (int i = 0; i < 2; ++i) {
        const nm_rotary_part &p = g.part[i];
        a.part[i] = {p.x, p.out, p.x_token, p.x_head, p.out_token, p.out_head, p.heads};
    }
    a.pos = g.pos;
    a.ld_pos = g.ld_pos;
    a.freq = g.freq;
    a.axis = g.axis;
    a.tokens = g.tokens;
    a.pos_float = g.pos_float != 0;
    a.pairs = g.pairs;
    a.d = g.d;
    a.interleaved = g.interleaved != 0;
    a.axes = g.axes;
    a.sign = g.back ? -1.f : 1.f;
    return launch_rotary(g.type, a, stream) == 0 ? NM_OK : NM_ERR_HIP;
}

// ---------------------------------------------------------------- differential attention

static nm_status check_forward(const nm_diff_args *args) {
    if (!args) return NM_ERR_ARG;
    const nm_diff_args &g = *args;
    nm_status st = check_heads(g.type, g.H, g.Hk, g.d, g.dv, g.scale);
    if (st == NM_OK) st = check_tokens(g.tokens);
    return st;
}

extern "C" nm_status nm_diff_attention_workspace(const nm_diff_args *args, size_t *bytes) {
    if (!bytes) return NM_ERR_ARG;
    const nm_status st = check_forward(args);
    if (st != NM_OK) return st;
    const Cut c = cut_of(args->tokens, args->H, args->Hk, width_class(args->d, args->dv));
    *bytes = parts_bytes(args->tokens, args->H, args->dv, c.splits);
    return NM_OK;
}

extern "C" nm_status nm_diff_attention(const nm_diff_args *args, void *ws, size_t ws_bytes, void *stream) {
    nm_status st = check_forward(args);
    if (st == NM_OK) st = check_weight(args->weight);
    if (st != NM_OK) return st;
    const nm_diff_args &g = *args;
    const int64_t rows = rows_of(g.tokens), keys = keys_of(g.tokens);
    const nm_heads q = extent(g.q, g.tokens, false, 2 * g.H, g.d), k = extent(g.k, g.tokens, true, 2 * g.Hk, g.d),
                   v = extent(g.v, g.tokens, true, g.Hk, g.dv), o = extent(g.o, g.tokens, false, g.H, g.dv);
    for (const nm_heads *t : {&q, &k, &v, &o})
        if ((st = check_tensor(*t, (t == &k || t == &v ? keys : rows) > 0)) != NM_OK) return st;
    if (!aligned(g.kept, 16) || !aligned(g.stats, 4) || !g.kept != !g.stats) return NM_ERR_ARG;
    if (rows == 0 || g.tokens.batch == 0 || g.tokens.tq == 0) return NM_OK;
    const Cut c = cut_of(g.tokens, g.H, g.Hk, width_class(g.d, g.dv));
    const size_t need = parts_bytes(g.tokens, g.H, g.dv, c.splits);
    if (need && (!ws || ws_bytes < need || !aligned(ws, 16))) return NM_ERR_WORKSPACE;
    AttnArgs a;
    fill(a, g.tokens, g.weight, g.H, g.Hk, g.d, g.dv, g.scale);
    if (!grid_fits((int64_t)a.batch * a.Hk * c.row_tiles * c.splits) || (int64_t)a.tq * a.group >= (1ll << 31) ||
        (c.splits > 1 && !grid_fits((int64_t)a.batch * a.H * a.tq)))
        return NM_ERR_SHAPE;
    a.q = heads_of(q);
    a.k = heads_of(k);
    a.v = heads_of(v);
    a.o = heads_of(o);
    a.kept = g.kept;
    a.stats = g.stats;
    a.pieces = pieces(q, g.d) && pieces(k, g.d) && pieces(v, g.dv);
    a.row_tiles = c.row_tiles;
    a.splits = c.splits;
    a.parts = (float *)ws;
    if (launch_diff_forward(g.type, width_class(g.d, g.dv), c.wide, a, stream) != 0) return NM_ERR_HIP;
    if (c.splits > 1 && launch_diff_join(g.type, a, stream) != 0) return NM_ERR_HIP;
    return NM_OK;
}

static nm_status check_backward(const nm_diff_grad_args *args) {
    if (!args) return NM_ERR_ARG;
    const nm_diff_grad_args &g = *args;
    nm_status st = check_heads(g.type, g.H, g.Hk, g.d, g.dv_width, g.scale);
    if (st == NM_OK) st = check_tokens(g.tokens);
    return st;
}
static int64_t grad_row_tiles(const nm_diff_grad_args &g) {
    return ((int64_t)g.tokens.tq * (g.H / g.Hk) + kGradRows - 1) / kGradRows;
}
// Parts of the rows for the gradients of the keys: up to two workgroups for each compute unit where the tiles of keys make
// fewer, of at least four steps of 32 rows on average.  A compute unit holds one at a time in every class (LDS of 135 KB at
// 64 + 128, 86 at 128 + 128, 136 at 128 + 256; at 32 + 64 the registers of eight waves), so beyond one for each the parts
// only even out unequal tiles, against sums in memory and their join.  Backward passes in one, two and four parts,
// * the rule's:
//   2 x 4096 rows of 8 heads, 4 key heads, 64 + 128, causal 419, 374*, 375 us; without a mask 513, 541*, 568
//   2 x 2048 rows of 4 heads, 64 + 128, causal 139, 122, 128*; without a mask 140, 128, 142*
//   the same, 128 + 256, causal 240, 230*, 238; without a mask 243, 271*, 296
static int key_splits(const nm_diff_grad_args &g) {
    const int64_t tiles = ((int64_t)g.tokens.tk + kGradKeys - 1) / kGradKeys;
    const int64_t groups = (int64_t)g.tokens.batch * g.Hk * tiles * (width_class(g.d, g.dv_width) == 3 ? 2 : 1);
    const int64_t steps = ((int64_t)g.tokens.tq + 31) / 32 * (g.H / g.Hk);
    if (groups == 0) return 1;
    int64_t splits = 2 * device_cu_count() / groups;
    if (splits > steps / 4) splits = steps / 4;
    return splits < 2 ? 1 : splits > 64 ? 64 : (int)splits;
}
static size_t key_parts_bytes(const nm_diff_grad_args &g) {
    const int splits = key_splits(g);
    return splits > 1 ? round256((size_t)g.tokens.batch * g.Hk * splits * g.tokens.tk * (2 * g.d + g.dv_width) * 4) : 0;
}
static size_t delta_bytes(const nm_diff_grad_args &g) { return round256((size_t)2 * g.H * rows_of(g.tokens) * 4); }
static size_t dlam_bytes(const nm_diff_grad_args &g) { return (size_t)g.H * g.tokens.batch * grad_row_tiles(g) * 16; }
static int64_t grad_key_tiles(const nm_diff_grad_args &g) { return ((int64_t)g.tokens.tk + kGradKeys - 1) / kGradKeys; }
static size_t norms_bytes(const nm_diff_grad_args &g) { return (size_t)g.Hk * g.tokens.batch * grad_key_tiles(g) * 4; }
static size_t tops_bytes(const nm_diff_grad_args &g) { return (size_t)g.Hk * g.tokens.batch * grad_row_tiles(g) * 16; }

extern "C" nm_status nm_diff_attention_backward_workspace(const nm_diff_grad_args *args, size_t *bytes) {
    if (!bytes) return NM_ERR_ARG;
    const nm_status st = check_backward(args);
    if (st != NM_OK) return st;
    *bytes = delta_bytes(*args) + key_parts_bytes(*args) + dlam_bytes(*args) + tops_bytes(*args) +
             norms_bytes(*args);
    return NM_OK;
}

extern "C" nm_status nm_diff_attention_backward(const nm_diff_grad_args *args, void *ws, size_t ws_bytes,
                                                void *stream) {
    nm_status st = check_backward(args);
    if (st == NM_OK) st = check_weight(args->weight);
    if (st != NM_OK) return st;
    const nm_diff_grad_args &g = *args;
    const int64_t rows = rows_of(g.tokens), keys = keys_of(g.tokens);
    const nm_heads q = extent(g.q, g.tokens, false, 2 * g.H, g.d), dq = extent(g.dq, g.tokens, false, 2 * g.H, g.d),
                   grad_o = extent(g.grad_o, g.tokens, false, g.H, g.dv_width),
                   k = extent(g.k, g.tokens, true, 2 * g.Hk, g.d), dk = extent(g.dk, g.tokens, true, 2 * g.Hk, g.d),
                   v = extent(g.v, g.tokens, true, g.Hk, g.dv_width), dv = extent(g.dv, g.tokens, true, g.Hk, g.dv_width);
    for (const nm_heads *t : {&q, &grad_o, &dq})
        if ((st = check_tensor(*t, rows > 0)) != NM_OK) return st;
    for (const nm_heads *t : {&k, &v, &dk, &dv})
        if ((st = check_tensor(*t, keys > 0)) != NM_OK) return st;
    if (!g.dlam || !aligned(g.dlam, 4) || !aligned(g.kept, 16) || !aligned(g.stats, 4) ||
        (rows > 0 && (!g.kept || !g.stats)))
        return NM_ERR_ARG;
    if (!g.weight.value)
        for (const float *p : {g.dq1, g.dk1, g.dq2, g.dk2})
            if (!p || !aligned(p, 4)) return NM_ERR_ARG;
    size_t need = 0;
    st = nm_diff_attention_backward_workspace(args, &need);
    if (st != NM_OK) return st;
    if (need && (!ws || ws_bytes < need || !aligned(ws, 16))) return NM_ERR_WORKSPACE;
    AttnArgs a;
    fill(a, g.tokens, g.weight, g.H, g.Hk, g.d, g.dv_width, g.scale);
    const int64_t row_tiles = grad_row_tiles(g), key_tiles = grad_key_tiles(g);
    const int splits = key_splits(g);
    if (!grid_fits((int64_t)a.batch * a.Hk * row_tiles) || (int64_t)a.tq * a.group >= (1ll << 31) ||
        !grid_fits((int64_t)a.batch * a.Hk * key_tiles * splits * 2 + 1) ||
        (int64_t)a.batch * row_tiles * 4 >= (1ll << 31))
        return NM_ERR_SHAPE;
    a.q = heads_of(q);
    a.k = heads_of(k);
    a.v = heads_of(v);
    a.grad = heads_of(grad_o);
    a.dq = heads_of(dq);
    a.dk = heads_of(dk);
    a.dv_ = heads_of(dv);
    a.kept = (int16_t *)g.kept;
    a.stats = (float *)g.stats;
    a.pieces = pieces(q, g.d) && pieces(k, g.d) && pieces(v, g.dv_width) && pieces(grad_o, g.dv_width);
    a.row_tiles = (int)row_tiles;
    a.key_tiles = (int)key_tiles;
    a.delta = (float *)ws;
    a.key_splits = splits;
    a.key_parts = (float *)((char *)ws + delta_bytes(g));
    a.dlam_parts = (float *)((char *)ws + delta_bytes(g) + key_parts_bytes(g));
    a.dlam_count = (int)((int64_t)a.batch * row_tiles * 4);
    a.tops = (float *)((char *)a.dlam_parts + dlam_bytes(g));
    a.norms = (float *)((char *)a.tops + tops_bytes(g));
    a.dlam = g.dlam;
    a.dq1 = g.dq1;
    a.dk1 = g.dk1;
    a.dq2 = g.dq2;
    a.dk2 = g.dk2;
    const int cls = width_class(g.d, g.dv_width);
    if (g.type == NM_TYPE_F16 && a.batch > 0 && row_tiles > 0 && key_tiles > 0 && launch_diff_norms(a, stream) != 0)
        return NM_ERR_HIP;
    if (a.batch > 0 && row_tiles > 0 && launch_diff_grad_q(g.type, cls, a, stream) != 0) return NM_ERR_HIP;
    if (launch_diff_grad_k(g.type, cls, a, stream) != 0) return NM_ERR_HIP;
    return a.key_splits == 1 || launch_diff_join_keys(g.type, a, stream) == 0 ? NM_OK : NM_ERR_HIP;
}
