// The host code of differential attention with its launches replaced by checks of their arguments: reads shapes from
// the standard input, prints the variant that each takes, and fails where a launch's workspaces leave the given memory or overlap.
//   line: forward|backward batch tq tk H Hk d dv lengths -> wide, parts of the keys; or parts of the rows
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "../../paper_2607_12505_amd/csrc/nmspmm_attn_internal.h"

namespace nmspmm {
static size_t ws_bytes;
static char *const ws = (char *)(1ull << 40);
static int wide_of = -1, launches = 0;
static AttnArgs last;

static void fail(const char *what) {
    printf("%s\n", what);
    exit(1);
}
// Regions of floats behind each other within the workspace, in their order.
static void inside(std::vector<std::pair<const float *, int64_t>> regions) {
    const char *end = ws;
    for (const auto &r : regions) {
        if (r.second == 0) continue;
        if ((const char *)r.first < end || ((uintptr_t)r.first & 3)) fail("workspaces overlap");
        end = (const char *)r.first + r.second * 4;
        if (end > ws + ws_bytes) fail("a workspace is too small");
    }
}
static int64_t outer(const AttnArgs &a) { return (int64_t)a.batch * a.Hk; }
static void backward(const AttnArgs &a) {
    ++launches;
    last = a;
    inside({{a.delta, 2 * a.H * a.rows},
            {a.key_parts, a.key_splits > 1 ? outer(a) * a.key_splits * a.tk * (2 * a.d + a.dv) : 0},
            {a.dlam_parts, (int64_t)a.H * a.dlam_count},
            {a.tops, outer(a) * a.row_tiles * 4},
            {a.norms, outer(a) * a.key_tiles}});
}
int device_cu_count() { return 256; }
int launch_rotary(int, const RotaryArgs &, void *) { return 0; }
int launch_diff_forward(int, int, bool wide, const AttnArgs &a, void *) {
    ++launches;
    last = a;
    wide_of = wide;
    if (a.splits > 1) inside({{a.parts, outer(a) * a.splits * a.tq * a.group * (4 + 2 * a.dv)}});
    return 0;
}
int launch_diff_join(int, const AttnArgs &, void *) { return 0; }
int launch_diff_norms(const AttnArgs &a, void *) { return backward(a), 0; }
int launch_diff_grad_q(int, int, const AttnArgs &a, void *) { return backward(a), 0; }
int launch_diff_grad_k(int, int, const AttnArgs &a, void *) { return backward(a), 0; }
int launch_diff_join_keys(int, const AttnArgs &a, void *) { return backward(a), 0; }
}  // namespace nmspmm

using namespace nmspmm;

int main() {
    char what[16];
    int batch, tq, tk, H, Hk, d, dv, lengths;
    while (scanf("%15s %d %d %d %d %d %d %d %d", what, &batch, &tq, &tk, &H, &Hk, &d, &dv, &lengths) == 9) {
        nm_tokens t = {};
        t.batch = batch, t.tq = tq, t.tk = tk, t.left = t.right = -1;
        int32_t *some = (int32_t *)(1ull << 30);
        if (lengths) t.k_lens = some;
        auto heads = [&](int64_t n, int count, int width) {
            return nm_heads{some, n * count * width, (int64_t)count * width, width};
        };
        const nm_heads q = heads(tq, 2 * H, d), k = heads(tk, 2 * Hk, d), v = heads(tk, Hk, dv), o = heads(tq, H, dv);
        nm_diff_weight w = {};
        w.value = (const float *)some;
        launches = 0;
        if (!strcmp(what, "forward")) {
            nm_diff_args a = {q, k, v, o, (int16_t *)some, (float *)some, t, w, NM_TYPE_F16, H, Hk, d, dv, 0.1f};
            if (nm_diff_attention_workspace(&a, &ws_bytes) != NM_OK || nm_diff_attention(&a, ws, ws_bytes, nullptr) != NM_OK ||
                launches != 1)
                fail("forward refused");
            printf("%d %d\n", wide_of, last.splits);
        } else {
            float *f = (float *)some;
            nm_diff_grad_args a = {q,       k, v, o, q, k, v, (int16_t *)some, f, f, f, f, f, f, t, w, NM_TYPE_F16, H, Hk, d,
                                   dv, 0.1f};
            if (nm_diff_attention_backward_workspace(&a, &ws_bytes) != NM_OK ||
                nm_diff_attention_backward(&a, ws, ws_bytes, nullptr) != NM_OK || launches < 1)
                fail("backward refused");
            printf("%d\n", last.key_splits);
        }
    }
    return 0;
}
