// C ABI of the attention to states that are not the sequence's own: argument validation and
// workspace layout.  The declarations and their contracts are in include/fibattn.h.
#include <math.h>

#include "checks.h"
#include "cross_launch.h"

using namespace fibattn;

namespace {

fibattn_status_t check_sizes(int B, int B_kv, int H, int H_kv, int T, int S, int d_head, fibattn_dtype_t dtype) {
    if (B < 1 || H < 1 || T < 1 || S < 1 || H_kv < 1 || H_kv > H || H % H_kv) return FIBATTN_ERR_INVALID_ARG;
    if (B_kv != B && B_kv != 1) return FIBATTN_ERR_INVALID_ARG;
    if (dtype != FIBATTN_FP32 && dtype != FIBATTN_BF16) return FIBATTN_ERR_INVALID_ARG;
    if (d_head != 32 && d_head != 64 && d_head != 128) return FIBATTN_ERR_UNSUPPORTED;
    // rows of queries and of one head's states are counted in 32 bits
    if ((long long)B * H > 65535 || (long long)B * H * T > (1ll << 30) || S > 1 << 30) return FIBATTN_ERR_UNSUPPORTED;
    return FIBATTN_OK;
}

// The caller's placements, or packed tensors [batch, heads, rows, d] where there are none.
struct Place {
    const fibattn_layout_t *l;
    fibattn_dtype_t dtype;
    int D;
    bool ok;
    bool near;  // 64 rows of a head span less than 2^31 bytes
    Layout next(int heads, int rows) {
        if (!l) return Layout::packed(heads, rows, D);
        const fibattn_layout_t x = *l++;
        ok = ok && strides_ok(x, dtype);
        near = near && x.pos < 1ll << 22;
        return {x.batch, x.head, x.pos};
    }
};

float tau_of(int D) { return (float)(1.0 / sqrt((double)D)); }
float scale_of(int D) { return (float)(1.4426950408889634073599246810019 / sqrt((double)D)); }

// Partial results: o of every slot, then lse of every slot.
size_t parts_bytes(int parts, long long rows, int D) {
    return parts < 2 ? 0 : align256(sizeof(float) * parts * rows * D) + align256(sizeof(float) * parts * rows);
}
void place_parts(Queries *a, void *workspace, int parts, int D) {
    const long long rows = (long long)a->B * a->H * a->T;
    a->part_o = parts < 2 ? nullptr : (float *)workspace;
    a->part_lse = parts < 2 ? nullptr : (float *)((char *)workspace + align256(sizeof(float) * parts * rows * D));
}

// States of S rows for a batch of B: its own (B_kv = B) or shared ones (B_kv = 1).
States states_of(int B, int B_kv, int H, int H_kv, int T, int S) {
    States s{};
    s.S = S;
    s.share = B / B_kv;
    s.rows = s.share * (H / H_kv) * T;
    return s;
}

// Bytes of the partial results, of both types the larger.
size_t forward_bytes(int D, States s0, States *s1, int prob0, int prob1, long long rows) {
    size_t most = 0;
    for (int t = 0; t < 2; ++t) {
        const size_t x = parts_bytes(plan_cross_forward(t, D, &s0, s1, prob0, prob1), rows, D);
        most = x > most ? x : most;
    }
    return most;
}

struct BackwardPlan {
    Gradients g;
    size_t dq, dk, dv, total;  // offsets behind the statistics
};
BackwardPlan plan_backward(int dtype, int B, int B_kv, int H, int H_kv, int T, int S, int D) {
    BackwardPlan p{};
    Gradients &g = p.g;
    g.B = B; g.Bkv = B_kv; g.H = H; g.Hkv = H_kv; g.G = H / H_kv; g.T = T; g.S = S;
    g.share = B / B_kv;
    g.rows = g.share * g.G * T;
    plan_cross_backward(dtype, D, &g);
    const size_t q = sizeof(float) * (size_t)B * H * T * D, k = sizeof(float) * (size_t)B_kv * H_kv * S * D;
    p.dq = align256(sizeof(float) * 64 * (size_t)B * H * ((T + 31) / 32));
    p.dk = p.dq + (g.dq_pieces > 1 ? align256(q * g.dq_pieces) : 0);
    p.dv = p.dk + (g.dkv_pieces > 1 ? align256(k * g.dkv_pieces) : 0);
    p.total = p.dv + (g.dkv_pieces > 1 ? align256(k * g.dkv_pieces) : 0);
    return p;
}

template <size_t N> bool all_aligned(const void *const (&p)[N]) {
    for (const void *x : p)
        if (!x || !aligned16(x)) return false;
    return true;
}

bool lens_ok(const int32_t *lens) { return ((uintptr_t)lens & 3u) == 0; }

}  // namespace

extern "C" {

size_t fibattn_cross_workspace_bytes(int B, int B_kv, int H, int H_kv, int T, int S, int d_head) {
    if (check_sizes(B, B_kv, H, H_kv, T, S, d_head, FIBATTN_BF16) != FIBATTN_OK) return 0;
    const States s = states_of(B, B_kv, H, H_kv, T, S);
    return forward_bytes(d_head, s, nullptr, B_kv * H_kv, 0, (long long)B * H * T);
}

fibattn_status_t fibattn_cross_forward(const void *q, const void *k, const void *v, void *o, float *lse,
                                       const int32_t *lens, void *workspace, size_t workspace_bytes,
                                       const fibattn_layout_t *layouts, int B, int B_kv, int H, int H_kv, int T, int S,
                                       int d_head, fibattn_dtype_t dtype, hipStream_t stream) {
    fibattn_status_t st = check_sizes(B, B_kv, H, H_kv, T, S, d_head, dtype);
    if (st != FIBATTN_OK) return st;
    if (!all_aligned({q, k, v, o, (const void *)lse}) || !lens_ok(lens)) return FIBATTN_ERR_INVALID_ARG;
    Place at = {layouts, dtype, d_head, true, true};
    Queries a{};
    States s = states_of(B, B_kv, H, H_kv, T, S);
    a.lq = at.next(H, T);
    s.lk = at.next(H_kv, S);
    s.lv = at.next(H_kv, S);
    a.lo = at.next(H, T);
    if (!at.ok) return FIBATTN_ERR_INVALID_ARG;
    if (!at.near) return FIBATTN_ERR_UNSUPPORTED;
    const int parts = plan_cross_forward((int)dtype, d_head, &s, nullptr, B_kv * H_kv, 0);
    const size_t need = parts_bytes(parts, (long long)B * H * T, d_head);
    if (need && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return FIBATTN_ERR_WORKSPACE;
    a.q = q; a.o = o; a.lse = lse;
    a.B = B; a.H = H; a.Hkv = H_kv; a.G = H / H_kv; a.T = T;
    a.scale = scale_of(d_head);
    place_parts(&a, workspace, parts, d_head);
    s.k = k; s.v = v; s.lens = lens;
    const hipError_t e = launch_cross_forward((int)dtype, d_head, a, s, nullptr, B_kv * H_kv, 0, stream);
    return e == hipSuccess ? FIBATTN_OK : FIBATTN_ERR_HIP;
}

size_t fibattn_cross_backward_workspace_bytes(int B, int B_kv, int H, int H_kv, int T, int S, int d_head) {
    if (check_sizes(B, B_kv, H, H_kv, T, S, d_head, FIBATTN_BF16) != FIBATTN_OK) return 0;
    const size_t x = plan_backward(0, B, B_kv, H, H_kv, T, S, d_head).total;
    const size_t y = plan_backward(1, B, B_kv, H, H_kv, T, S, d_head).total;
    return x > y ? x : y;  // of both types
}

fibattn_status_t fibattn_cross_backward(const void *q, const void *k, const void *v, const void *o, const float *lse,
                                        const void *dO, void *dq, void *dk, void *dv, const int32_t *lens,
                                        void *workspace, size_t workspace_bytes, const fibattn_layout_t *layouts,
                                        int B, int B_kv, int H, int H_kv, int T, int S, int d_head,
                                        fibattn_dtype_t dtype, hipStream_t stream) {
    fibattn_status_t st = check_sizes(B, B_kv, H, H_kv, T, S, d_head, dtype);
    if (st != FIBATTN_OK) return st;
    if (!all_aligned({q, k, v, o, (const void *)lse, dO, dq, dk, dv}) || !lens_ok(lens)) return FIBATTN_ERR_INVALID_ARG;
    const BackwardPlan p = plan_backward((int)dtype, B, B_kv, H, H_kv, T, S, d_head);
    if (!workspace || !aligned16(workspace) || workspace_bytes < p.total) return FIBATTN_ERR_WORKSPACE;
    Gradients g = p.g;
    Place at = {layouts, dtype, d_head, true, true};
    g.lq = at.next(H, T);
    g.lk = at.next(H_kv, S);
    g.lv = at.next(H_kv, S);
    g.lo = at.next(H, T);
    g.lg = at.next(H, T);
    g.ldq = at.next(H, T);
    g.ldk = at.next(H_kv, S);
    g.ldv = at.next(H_kv, S);
    if (!at.ok) return FIBATTN_ERR_INVALID_ARG;
    if (!at.near) return FIBATTN_ERR_UNSUPPORTED;
    g.q = q; g.k = k; g.v = v; g.o = o; g.g = dO; g.lse = lse;
    g.dq = dq; g.dk = dk; g.dv = dv;
    g.lens = lens;
    char *ws = (char *)workspace;
    g.stats = (float *)ws;
    g.dq_part = (float *)(ws + p.dq);
    g.dk_part = (float *)(ws + p.dk);
    g.dv_part = (float *)(ws + p.dv);
    g.tau = tau_of(d_head);
    g.scale = scale_of(d_head);
    const hipError_t e = launch_cross_backward((int)dtype, d_head, g, stream);
    return e == hipSuccess ? FIBATTN_OK : FIBATTN_ERR_HIP;
}

size_t fibattn_prefix_workspace_bytes(int B, int H, int H_kv, int T, int P, int S, int d_head) {
    if (check_sizes(B, 1, H, H_kv, T, P, d_head, FIBATTN_BF16) != FIBATTN_OK ||
        check_sizes(B, B, H, H_kv, T, S, d_head, FIBATTN_BF16) != FIBATTN_OK)
        return 0;
    States own = states_of(B, B, H, H_kv, T, S);
    return forward_bytes(d_head, states_of(B, 1, H, H_kv, T, P), &own, H_kv, B * H_kv, (long long)B * H * T);
}

fibattn_status_t fibattn_prefix_forward(const void *q, const void *k_prefix, const void *v_prefix, const void *k,
                                        const void *v, void *o, float *lse, const int32_t *lens, void *workspace,
                                        size_t workspace_bytes, const fibattn_layout_t *layouts, int B, int H,
                                        int H_kv, int T, int P, int S, int d_head, fibattn_dtype_t dtype,
                                        hipStream_t stream) {
    fibattn_status_t st = check_sizes(B, 1, H, H_kv, T, P, d_head, dtype);
    if (st == FIBATTN_OK) st = check_sizes(B, B, H, H_kv, T, S, d_head, dtype);
    if (st != FIBATTN_OK) return st;
    if (!all_aligned({q, k_prefix, v_prefix, k, v, o, (const void *)lse}) || !lens_ok(lens))
        return FIBATTN_ERR_INVALID_ARG;
    Place at = {layouts, dtype, d_head, true, true};
    Queries a{};
    States pre = states_of(B, 1, H, H_kv, T, P), own = states_of(B, B, H, H_kv, T, S);
    a.lq = at.next(H, T);
    pre.lk = at.next(H_kv, P);
    pre.lv = at.next(H_kv, P);
    own.lk = at.next(H_kv, S);
    own.lv = at.next(H_kv, S);
    a.lo = at.next(H, T);
    if (!at.ok) return FIBATTN_ERR_INVALID_ARG;
    if (!at.near) return FIBATTN_ERR_UNSUPPORTED;
    const int parts = plan_cross_forward((int)dtype, d_head, &pre, &own, H_kv, B * H_kv);
    const size_t need = parts_bytes(parts, (long long)B * H * T, d_head);
    if (!workspace || !aligned16(workspace) || workspace_bytes < need) return FIBATTN_ERR_WORKSPACE;
    a.q = q; a.o = o; a.lse = lse;
    a.B = B; a.H = H; a.Hkv = H_kv; a.G = H / H_kv; a.T = T;
    a.scale = scale_of(d_head);
    place_parts(&a, workspace, parts, d_head);
    pre.k = k_prefix; pre.v = v_prefix;
    own.k = k; own.v = v; own.lens = lens;
    own.causal = 1;
    const hipError_t e = launch_cross_forward((int)dtype, d_head, a, pre, &own, H_kv, B * H_kv, stream);
    return e == hipSuccess ? FIBATTN_OK : FIBATTN_ERR_HIP;
}

fibattn_status_t fibattn_join(const void *o_a, const float *lse_a, const void *o_b, const float *lse_b, void *o,
                              float *lse, const fibattn_layout_t *layouts, int B, int H, int T, int d_head,
                              fibattn_dtype_t dtype, hipStream_t stream) {
    const fibattn_status_t st = check_sizes(B, B, H, H, T, 1, d_head, dtype);
    if (st != FIBATTN_OK) return st;
    if (!all_aligned({o_a, (const void *)lse_a, o_b, (const void *)lse_b, (const void *)o, (const void *)lse}))
        return FIBATTN_ERR_INVALID_ARG;
    Place at = {layouts, dtype, d_head, true, true};
    JoinArgs j{o_a, o_b, lse_a, lse_b, o, lse, {}, {}, {}, B, H, T};
    j.la = at.next(H, T);
    j.lb = at.next(H, T);
    j.lo = at.next(H, T);
    if (!at.ok) return FIBATTN_ERR_INVALID_ARG;
    if (!at.near) return FIBATTN_ERR_UNSUPPORTED;
    const hipError_t e = launch_join((int)dtype, d_head, j, stream);
    return e == hipSuccess ? FIBATTN_OK : FIBATTN_ERR_HIP;
}

}  // extern "C"
