// The first half of a gated feed-forward layer of experts, out = f(in Wg_e^T) (in Wu_e^T), and the gradients of its gate and up through the second layer's product:
// dact = dout W_e, dgate = dact up f'(gate), dup = dact f(gate).  W is [E][2][h][K], so that [dgate, dup] and W are an ordinary layer's (N = 2 h) for the products that remain.
#include "moe_tiles.h"

namespace {

template <int DIR>
__global__ __launch_bounds__(256, 2) void k_gated_any(Args p, Gate gate, int units, int ct)
{
    product_tiles_any<DIR, bf16_t>(p, gate, units, ct, 1, Shares{}, nullptr);
}

int check(const moe_gated_shape* s, const std::string& who)
{
    if (!s) return fail(DYNB_E_INVAL, who + ": NULL shape");
    if (s->M < 0 || s->K <= 0 || s->h <= 0 || s->E <= 0) return fail(DYNB_E_INVAL, who + ": sizes must be positive");
    if (s->dtype != DYNB_BF16) return fail(DYNB_E_UNSUPPORTED, who + ": only DYNB_BF16");
    if (s->flags > MOE_GATE_GELU) return fail(DYNB_E_UNSUPPORTED, who + ": unknown flag");
    if (s->M > 1 << 30 || s->E > 1 << 20 || s->K > 1 << 22 || s->h > 1 << 21) return fail(DYNB_E_UNSUPPORTED, who + ": more than 2^30 rows, 2^22 channels, 2^21 hidden features or 2^20 experts");
    return DYNB_OK;
}
int check_pre(const moe_gated_shape* s, const moe_gated_pre* p, const std::string& who)
{
    if (p->dtype != DYNB_BF16 && p->dtype != DYNB_I8) return fail(DYNB_E_UNSUPPORTED, who + ": unknown dtype of what is kept");
    if (!p->rows || (p->dtype == DYNB_I8 && !p->scale)) return fail(DYNB_E_INVAL, who + ": NULL pre");
    if (p->stride < 2 * int64_t(s->h) || (p->dtype == DYNB_I8 && p->scale_stride < 2 * ((int64_t(s->h) + BLOCK8 - 1) / BLOCK8)))
        return fail(DYNB_E_INVAL, who + ": rows of pre overlap (stride below their length)");
    if ((p->dtype == DYNB_BF16 && odd(p->rows)) || (p->dtype == DYNB_I8 && odd(p->scale))) return fail(DYNB_E_INVAL, who + ": misaligned pre");
    return DYNB_OK;
}
Gate gate_of(const moe_gated_shape* s, const moe_gated_pre* p, void* hidden, int64_t hidden_stride)
{
    constexpr double LOG2E = 1.4426950408889634, C = 1.5957691216057308;                   // 2 sqrt(2 / pi)
    const double a = s->flags == MOE_GATE_GELU ? C : 1.0, b = s->flags == MOE_GATE_GELU ? C * 0.044715 : 0.0;
    Gate g = {};
    g.form = GateForm{float(-LOG2E * a), float(-LOG2E * b), float(a), float(3 * b)};
    g.h = s->h;
    g.keep = !p ? KEEP_NOTHING : p->dtype == DYNB_BF16 ? KEEP_BF16 : KEEP_8;
    if (p) {
        g.pre = p->rows;
        g.pre_stride = p->stride;
        g.scale = static_cast<bf16_t*>(p->scale);
        g.scale_stride = p->scale_stride;
    }
    g.hidden = static_cast<bf16_t*>(hidden);
    g.hidden_stride = hidden_stride;
    return g;
}

template <int DIR>
int launch_gated(const moe_product_shape* s, const Args& p, const Gate& gate, hipStream_t st, const char* who)
{
    const int wide = DIR == FORWARD ? Mid::COLS / 2 : Mid::COLS, ct = (gate.h + wide - 1) / wide;
    const int64_t units = most_pieces(s->M, s->E, Mid::ROWS) * ct;
    if (units > MOST_GROUPS) return fail(DYNB_E_UNSUPPORTED, std::string(who) + ": too many results");
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k_gated_any<DIR>), hipFuncAttributeMaxDynamicSharedMemorySize, int(LDS_BYTES<DIR, Mid>));
    if (e != hipSuccess) return fail(DYNB_E_HIP, std::string(who) + ": " + hipGetErrorString(e));
    hipLaunchKernelGGL((k_gated_any<DIR>), dim3(unsigned(units)), dim3(256), (LDS_BYTES<DIR, Mid>), st, p, gate, int(units), ct);
    return launched(who);
}

}  // namespace

extern "C" int moe_gated(const moe_gated_shape* s, const moe_groups* g, const void* in, int64_t in_stride, const void* W, void* out, int64_t out_stride, const moe_gated_pre* pre, void* stream)
{
    int rc = check(s, "moe_gated");
    if (rc != DYNB_OK) return rc;
    const moe_product_shape as = {s->M, s->K, 2 * s->h, s->E, DYNB_BF16, 0};
    rc = check_groups(&as, g, true, "moe_gated");
    if (rc == DYNB_OK && pre && s->M > 0) rc = check_pre(s, pre, "moe_gated");
    if (rc != DYNB_OK || s->M == 0) return rc;
    if (!in || !W || !out) return fail(DYNB_E_INVAL, "moe_gated: NULL argument");
    if (in_stride < s->K || out_stride < s->h) return fail(DYNB_E_INVAL, "moe_gated: rows overlap (stride below their length)");
    if (odd(in) || odd(W) || odd(out)) return fail(DYNB_E_INVAL, "moe_gated: misaligned pointer");
    const Args p = {groups_of(&as, g), static_cast<const bf16_t*>(W), static_cast<const bf16_t*>(in), 0, in_stride, nullptr, 0, out, out_stride, as.K, as.N, 0};
    return launch_gated<FORWARD>(&as, p, gate_of(s, pre, nullptr, 0), static_cast<hipStream_t>(stream), "moe_gated");
}

extern "C" int moe_gated_grad(const moe_gated_shape* s, const moe_groups* g, const void* dout, int64_t dout_stride, const void* W, const moe_gated_pre* pre, void* dpre, int64_t dpre_stride,
                              void* hidden, int64_t hidden_stride, void* stream)
{
    int rc = check(s, "moe_gated_grad");
    if (rc != DYNB_OK) return rc;
    const moe_product_shape as = {s->M, s->h, s->K, s->E, DYNB_BF16, 0};
    rc = check_groups(&as, g, false, "moe_gated_grad");
    if (rc != DYNB_OK || s->M == 0) return rc;
    if (!dout || !W || !pre || !dpre) return fail(DYNB_E_INVAL, "moe_gated_grad: NULL argument");
    rc = check_pre(s, pre, "moe_gated_grad");
    if (rc != DYNB_OK) return rc;
    if (dout_stride < s->K || dpre_stride < 2 * int64_t(s->h) || (hidden && hidden_stride < s->h)) return fail(DYNB_E_INVAL, "moe_gated_grad: rows overlap (stride below their length)");
    if (odd(dout) || odd(W) || odd(dpre) || odd(hidden)) return fail(DYNB_E_INVAL, "moe_gated_grad: misaligned pointer");
    const Args p = {groups_of(&as, g), static_cast<const bf16_t*>(W), static_cast<const bf16_t*>(dout), 0, dout_stride, nullptr, 0, dpre, dpre_stride, as.K, as.N, 0};
    return launch_gated<GRAD_INPUT>(&as, p, gate_of(s, pre, hidden, hidden_stride), static_cast<hipStream_t>(stream), "moe_gated_grad");
}
