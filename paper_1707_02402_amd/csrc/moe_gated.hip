// The first half of a gated feed-forward layer of experts, out = f(in Wg_e^T) (in Wu_e^T), and the gradients of its gate and up through the second layer's product:
// dact = dout W_e, dgate = dact up f'(gate), dup = dact f(gate).  W is [E][2][h][K], so that [dgate, dup] and W are an ordinary layer's (N = 2 h) for the products that remain.
#include "moe_tiles.h"

namespace {

template <int DIR>
__global__ __launch_bounds__(256, 2) void k_gated_any(Args p, Gate gate, int units, int ct)
{
    product_tiles_any<DIR, bf16_t>(p, gate, units, ct, 1, Shares{}, nullptr);
}

template <int DIR, class S, int KEEP>
__global__ __launch_bounds__(S::THREADS, S::SIMD) void k_gated(Args p, GateKeeping<KEEP> gate, int units, int ct)
{
    product_tiles<DIR, bf16_t, S, false>(p, gate, units, ct, 1, Shares{}, nullptr);
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

// LDS beyond 64 KB has to be asked for: a kernel is asked for once on every device (beyond DEVICES, at every call)
template <class K, class... A>
int launch_with(K kernel, std::atomic<bool>* asked, uint32_t lds, int64_t grid, int threads, hipStream_t st, const char* who, A... args)
{
    constexpr int DEVICES = 64;
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e == hipSuccess && (dev < 0 || dev >= DEVICES || !asked[dev].load())) {
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
        if (e == hipSuccess && dev >= 0 && dev < DEVICES) asked[dev].store(true);
    }
    if (e != hipSuccess) return fail(DYNB_E_HIP, std::string(who) + ": " + hipGetErrorString(e));
    hipLaunchKernelGGL(kernel, dim3(unsigned(grid)), dim3(unsigned(threads)), lds, st, args...);
    return launched(who);
}

template <int DIR>
int launch_gated(const moe_product_shape* s, const Args& p, const Gate& gate, bool fast, hipStream_t st, const char* who)
{
    auto launch = [&](auto kind, auto keep) {
        using S = decltype(kind);
        constexpr int KEEP = decltype(keep)::value;
        static std::atomic<bool> asked[64];
        const int wide = DIR == FORWARD ? S::COLS / 2 : S::COLS, ct = (gate.h + wide - 1) / wide;
        const int64_t units = (S::BIG ? int64_t(s->M) / S::ROWS + s->E + 1 : most_pieces(s->M, s->E, S::ROWS)) * ct;
        if (units > MOST_GROUPS) return fail(DYNB_E_UNSUPPORTED, std::string(who) + ": too many results");
        GateKeeping<KEEP> g = {};
        static_cast<Gate&>(g) = gate;
        return launch_with(k_gated<DIR, S, KEEP>, asked, LDS_BYTES<DIR, S>, S::BIG ? std::min<int64_t>(units, CUS) : units, S::THREADS, st, who, p, g, int(units), ct);
    };
    auto keeping = [&](auto kind) {
        if (gate.keep == KEEP_8) return launch(kind, std::integral_constant<int, KEEP_8>{});
        if constexpr (DIR == FORWARD)
            if (gate.keep == KEEP_NOTHING) return launch(kind, std::integral_constant<int, KEEP_NOTHING>{});
        return launch(kind, std::integral_constant<int, KEEP_BF16>{});
    };
    if (fast) switch (kind_of(s, DIR == FORWARD ? s->N : s->K, DIR == FORWARD ? s->K : s->N)) {
        case BIG: return keeping(Big{});
        case MID: return keeping(Mid{});
        default:
            if constexpr (DIR == FORWARD) {                    // (8 bits: 32 features have to be a wave's)
                if (gate.keep == KEEP_8) return launch(Mid{}, std::integral_constant<int, KEEP_8>{});
                if (gate.keep == KEEP_NOTHING) return launch(Few{}, std::integral_constant<int, KEEP_NOTHING>{});
                return launch(Few{}, std::integral_constant<int, KEEP_BF16>{});
            } else return keeping(Few{});
        }
    static std::atomic<bool> asked[64];
    const int wide = DIR == FORWARD ? Mid::COLS / 2 : Mid::COLS, ct = (gate.h + wide - 1) / wide;
    const int64_t units = most_pieces(s->M, s->E, Mid::ROWS) * ct;
    if (units > MOST_GROUPS) return fail(DYNB_E_UNSUPPORTED, std::string(who) + ": too many results");
    return launch_with(k_gated_any<DIR>, asked, LDS_BYTES<DIR, Mid>, units, 256, st, who, p, gate, int(units), ct);
}

// whether what is kept lies on borders of 8 elements
bool kept_on_8(const moe_gated_pre* p)
{
    if (!p) return true;
    if (p->dtype == DYNB_BF16) return p->stride % 8 == 0 && on_16({p->rows});
    return p->stride % 8 == 0 && (reinterpret_cast<uintptr_t>(p->rows) & 7) == 0;
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
    // (32-bit offsets within an expert's two matrices: up's rows lie h rows behind gate's)
    const bool fast = s->K % 8 == 0 && s->h % 8 == 0 && in_stride % 8 == 0 && out_stride % 8 == 0 && on_16({in, W, out}) && kept_on_8(pre) && reached(g, in_stride, 0) &&
                      (int64_t(s->h) + 256) * s->K * 2 < int64_t(1) << 32;
    return launch_gated<FORWARD>(&as, p, gate_of(s, pre, nullptr, 0), fast, static_cast<hipStream_t>(stream), "moe_gated");
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
    const bool fast = s->K % 8 == 0 && s->h % 8 == 0 && dout_stride % 8 == 0 && dpre_stride % 8 == 0 && hidden_stride % 8 == 0 && on_16({dout, W, dpre, hidden}) && kept_on_8(pre) &&
                      reached(g, 0, dout_stride);
    return launch_gated<GRAD_INPUT>(&as, p, gate_of(s, pre, hidden, hidden_stride), fast, static_cast<hipStream_t>(stream), "moe_gated_grad");
}
