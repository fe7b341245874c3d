// C ABI of the operators around a frozen layer: the layer with adapters, the norm in front of it, and clipping by the global norm.
// Validation, workspace carving and launch sequences; documented in include/abtrain.h.
#include <climits>
#include <cmath>
#include <vector>

#include "adapters.h"
#include "api_util.h"

using namespace abt;

namespace {

constexpr int64_t kMaxWidth = 1 << 20, kMaxRows = 1 << 28;     // (launches have fewer than 2^32 threads)

// columns: what m and n are multiples of
int check_adapters(const abt_adapters* ad, const int32_t* row_adapter, int64_t M, int64_t m, int64_t n, int columns) {
    if (!ad || !ad->A || !ad->B || !row_adapter) return ABT_EINVAL;
    if (M < 1 || M > kMaxRows || m < 1 || n < 1 || m > kMaxWidth || n > kMaxWidth || m % 8 || n % columns) return ABT_ESHAPE;
    if (ad->count < 1 || ad->count > 65535 || ad->r < 8 || ad->r > ABT_ADAPTERS_MAX_RANK || ad->r % 8) return ABT_ESHAPE;
    if (!aligned(ad->A, 16) || !aligned(ad->B, 16) || !aligned(ad->ranks, 4) || !aligned(ad->scales, 4) || !aligned(row_adapter, 4)) return ABT_EALIGN;
    return ABT_OK;
}
int check_workspace(const void* ws, size_t have, size_t need) {
    if (!ws || have < need) return ABT_EWORKSPACE;
    return aligned(ws, 256) ? ABT_OK : ABT_EALIGN;
}
AdapterProduct product(const abt_adapters* ad, const int32_t* row_adapter, int64_t M) {
    AdapterProduct p{};
    p.row_adapter = row_adapter; p.ranks = ad->ranks; p.scales = ad->scales; p.M = M; p.count = ad->count; p.r = ad->r;
    return p;
}

size_t t_bytes(int64_t M, int64_t r) { return align_up((size_t)M * (size_t)r * 2, 256); }

// T = X B^T; Tb: scaled and rounded, T: as it is, either may be NULL
hipError_t make_t(const abt_adapters* ad, const int32_t* row_adapter, const void* X, float* T, uint16_t* Tb, int64_t M, int64_t n, hipStream_t s) {
    AdapterProduct p = product(ad, row_adapter, M);
    p.E = (const uint16_t*)X; p.F = (const uint16_t*)ad->B; p.Q = ad->r; p.ke = (int)n; p.e_pitch = (int)n; p.T = T; p.Tb = Tb;
    return launch_adapters_t(p, s);
}

int adapters_fwd(const void* X, const void* main, const float* x_scale, const void* W, const float* w_scale, const abt_adapters* ad, const int32_t* row_adapter,
                 void* Y, float* T, int64_t M, int64_t m, int64_t n, bool fp8, void* ws, hipStream_t s) {
    uint16_t* const Tb = (uint16_t*)ws;
    const bool few = M <= kAdapterFewRows;
    if (!few && make_t(ad, row_adapter, X, T, Tb, M, n, s) != hipSuccess) return ABT_EHIP;
    AdapterProduct p = product(ad, row_adapter, M);
    p.X = main; p.W = W; p.x_scale = x_scale; p.w_scale = w_scale;
    p.E = Tb; p.F = (const uint16_t*)ad->A; p.Q = (int)m; p.kmain = (int)n; p.ke = ad->r; p.e_pitch = ad->r; p.Y = (uint16_t*)Y;
    if (few) { p.T = T; p.Tb = Tb; }
    const hipError_t e = few ? launch_adapters_few(p, (const uint16_t*)X, (const uint16_t*)ad->B, (float*)((char*)ws + t_bytes(M, ad->r)), fp8, s)
                             : launch_adapters_y(p, fp8, s);
    return e == hipSuccess ? ABT_OK : ABT_EHIP;
}

struct BwdPlaces {
    size_t Wt, Bt, T, dT_planes, T_planes, order, offsets, partials, bytes;
};
BwdPlaces bwd_places(int64_t M, int64_t m, int64_t n, int64_t r, int64_t count) {
    BwdPlaces p{};
    size_t at = 0;
    auto take = [&](size_t& where, int64_t bytes) {
        where = at;
        at = align_up(at + (size_t)bytes, 256);
    };
    const int64_t rp = plane_columns((int)r);
    take(p.Wt, m * n * 2);
    take(p.Bt, count * n * r * 2);
    take(p.T, M * r * 4);
    take(p.dT_planes, M * 3 * rp * 2);
    take(p.T_planes, M * 3 * rp * 2);
    take(p.order, M * 4);
    take(p.offsets, (count + 1) * 4);
    take(p.partials, (int64_t)adapters_grad_partial_bytes(M, (int)m, (int)n, (int)r, (int)count));
    p.bytes = at;
    return p;
}

int check_grad_tensors(const abt_grad_tensor* tensors, int n, bool with_out, std::vector<GradTensor>& v) {
    if (n < 0 || (n > 0 && !tensors)) return ABT_EINVAL;
    v.reserve((size_t)n);
    for (int i = 0; i < n; ++i) {
        const abt_grad_tensor& t = tensors[i];
        if (t.dt != ABT_F32 && t.dt != ABT_BF16) return ABT_EDTYPE;
        if (t.count < 0 || t.count > (1ll << 40)) return ABT_ESHAPE;
        if (t.count == 0) continue;
        if (!t.grad) return ABT_EINVAL;
        void* const out = with_out ? (t.out ? t.out : const_cast<void*>(t.grad)) : nullptr;
        if (!aligned(t.grad, 16) || !aligned(out, 16)) return ABT_EALIGN;
        v.push_back(GradTensor{t.grad, out, t.count, t.dt == ABT_BF16});
    }
    return ABT_OK;
}

}  // namespace

extern "C" {

size_t lr_adapters_fwd_workspace_bytes(int64_t M, int64_t m, int64_t n, int64_t r, int64_t count) {
    if (M < 1 || M > kMaxRows || m < 1 || m > kMaxWidth || m % 8 || n < 1 || n > kMaxWidth || n % 8 || r < 8 || r > ABT_ADAPTERS_MAX_RANK || r % 8 || count < 1 || count > 65535)
        return 0;
    return t_bytes(M, r) + (M <= kAdapterFewRows ? align_up(adapters_few_sums_bytes(M, (int)m, (int)n), 256) : 0);
}

int lr_adapters_fwd(const void* X, const void* W, const abt_adapters* adapters, const int32_t* row_adapter, void* Y, float* T_save,
                    int64_t M, int64_t m, int64_t n, int dt, void* workspace, size_t workspace_bytes, void* stream) {
    if (dt != ABT_BF16) return ABT_EDTYPE;
    if (!X || !W || !Y) return ABT_EINVAL;
    int st = check_adapters(adapters, row_adapter, M, m, n, 8);
    if (st != ABT_OK) return st;
    if (!aligned(X, 16) || !aligned(W, 16) || !aligned(Y, 16) || !aligned(T_save, 16)) return ABT_EALIGN;
    st = check_workspace(workspace, workspace_bytes, lr_adapters_fwd_workspace_bytes(M, m, n, adapters->r, adapters->count));
    if (st != ABT_OK) return st;
    return guarded([&] { return adapters_fwd(X, X, nullptr, W, nullptr, adapters, row_adapter, Y, T_save, M, m, n, false, workspace, (hipStream_t)stream); });
}

int lr_adapters_fwd_q8(const void* X, const void* Xq, const float* x_scale, const void* Wq, const float* w_scale, const abt_adapters* adapters,
                       const int32_t* row_adapter, void* Y, int64_t M, int64_t m, int64_t n, void* workspace, size_t workspace_bytes, void* stream) {
    if (!X || !Xq || !x_scale || !Wq || !w_scale || !Y) return ABT_EINVAL;
    int st = check_adapters(adapters, row_adapter, M, m, n, 16);
    if (st != ABT_OK) return st;
    if (!aligned(X, 16) || !aligned(Xq, 16) || !aligned(Wq, 16) || !aligned(Y, 16) || !aligned(x_scale, 4) || !aligned(w_scale, 4)) return ABT_EALIGN;
    st = check_workspace(workspace, workspace_bytes, lr_adapters_fwd_workspace_bytes(M, m, n, adapters->r, adapters->count));
    if (st != ABT_OK) return st;
    return guarded([&] { return adapters_fwd(X, Xq, x_scale, Wq, w_scale, adapters, row_adapter, Y, nullptr, M, m, n, true, workspace, (hipStream_t)stream); });
}

size_t lr_adapters_bwd_workspace_bytes(int64_t M, int64_t m, int64_t n, int64_t r, int64_t count) {
    if (lr_adapters_fwd_workspace_bytes(M, m, n, r, count) == 0) return 0;
    return bwd_places(M, m, n, r, count).bytes;
}

int lr_adapters_bwd(const void* dY, const void* X, const float* T, const void* W, const abt_adapters* adapters, const int32_t* row_adapter,
                    void* dX, float* dA, float* dB, int64_t M, int64_t m, int64_t n, int dt, int accumulate,
                    void* workspace, size_t workspace_bytes, void* stream) {
    if (dt != ABT_BF16) return ABT_EDTYPE;
    if (!dY || (dX && !W) || ((dB || (dA && !T)) && !X)) return ABT_EINVAL;
    int st = check_adapters(adapters, row_adapter, M, m, n, 8);
    if (st != ABT_OK) return st;
    if (!aligned(dY, 16) || !aligned(X, 16) || !aligned(T, 16) || !aligned(W, 16) || !aligned(dX, 16) || !aligned(dA, 16) || !aligned(dB, 16)) return ABT_EALIGN;
    const int64_t r = adapters->r, count = adapters->count;
    const BwdPlaces at = bwd_places(M, m, n, r, count);
    st = check_workspace(workspace, workspace_bytes, at.bytes);
    if (st != ABT_OK) return st;
    if (!dX && !dA && !dB) return ABT_OK;
    return guarded([&]() -> int {
        const hipStream_t s = (hipStream_t)stream;
        char* const ws = (char*)workspace;
        const bool grads = dA || dB;
        if (dA && !T) {
            float* const again = (float*)(ws + at.T);
            if (make_t(adapters, row_adapter, X, again, nullptr, M, n, s) != hipSuccess) return ABT_EHIP;
            T = again;
        }
        AdapterPrep prep{};
        if (dX) { prep.W = (const uint16_t*)W; prep.B = (const uint16_t*)adapters->B; }
        prep.Wt = (uint16_t*)(ws + at.Wt); prep.Bt = (uint16_t*)(ws + at.Bt);
        prep.row_adapter = row_adapter; prep.offsets = (int32_t*)(ws + at.offsets);
        if (grads) prep.order = (int32_t*)(ws + at.order);
        prep.M = M; prep.m = (int)m; prep.n = (int)n; prep.r = (int)r; prep.count = (int)count;
        AdapterProduct p = product(adapters, row_adapter, M);
        p.E = (const uint16_t*)dY; p.F = (const uint16_t*)adapters->A; p.Q = (int)r; p.ke = (int)m; p.e_pitch = (int)m;
        p.dT_planes = (uint16_t*)(ws + at.dT_planes);
        if (dA) { p.T_in = T; p.T_planes = (uint16_t*)(ws + at.T_planes); }
        if (launch_adapters_dt(p, prep, s) != hipSuccess) return ABT_EHIP;
        AdapterProduct x = product(adapters, row_adapter, M);
        x.X = dY; x.W = prep.Wt; x.E = p.dT_planes; x.F = prep.Bt; x.Q = (int)n; x.kmain = (int)m; x.ke = (int)r;
        x.e_pitch = 3 * plane_columns((int)r); x.Y = (uint16_t*)dX;         // the first plane is dT rounded to bf16
        AdapterGrads g{};
        g.dY = (const uint16_t*)dY; g.T_planes = p.T_planes; g.dA = dA; g.X = (const uint16_t*)X; g.dT_planes = p.dT_planes; g.dB = dB;
        g.order = prep.order; g.offsets = prep.offsets; g.partials = (float*)(ws + at.partials);
        g.M = M; g.m = (int)m; g.n = (int)n; g.r = (int)r; g.count = (int)count; g.accumulate = accumulate;
        if (grads && M <= kAdapterFewGradRows) return launch_adapters_few_dx_grads(dX ? &x : nullptr, g, s) == hipSuccess ? ABT_OK : ABT_EHIP;
        const bool beside = dX && grads && adapters_dx_beside_grads(x, g);
        if (dX && !beside && launch_adapters_y(x, false, s) != hipSuccess) return ABT_EHIP;
        if (grads && launch_adapters_grads(g, beside ? &x : nullptr, s) != hipSuccess) return ABT_EHIP;
        return ABT_OK;
    });
}

// ------------------------------------------------------------------------------------------ norm
int lr_rms_norm_fwd(const void* X, const void* residual, const float* gain, double eps, void* H, void* Y, void* Yq, float* y_scale,
                    int64_t M, int64_t n, int dt, void* stream) {
    if (dt != ABT_F32 && dt != ABT_BF16) return ABT_EDTYPE;
    if (!X || !gain || (!Y && !Yq) || (!Yq) != (!y_scale) || !(eps >= 0.0) || !std::isfinite(eps)) return ABT_EINVAL;
    if (M < 1 || n < 8 || n % 8 || n > ABT_RMS_NORM_MAX_WIDTH || M > INT_MAX) return ABT_ESHAPE;
    if (!aligned(X, 16) || !aligned(residual, 16) || !aligned(gain, 16) || !aligned(H, 16) || !aligned(Y, 16) || !aligned(Yq, 16) || !aligned(y_scale, 4))
        return ABT_EALIGN;
    return launch_rms_norm_fwd(X, residual, gain, (float)eps, H, Y, Yq, y_scale, M, (int)n, dt == ABT_BF16, (hipStream_t)stream) == hipSuccess ? ABT_OK : ABT_EHIP;
}

size_t lr_rms_norm_bwd_workspace_bytes(int64_t M, int64_t n, int dt) {
    if (M < 1 || n < 8 || n % 8 || n > ABT_RMS_NORM_MAX_WIDTH || M > INT_MAX || (dt != ABT_F32 && dt != ABT_BF16)) return 0;
    return align_up((size_t)rms_norm_bwd_blocks(M, (int)n, dt == ABT_BF16) * (size_t)n * 4, 256);
}

int lr_rms_norm_bwd(const void* dY, const void* H, const float* gain, double eps, const void* dH, void* dX, float* dgain,
                    int64_t M, int64_t n, int dt, int accumulate, void* workspace, size_t workspace_bytes, void* stream) {
    if (dt != ABT_F32 && dt != ABT_BF16) return ABT_EDTYPE;
    if (!dY || !H || !gain || !(eps >= 0.0) || !std::isfinite(eps)) return ABT_EINVAL;
    if (M < 1 || n < 8 || n % 8 || n > ABT_RMS_NORM_MAX_WIDTH || M > INT_MAX) return ABT_ESHAPE;
    if (!aligned(dY, 16) || !aligned(H, 16) || !aligned(gain, 16) || !aligned(dH, 16) || !aligned(dX, 16) || !aligned(dgain, 16)) return ABT_EALIGN;
    if (dgain) {
        const int st = check_workspace(workspace, workspace_bytes, lr_rms_norm_bwd_workspace_bytes(M, n, dt));
        if (st != ABT_OK) return st;
    }
    if (!dX && !dgain) return ABT_OK;
    return launch_rms_norm_bwd(dY, H, gain, (float)eps, dH, dX, dgain, (float*)workspace, M, (int)n, dt == ABT_BF16, accumulate, (hipStream_t)stream) == hipSuccess
               ? ABT_OK : ABT_EHIP;
}

// ------------------------------------------------------------------------------------------ global norm
size_t ab_grad_norm_workspace_bytes(int n) { return n < 0 ? 0 : align_up((size_t)grad_sums_capacity(n) * sizeof(double), 256); }

int ab_grad_norm(const abt_grad_tensor* tensors, int n, float* norm_out, void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&]() -> int {
        std::vector<GradTensor> v;
        int st = check_grad_tensors(tensors, n, false, v);
        if (st != ABT_OK) return st;
        if (!norm_out) return ABT_EINVAL;
        if (!aligned(norm_out, 4)) return ABT_EALIGN;
        st = check_workspace(workspace, workspace_bytes, ab_grad_norm_workspace_bytes(n));
        if (st != ABT_OK) return st;
        int nsums = 0;
        if (launch_grad_sums(v.data(), (int)v.size(), (double*)workspace, &nsums, (hipStream_t)stream) != hipSuccess) return ABT_EHIP;
        return launch_grad_norm((const double*)workspace, nsums, norm_out, (hipStream_t)stream) == hipSuccess ? ABT_OK : ABT_EHIP;
    });
}

int ab_clip_grads(const abt_grad_tensor* tensors, int n, double max_norm, float* norm_out, void* workspace, size_t workspace_bytes, void* stream) {
    if (!(max_norm >= 0.0) || !std::isfinite(max_norm)) return ABT_EINVAL;
    return guarded([&]() -> int {
        std::vector<GradTensor> v;
        int st = check_grad_tensors(tensors, n, true, v);
        if (st != ABT_OK) return st;
        if (!aligned(norm_out, 4)) return ABT_EALIGN;
        st = check_workspace(workspace, workspace_bytes, ab_grad_norm_workspace_bytes(n));
        if (st != ABT_OK) return st;
        int nsums = 0;
        if (launch_grad_sums(v.data(), (int)v.size(), (double*)workspace, &nsums, (hipStream_t)stream) != hipSuccess) return ABT_EHIP;
        return launch_grad_clip(v.data(), (int)v.size(), (const double*)workspace, nsums, max_norm, norm_out, (hipStream_t)stream) == hipSuccess ? ABT_OK : ABT_EHIP;
    });
}

}  // extern "C"
