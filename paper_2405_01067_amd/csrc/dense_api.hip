// C ABI of the dense layer with its epilogue and of dropout: validation, workspace carving and launch sequences; documented in
// include/abtrain.h.
#include "api_util.h"
#include "dense.h"

using namespace abt;

namespace {

constexpr int64_t kMaxWidth = 1 << 20, kMaxRows = 1 << 28;

bool sizes_fit(int64_t M, int64_t m, int64_t n) { return M >= 1 && M <= kMaxRows && m >= 1 && m <= kMaxWidth && m % 8 == 0 && n >= 1 && n <= kMaxWidth && n % 8 == 0; }
int check_dropout(const abt_dropout* d) {
    if (!d) return ABT_OK;
    if (!d->state || !(d->p >= 0.0 && d->p <= 1.0)) return ABT_EINVAL;
    return aligned(d->state, 8) ? ABT_OK : ABT_EALIGN;
}
int check_dense(int64_t M, int64_t m, int64_t n, int act, const abt_dropout* dropout) {
    if (act < ABT_ACT_NONE || act > ABT_ACT_SILU) return ABT_EINVAL;
    const int st = check_dropout(dropout);
    if (st != ABT_OK) return st;
    return sizes_fit(M, m, n) ? ABT_OK : ABT_ESHAPE;
}

struct Places { size_t Wt, two, third, sums, parts, partials, bytes; };
Places places(int64_t M, int64_t m, int64_t n) {
    Places p{};
    size_t at = 0;
    auto take = [&](size_t& where, size_t bytes) {
        where = at;
        at = align_up(at + bytes, 256);
    };
    take(p.Wt, (size_t)(m * n * 4));                      // twice; and two parts of dZ beside each other, and the third
    take(p.two, (size_t)(M * m * 4));
    take(p.third, (size_t)(M * m * 2));
    take(p.sums, (size_t)(ceil_div(M, dense_piece_rows(M, (int)m)) * m * 4));
    const size_t once = dense_part_bytes(M, (int)n, (int)m), twice = dense_part_bytes(M, (int)n, (int)(2 * m));
    take(p.parts, once > twice ? once : twice);
    take(p.partials, dense_grad_partial_bytes(M, (int)m, (int)n));
    p.bytes = at;
    return p;
}

}  // namespace

extern "C" {

size_t lr_dense_fwd_workspace_bytes(int64_t M, int64_t m, int64_t n) {
    return sizes_fit(M, m, n) ? align_up(dense_part_bytes(M, (int)m, (int)n), 256) : 0;
}

int lr_dense_fwd(const void* X, const void* W, const float* bias, const void* residual, void* Y, void* Z_save,
                 int64_t M, int64_t m, int64_t n, int act, const abt_dropout* dropout, int dt, void* workspace, size_t workspace_bytes, void* stream) {
    if (dt != ABT_BF16) return ABT_EDTYPE;
    if (!X || !W || !Y) return ABT_EINVAL;
    const int st = check_dense(M, m, n, act, dropout);
    if (st != ABT_OK) return st;
    if (!aligned(X, 16) || !aligned(W, 16) || !aligned(bias, 16) || !aligned(residual, 16) || !aligned(Y, 16) || !aligned(Z_save, 16)) return ABT_EALIGN;
    const size_t need = lr_dense_fwd_workspace_bytes(M, m, n);
    if (need && (!workspace || workspace_bytes < need)) return ABT_EWORKSPACE;
    if (need && !aligned(workspace, 256)) return ABT_EALIGN;
    const DenseProduct p{(const uint16_t*)X, (const uint16_t*)W, (uint16_t*)Y, bias, (const uint16_t*)residual, (uint16_t*)Z_save, M, (int)m, (int)n, act, 1.0f, drop_of(dropout),
                         (float*)workspace, 0};
    return launch_dense(p, (hipStream_t)stream) == hipSuccess ? ABT_OK : ABT_EHIP;
}

size_t lr_dense_bwd_workspace_bytes(int64_t M, int64_t m, int64_t n) { return sizes_fit(M, m, n) ? places(M, m, n).bytes : 0; }

int lr_dense_bwd(const void* dY, const void* X, const void* W, const void* Z, void* dX, float* dW, float* dbias,
                 int64_t M, int64_t m, int64_t n, int act, const abt_dropout* dropout, int dt, int accumulate,
                 void* workspace, size_t workspace_bytes, void* stream) {
    if (dt != ABT_BF16) return ABT_EDTYPE;
    if (!dY || (dX && !W) || (dW && !X) || (act != ABT_ACT_NONE && !Z)) return ABT_EINVAL;
    const int st = check_dense(M, m, n, act, dropout);
    if (st != ABT_OK) return st;
    if (!aligned(dY, 16) || !aligned(X, 16) || !aligned(W, 16) || !aligned(Z, 16) || !aligned(dX, 16) || !aligned(dW, 16) || !aligned(dbias, 16)) return ABT_EALIGN;
    const Places at = places(M, m, n);
    if (!workspace || workspace_bytes < at.bytes) return ABT_EWORKSPACE;
    if (!aligned(workspace, 256)) return ABT_EALIGN;
    if (!dX && !dW && !dbias) return ABT_OK;
    const hipStream_t s = (hipStream_t)stream;
    char* const ws = (char*)workspace;
    const Drop drop = drop_of(dropout);
    const bool smooth = act != ABT_ACT_NONE && act != ABT_ACT_RELU;

    DenseSlope z{};
    z.dY = (const uint16_t*)dY; z.Z = act == ABT_ACT_NONE ? nullptr : (const uint16_t*)Z;
    const int values = smooth ? 3 : 1;
    if ((dX || dW) && (z.Z || drop.state)) {
        z.value[0] = (uint16_t*)(ws + at.two);
        if (values > 1) z.value[1] = z.value[0] + m;
        if (values > 1 && dW) z.value[2] = (uint16_t*)(ws + at.third);
    }
    if (dbias) z.sums = (float*)(ws + at.sums);
    if (dX) { z.W = (const uint16_t*)W; z.Wt = (uint16_t*)(ws + at.Wt); }
    z.values = values; z.M = M; z.m = (int)m; z.n = (int)n; z.act = act; z.scaled = smooth; z.rows = dense_piece_rows(M, (int)m); z.drop = drop;
    if (launch_dense_slope(z, s) != hipSuccess) return ABT_EHIP;
    const uint16_t* const dZ = z.value[0] ? z.value[0] : z.dY;
    const float alpha = smooth ? 1.0f : drop.scale;       // what dZ was left without
    const DenseProduct x{dZ, z.Wt, (uint16_t*)dX, nullptr, nullptr, nullptr, M, (int)n, pitch_of(values) * (int)m, ABT_ACT_NONE, alpha, Drop{nullptr, 0, 0, 1.0f}, (float*)(ws + at.parts), 0};
    const DenseGrads g{{dZ, z.value[1], z.value[2]}, (const uint16_t*)X, dW, (float*)(ws + at.partials), z.sums, dbias, M, (int)m, (int)n, (int)ceil_div(M, z.rows), accumulate, values, alpha};
    return launch_dense_bwd(x, g, s) == hipSuccess ? ABT_OK : ABT_EHIP;
}

int lr_dropout(const void* X, const void* residual, void* Y, int64_t count, const abt_dropout* dropout, int dt, void* stream) {
    if (dt != ABT_F32 && dt != ABT_BF16) return ABT_EDTYPE;
    if (!dropout) return ABT_EINVAL;
    const int st = check_dropout(dropout);
    if (st != ABT_OK) return st;
    if (count < 0 || count > (1ll << 45)) return ABT_ESHAPE;
    if (count == 0) return ABT_OK;
    if (!X || !Y) return ABT_EINVAL;
    if (!aligned(X, 16) || !aligned(residual, 16) || !aligned(Y, 16)) return ABT_EALIGN;
    return launch_dropout(X, residual, Y, count, drop_of(dropout), dt == ABT_BF16, (hipStream_t)stream) == hipSuccess ? ABT_OK : ABT_EHIP;
}

}  // extern "C"
