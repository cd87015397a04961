// extern "C" entry points of layer norm, router and exchange of rows: synchronous
// argument checks, then the launches.  The semantics of every call are documented
// in include/shiftquant.h.
#include <cmath>
#include <cstdint>

#include "sq_block.h"
#include "sq_checks.h"

namespace {

using namespace sq;

sq_status check_norm(int32_t type, int32_t param_type, int64_t M, int64_t C, const void* gamma) {
    SQ_TRY(check_type(type));
    SQ_TRY(check_type(param_type));
    SQ_TRY(check_dim(M, kMaxRows, "M"));
    SQ_TRY(check_dim(C, kMaxCols, "C"));
    if (C > 0) SQ_TRY(check_values(gamma, param_type, C, C, "gamma"));
    return SQ_OK;
}

sq_status check_stats(const float* stats) {
    if (!aligned(stats, 16)) return invalid("stats must be 16-byte aligned");
    return SQ_OK;
}

sq_status check_route_tokens(int64_t T) {
    SQ_TRY(check_dim(T, kMaxRows, "T"));
    if (T > kRouteMaxTokens) return fail(SQ_ERR_UNSUPPORTED, "more than 2^26 - 4 tokens");
    return SQ_OK;
}

sq_status check_router(int32_t type, int64_t T, int64_t E, int32_t k, int32_t score, int32_t groups, int32_t top_groups,
                       int32_t renormalize, float scale, int64_t ld) {
    SQ_TRY(check_type(type));
    if (score != SQ_SCORE_SOFTMAX && score != SQ_SCORE_SIGMOID) return invalid("score must be SQ_SCORE_SOFTMAX or SQ_SCORE_SIGMOID");
    if (renormalize != 0 && renormalize != 1) return invalid("renormalize must be 0 or 1");
    SQ_TRY(check_route_tokens(T));
    if (E < 1 || k < 1 || k > E) return invalid("E and k must be positive and k at most E");
    if (E > kRouteMaxExperts || k > kRouteMaxTopK) return fail(SQ_ERR_UNSUPPORTED, "more than 1024 experts or 64 slots");
    if (groups < 1 || E % groups) return invalid("groups must divide E");
    if (groups > kRouteMaxGroups) return fail(SQ_ERR_UNSUPPORTED, "more than 64 groups");
    if (top_groups < 1 || top_groups > groups) return invalid("top_groups must be in 1 .. groups");
    if (k > E / groups * top_groups) return invalid("k is more than the kept groups hold");
    if (!std::isfinite(scale)) return invalid("scale is not finite");
    if (T * k >= kMaxRows) return fail(SQ_ERR_UNSUPPORTED, "T k is 2^31 or more");
    if (ld < E) return invalid("the row stride of the logits is smaller than their row");
    return SQ_OK;
}

struct RouteWorkspace {
    size_t counts = 0, base = 0;
    size_t bytes() const { return counts + base; }
};
RouteWorkspace route_workspace(int64_t T, int64_t E) {
    RouteWorkspace w;
    const int64_t blocks = route_blocks(T);
    if (blocks <= 1) return w;
    w.counts = (size_t)round_up(blocks * route_stride(E), 256);
    w.base = (size_t)round_up((blocks + 1) * E * 4, 256);
    return w;
}

sq_status check_exchange(int32_t type, int64_t T, int64_t rows, int64_t D, int32_t k) {
    SQ_TRY(check_type(type));
    SQ_TRY(check_dim(T, kMaxRows, "T"));
    SQ_TRY(check_dim(rows, kMaxRows, "rows"));
    SQ_TRY(check_dim(D, kMaxCols, "D"));
    if (k < 1) return invalid("k must be positive");
    if (k > kExchangeMaxTopK) return fail(SQ_ERR_UNSUPPORTED, "more than 64 slots");
    if (T * k >= kMaxRows) return fail(SQ_ERR_UNSUPPORTED, "T k is 2^31 or more");
    return SQ_OK;
}

ExchangeArgs exchange_args(int32_t type, int64_t T, int64_t rows, int64_t D, int32_t k, const int32_t* place, const float* share) {
    ExchangeArgs a{};
    a.type = type;
    a.T = T;
    a.rows = rows;
    a.D = D;
    a.k = k;
    a.place = place;
    a.share = share;
    return a;
}

}  // namespace

extern "C" {

sq_status sq_norm_forward(const void* X, const void* residual, int32_t type, int64_t M, int64_t C, int64_t ld_x, int64_t ld_r,
                          const void* gamma, const void* beta, int32_t param_type, float eps, void* H, int64_t ld_h, void* Y,
                          int64_t ld_y, float* stats, void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_norm(type, param_type, M, C, gamma));
        if (!(eps >= 0.0f) || !std::isfinite(eps)) return invalid("eps must be finite and not negative");
        if (C > 0) SQ_TRY(check_values(beta, param_type, C, C, "beta"));
        if (M == 0 || C == 0) return SQ_OK;
        SQ_TRY(check_values(X, type, ld_x, C, "X"));
        SQ_TRY(check_values(Y, type, ld_y, C, "Y"));
        if ((residual == nullptr) != (H == nullptr)) return invalid("residual and H go together");
        if (residual) {
            SQ_TRY(check_values(residual, type, ld_r, C, "residual"));
            SQ_TRY(check_values(H, type, ld_h, C, "H"));
        }
        SQ_TRY(check_stats(stats));
        NormArgs a{};
        a.type = type;
        a.param_type = param_type;
        a.M = M;
        a.C = C;
        a.eps = eps;
        a.x = X;
        a.residual = residual;
        a.h = H;
        a.y = Y;
        a.gamma = gamma;
        a.beta = beta;
        a.stats = stats;
        a.ld_x = ld_x;
        a.ld_r = ld_r;
        a.ld_h = ld_h;
        a.ld_y = ld_y;
        return hip_status(launch_norm_forward(a, static_cast<hipStream_t>(stream)), "norm forward");
    });
}

sq_status sq_norm_backward_workspace_size(int64_t M, int64_t C, size_t* bytes) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_dim(M, kMaxRows, "M"));
        SQ_TRY(check_dim(C, kMaxCols, "C"));
        if (!bytes) return invalid("bytes is NULL");
        *bytes = (size_t)std::max(norm_parts(M, C, SQ_TYPE_F32), norm_parts(M, C, SQ_TYPE_BF16)) * 2 * C * 4;
        return SQ_OK;
    });
}

sq_status sq_norm_backward(const void* dY, const void* H, const void* dH, int32_t type, int64_t M, int64_t C, int64_t ld_dy,
                           int64_t ld_h, int64_t ld_dh, const void* gamma, int32_t param_type, const float* stats, void* dX,
                           int64_t ld_dx, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_norm(type, param_type, M, C, gamma));
        if (C == 0) return SQ_OK;
        SQ_TRY(check_words(dgamma, "dgamma"));
        SQ_TRY(check_words(dbeta, "dbeta"));
        if (M > 0) {
            SQ_TRY(check_values(dY, type, ld_dy, C, "dY"));
            SQ_TRY(check_values(H, type, ld_h, C, "H"));
            if (dH) SQ_TRY(check_values(dH, type, ld_dh, C, "dH"));
            SQ_TRY(check_values(dX, type, ld_dx, C, "dX"));
            if (!stats) return invalid("stats is NULL");
            SQ_TRY(check_stats(stats));
        }
        SQ_TRY(check_workspace(workspace, workspace_bytes, (size_t)norm_parts(M, C, type) * 2 * C * 4));
        NormArgs a{};
        a.type = type;
        a.param_type = param_type;
        a.M = M;
        a.C = C;
        a.x = H;
        a.dy = dY;
        a.dh = dH;
        a.gamma = gamma;
        a.stats = const_cast<float*>(stats);
        a.dx = dX;
        a.dgamma = dgamma;
        a.dbeta = dbeta;
        a.part = static_cast<float*>(workspace);
        a.ld_x = ld_h;
        a.ld_dy = ld_dy;
        a.ld_dh = ld_dh;
        a.ld_dx = ld_dx;
        return hip_status(launch_norm_backward(a, static_cast<hipStream_t>(stream)), "norm backward");
    });
}

// ---------------------------------------------------------------------------
sq_status sq_route_workspace_size(int64_t T, int64_t E, size_t* bytes) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_route_tokens(T));
        if (E < 1 || E > kRouteMaxExperts) return invalid("E must be in 1 .. 1024");
        if (!bytes) return invalid("bytes is NULL");
        *bytes = route_workspace(T, E).bytes();
        return SQ_OK;
    });
}

sq_status sq_route_forward(const void* logits, int32_t type, int64_t T, int64_t E, int64_t ld, const float* bias, int32_t score,
                           int32_t k, int32_t groups, int32_t top_groups, int32_t renormalize, float scale, float* share,
                           int32_t* chosen, int32_t* place, int32_t* offsets, void* workspace, size_t workspace_bytes,
                           void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_router(type, T, E, k, score, groups, top_groups, renormalize, scale, ld));
        SQ_TRY(check_words(offsets, "offsets"));
        if (bias) SQ_TRY(check_words(bias, "bias"));
        if (T > 0) {
            SQ_TRY(check_values(logits, type, ld, E, "logits"));
            SQ_TRY(check_words(share, "share"));
            SQ_TRY(check_words(chosen, "chosen"));
            SQ_TRY(check_words(place, "place"));
        }
        const RouteWorkspace w = route_workspace(T, E);
        SQ_TRY(check_workspace(workspace, workspace_bytes, w.bytes()));
        RouteArgs a{};
        a.type = type;
        a.score = score;
        a.renorm = renormalize;
        a.T = T;
        a.ld = ld;
        a.E = (int)E;
        a.k = k;
        a.groups = groups;
        a.top_groups = top_groups;
        a.scale = scale;
        a.logits = logits;
        a.bias = bias;
        a.share = share;
        a.chosen = chosen;
        a.place = place;
        a.offsets = offsets;
        a.counts = static_cast<uint8_t*>(workspace);
        a.base = reinterpret_cast<int32_t*>(a.counts + w.counts);
        return hip_status(launch_route_forward(a, static_cast<hipStream_t>(stream)), "route forward");
    });
}

sq_status sq_route_backward(const float* dshare, const void* logits, int32_t type, int64_t T, int64_t E, int64_t ld, int32_t score,
                            int32_t k, int32_t renormalize, float scale, const float* share, const int32_t* chosen, void* dlogits,
                            int64_t ld_d, void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_router(type, T, E, k, score, 1, 1, renormalize, scale, ld));
        if (T == 0) return SQ_OK;
        SQ_TRY(check_values(logits, type, ld, E, "logits"));
        SQ_TRY(check_values(dlogits, type, ld_d, E, "dlogits"));
        SQ_TRY(check_words(dshare, "dshare"));
        SQ_TRY(check_words(share, "share"));
        SQ_TRY(check_words(chosen, "chosen"));
        RouteArgs a{};
        a.type = type;
        a.score = score;
        a.renorm = renormalize;
        a.T = T;
        a.ld = ld;
        a.E = (int)E;
        a.k = k;
        a.scale = scale;
        a.logits = logits;
        a.share = const_cast<float*>(share);
        a.chosen = const_cast<int32_t*>(chosen);
        a.dshare = dshare;
        a.dlogits = dlogits;
        a.ld_d = ld_d;
        return hip_status(launch_route_backward(a, static_cast<hipStream_t>(stream)), "route backward");
    });
}

// ---------------------------------------------------------------------------
sq_status sq_exchange_dispatch(const void* X, int32_t type, int64_t T, int64_t D, int64_t ld_x, const int32_t* place, int32_t k,
                               void* R, int64_t rows, int64_t ld_r, void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_exchange(type, T, rows, D, k));
        if (T == 0 || D == 0 || rows == 0) return SQ_OK;
        SQ_TRY(check_values(X, type, ld_x, D, "X"));
        SQ_TRY(check_values(R, type, ld_r, D, "R"));
        SQ_TRY(check_words(place, "place"));
        ExchangeArgs a = exchange_args(type, T, rows, D, k, place, nullptr);
        a.x = X;
        a.ld_x = ld_x;
        a.rows_out = R;
        a.ld_rows = ld_r;
        return hip_status(launch_dispatch(a, static_cast<hipStream_t>(stream)), "dispatch");
    });
}

sq_status sq_exchange_combine(const void* R, int32_t type, int64_t rows, int64_t D, int64_t ld_r, const int32_t* place,
                              const float* share, int64_t T, int32_t k, const void* add, int64_t ld_add, void* out,
                              int64_t ld_out, void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_exchange(type, T, rows, D, k));
        if (T == 0 || D == 0) return SQ_OK;
        if (rows > 0) SQ_TRY(check_values(R, type, ld_r, D, "R"));
        if (add) SQ_TRY(check_values(add, type, ld_add, D, "add"));
        SQ_TRY(check_values(out, type, ld_out, D, "out"));
        SQ_TRY(check_words(place, "place"));
        if (share) SQ_TRY(check_words(share, "share"));
        ExchangeArgs a = exchange_args(type, T, rows, D, k, place, share);
        a.rows_in = R;
        a.ld_in = ld_r;
        a.add = add;
        a.ld_add = ld_add;
        a.out = out;
        a.ld_out = ld_out;
        return hip_status(launch_combine(a, static_cast<hipStream_t>(stream)), "combine");
    });
}

sq_status sq_exchange_combine_backward(const void* dout, const void* R, int32_t type, int64_t rows, int64_t D, int64_t ld_dout,
                                       int64_t ld_r, const int32_t* place, const float* share, int64_t T, int32_t k, void* dR,
                                       int64_t ld_dr, float* dshare, void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_exchange(type, T, rows, D, k));
        if (T == 0) return SQ_OK;
        if (D > 0) {
            SQ_TRY(check_values(dout, type, ld_dout, D, "dout"));
            if (rows > 0) {
                SQ_TRY(check_values(R, type, ld_r, D, "R"));
                SQ_TRY(check_values(dR, type, ld_dr, D, "dR"));
            }
        }
        SQ_TRY(check_words(place, "place"));
        SQ_TRY(check_words(share, "share"));
        SQ_TRY(check_words(dshare, "dshare"));
        ExchangeArgs a = exchange_args(type, T, rows, D, k, place, share);
        a.x = dout;
        a.ld_x = ld_dout;
        a.rows_in = R;
        a.ld_in = ld_r;
        a.rows_out = dR;
        a.ld_rows = ld_dr;
        a.dshare = dshare;
        return hip_status(launch_combine_backward(a, static_cast<hipStream_t>(stream)), "combine backward");
    });
}

}  // extern "C"
