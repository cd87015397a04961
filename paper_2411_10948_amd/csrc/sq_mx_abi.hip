// extern "C" entry points of the microscaled 4-bit path and of the activations
// with 8-bit checkpoints: synchronous argument checks, then the launches.  The
// semantics of every call are documented in include/shiftquant.h.
#include <algorithm>
#include <cstdint>
#include <string>

#include "sq_checks.h"
#include "sq_mx.h"

namespace {

using namespace sq;

sq_status check_experts(const int32_t* offsets, int64_t experts) {
    if (experts < 1 || experts >= kMaxExperts) return invalid("experts is out of range");
    if (!offsets || !aligned(offsets, 4)) return invalid("offsets is NULL or misaligned");
    return SQ_OK;
}

// the inner axis of a transpose by expert: whole units for each, twice as long at most
sq_status check_segments(int64_t rows, int64_t experts) {
    SQ_TRY(check_inner(rows));
    if (mx_segment_cols(rows, experts) >= 2 * kMaxInner)
        return fail(SQ_ERR_UNSUPPORTED, "the experts' rows, each rounded up to 512, are 2^24 or more");
    return SQ_OK;
}

size_t part_bytes(const MxGemmArgs& a) {
    const int64_t s = mx_gemm_splits(a);
    return s > 1 ? (size_t)round_up(s * a.M * a.N * 4, 256) : 0;
}

// codes and scales of X between the quantizer and the product
struct LinearWorkspace {
    size_t codes = 0, scales = 0, part = 0;
    size_t bytes() const { return codes + scales + part; }
};
LinearWorkspace linear_workspace(int64_t M, int64_t K, int64_t N, int64_t experts, int type) {
    LinearWorkspace w;
    if (M == 0 || N == 0 || mx_rows_ok(M, K, N, experts, type)) return w;
    w.codes = (size_t)round_up(mx_code_bytes(M, K), 256);
    w.scales = (size_t)round_up(mx_scale_bytes(M, K), 256);
    MxGemmArgs a{};
    a.mode = experts ? kExpertRows : kDense;
    a.M = M;
    a.N = N;
    a.K = K;
    a.experts = (int)experts;
    w.part = part_bytes(a);
    return w;
}

sq_status check_product(int64_t M, int64_t N, int64_t K, int64_t experts) {
    SQ_TRY(check_dim(M, kMaxRows, "M"));
    SQ_TRY(check_dim(N, kMaxCols, "N"));
    SQ_TRY(check_dim(K, kMaxRows, "K"));
    SQ_TRY(check_inner(K));
    return check_blocks(M, 16, N, 16, experts, 1);
}

// of a product whose A is quantized on the way: K is the columns of its values too
sq_status check_linear(int64_t M, int64_t N, int64_t K, int64_t experts) {
    SQ_TRY(check_product(M, N, K, experts));
    return M == 0 || N == 0 ? SQ_OK : check_dim(K, kMaxCols, "K");
}

MxGemmArgs dense_args(int64_t M, int64_t N, int64_t K) {
    MxGemmArgs a{};
    a.mode = kDense;
    a.M = M;
    a.N = N;
    a.K = K;
    return a;
}

// sq_mx_quantize, with a copy of the offsets in `keep` (may be NULL)
sq_status quantize(const void* X, int32_t type, int64_t batch, int64_t rows, int64_t cols, int64_t ld, int64_t stride,
                   const int32_t* offsets, int64_t experts, uint8_t* codes, uint8_t* scales, uint8_t* codes_t,
                   uint8_t* scales_t, int32_t* keep, void* stream) {
    SQ_TRY(check_type(type));
    SQ_TRY(check_dim(batch, 65536, "batch"));
    SQ_TRY(check_dim(rows, kMaxRows, "rows"));
    SQ_TRY(check_dim(cols, kMaxCols, "cols"));
    if (offsets || experts) {
        SQ_TRY(check_experts(offsets, experts));
        if (batch != 1) return invalid("offsets split the rows of one matrix: batch must be 1");
    }
    if (batch == 0 || rows == 0 || cols == 0) return SQ_OK;
    if (!codes && !codes_t) return invalid("codes and codes_t are both NULL");
    if (codes || scales) SQ_TRY(check_mx(codes, scales, "codes"));
    if (codes_t || scales_t) {
        SQ_TRY(check_mx(codes_t, scales_t, "codes_t"));
        SQ_TRY(experts ? check_segments(rows, experts) : check_inner(rows));
    }
    SQ_TRY(check_values(X, type, ld, cols, "X"));
    if (batch > 1 && (stride < 0 || stride < (rows - 1) * ld + cols)) return invalid("stride is smaller than a matrix");
    SQ_TRY(check_blocks(rows, 128, cols, 64, experts, 2));
    MxQuantArgs a{};
    a.x = X;
    a.type = type;
    a.batch = batch;
    a.rows = rows;
    a.cols = cols;
    a.ld = ld;
    a.stride = stride;
    a.offsets = offsets;
    a.experts = (int)experts;
    a.codes = codes;
    a.scales = scales;
    a.codes_t = codes_t;
    a.scales_t = scales_t;
    a.cap_t = offsets ? mx_segment_cols(rows, experts) : mx_units(rows) * kMxUnit;
    a.keep = keep;
    return hip_status(launch_mx_quantize(a, static_cast<hipStream_t>(stream)), "mx quantize");
}

}  // namespace

extern "C" {

sq_status sq_mx_size(int64_t rows, int64_t cols, size_t* code_bytes, size_t* scale_bytes) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_dim(rows, kMaxRows, "rows"));
        SQ_TRY(check_dim(cols, kMaxRows, "cols"));
        if (!code_bytes || !scale_bytes) return invalid("a size output is NULL");
        *code_bytes = (size_t)mx_code_bytes(rows, cols);
        *scale_bytes = (size_t)mx_scale_bytes(rows, cols);
        return SQ_OK;
    });
}

sq_status sq_mx_segment_cols(int64_t rows, int64_t experts, int64_t* cols) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_dim(rows, kMaxRows, "rows"));
        if (experts < 1 || experts >= kMaxExperts) return invalid("experts is out of range");
        if (!cols) return invalid("cols is NULL");
        *cols = mx_segment_cols(rows, experts);
        return SQ_OK;
    });
}

sq_status sq_mx_quantize(const void* X, int32_t type, int64_t batch, int64_t rows, int64_t cols, int64_t ld, int64_t stride,
                         const int32_t* offsets, int64_t experts, uint8_t* codes, uint8_t* scales, uint8_t* codes_t,
                         uint8_t* scales_t, void* stream) {
    return guarded([&]() -> sq_status {
        return quantize(X, type, batch, rows, cols, ld, stride, offsets, experts, codes, scales, codes_t, scales_t, nullptr,
                        stream);
    });
}

sq_status sq_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* out, int32_t type,
                           int64_t ld, void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_type(type));
        SQ_TRY(check_dim(rows, kMaxRows, "rows"));
        SQ_TRY(check_dim(cols, kMaxRows, "cols"));
        if (rows == 0 || cols == 0) return SQ_OK;
        SQ_TRY(check_mx(codes, scales, "codes"));
        SQ_TRY(check_values(out, type, ld, cols, "out"));
        SQ_TRY(check_blocks(rows, 1, cols, 32 * 256, 0, 1));
        return hip_status(launch_mx_dequantize(codes, scales, rows, cols, out, type, ld, static_cast<hipStream_t>(stream)),
                          "mx dequantize");
    });
}

sq_status sq_mx_gemm_workspace_size(int64_t M, int64_t N, int64_t K, size_t* bytes) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_product(M, N, K, 0));
        if (!bytes) return invalid("bytes is NULL");
        *bytes = M == 0 || N == 0 ? 0 : part_bytes(dense_args(M, N, K));
        return SQ_OK;
    });
}

sq_status sq_mx_gemm(const uint8_t* A, const uint8_t* A_scales, const uint8_t* B, const uint8_t* B_scales, int64_t M,
                     int64_t N, int64_t K, void* C, int32_t type, int64_t ldc, void* workspace, size_t workspace_bytes,
                     void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_type(type));
        SQ_TRY(check_product(M, N, K, 0));
        if (M == 0 || N == 0) return SQ_OK;
        if (K > 0) {
            SQ_TRY(check_mx(A, A_scales, "A"));
            SQ_TRY(check_mx(B, B_scales, "B"));
        }
        SQ_TRY(check_values(C, type, ldc, N, "C"));
        MxGemmArgs a = dense_args(M, N, K);
        SQ_TRY(check_workspace(workspace, workspace_bytes, part_bytes(a)));
        a.A = A;
        a.As = A_scales;
        a.B = B;
        a.Bs = B_scales;
        a.C = C;
        a.type = type;
        a.ldc = ldc;
        a.part = static_cast<float*>(workspace);
        return hip_status(launch_mx_gemm(a, static_cast<hipStream_t>(stream)), "mx gemm");
    });
}

sq_status sq_mx_gemm_experts(const uint8_t* A, const uint8_t* A_scales, int64_t M, int64_t K, const int32_t* offsets,
                             int64_t experts, const uint8_t* B, const uint8_t* B_scales, int64_t N, void* C, int32_t type,
                             int64_t ldc, void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_type(type));
        SQ_TRY(check_experts(offsets, experts));
        SQ_TRY(check_product(M, N, K, experts));
        if (M == 0 || N == 0) return SQ_OK;
        if (K > 0) {
            SQ_TRY(check_mx(A, A_scales, "A"));
            SQ_TRY(check_mx(B, B_scales, "B"));
        }
        SQ_TRY(check_values(C, type, ldc, N, "C"));
        MxGemmArgs a = dense_args(M, N, K);
        a.mode = kExpertRows;
        a.A = A;
        a.As = A_scales;
        a.B = B;
        a.Bs = B_scales;
        a.offsets = offsets;
        a.experts = (int)experts;
        a.C = C;
        a.type = type;
        a.ldc = ldc;
        return hip_status(launch_mx_gemm(a, static_cast<hipStream_t>(stream)), "mx gemm by expert");
    });
}

sq_status sq_mx_gemm_experts_wgrad_workspace_size(int64_t rows, int64_t experts, int64_t M, int64_t N, size_t* bytes) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_dim(rows, kMaxRows, "rows"));
        if (experts < 1 || experts >= kMaxExperts) return invalid("experts is out of range");
        SQ_TRY(check_segments(rows, experts));
        SQ_TRY(check_dim(M, kMaxCols, "M"));
        SQ_TRY(check_dim(N, kMaxCols, "N"));
        if (!bytes) return invalid("bytes is NULL");
        *bytes = 0;
        return SQ_OK;
    });
}

sq_status sq_mx_gemm_experts_wgrad(const uint8_t* A, const uint8_t* A_scales, const uint8_t* B, const uint8_t* B_scales,
                                   int64_t rows, const int32_t* offsets, int64_t experts, int64_t M, int64_t N, void* C,
                                   int32_t type, int64_t ldc, void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&]() -> sq_status {
        size_t need = 0;
        SQ_TRY(check_type(type));
        SQ_TRY(check_experts(offsets, experts));
        SQ_TRY(sq_mx_gemm_experts_wgrad_workspace_size(rows, experts, M, N, &need));
        SQ_TRY(check_blocks(M, 16, N, 16, 0, experts));
        if (M == 0 || N == 0) return SQ_OK;
        if (rows > 0) {
            SQ_TRY(check_mx(A, A_scales, "A"));
            SQ_TRY(check_mx(B, B_scales, "B"));
        }
        SQ_TRY(check_values(C, type, ldc, N, "C"));
        SQ_TRY(check_workspace(workspace, workspace_bytes, need));
        MxGemmArgs a = dense_args(M, N, mx_segment_cols(rows, experts));
        a.mode = kExpertInner;
        a.A = A;
        a.As = A_scales;
        a.B = B;
        a.Bs = B_scales;
        a.offsets = offsets;
        a.experts = (int)experts;
        a.rows = rows;
        a.C = C;
        a.type = type;
        a.ldc = ldc;
        return hip_status(launch_mx_gemm(a, static_cast<hipStream_t>(stream)), "mx weight gradient by expert");
    });
}

sq_status sq_mx_linear_workspace_size(int64_t M, int64_t K, int64_t N, int64_t experts, size_t* bytes) {
    return guarded([&]() -> sq_status {
        if (experts < 0 || experts >= kMaxExperts) return invalid("experts is out of range");
        SQ_TRY(check_linear(M, N, K, experts));
        if (!bytes) return invalid("bytes is NULL");
        *bytes = std::max(linear_workspace(M, K, N, experts, SQ_TYPE_F32).bytes(),
                          linear_workspace(M, K, N, experts, SQ_TYPE_BF16).bytes());
        return SQ_OK;
    });
}

sq_status sq_mx_linear(const void* X, int32_t type, int64_t M, int64_t K, int64_t ld, const int32_t* offsets, int64_t experts,
                       const uint8_t* W, const uint8_t* W_scales, int64_t N, void* Y, int32_t out_type, int64_t ldy,
                       void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_type(type));
        SQ_TRY(check_type(out_type));
        if (offsets || experts) SQ_TRY(check_experts(offsets, experts));
        SQ_TRY(check_linear(M, N, K, experts));
        if (M == 0 || N == 0) return SQ_OK;
        if (K > 0) {
            SQ_TRY(check_values(X, type, ld, K, "X"));
            SQ_TRY(check_mx(W, W_scales, "W"));
        }
        SQ_TRY(check_values(Y, out_type, ldy, N, "Y"));
        const LinearWorkspace w = linear_workspace(M, K, N, experts, type);
        SQ_TRY(check_workspace(workspace, workspace_bytes, w.bytes()));
        hipStream_t s = static_cast<hipStream_t>(stream);
        if (mx_rows_ok(M, K, N, experts, type)) {
            MxRowsArgs r{};
            r.x = X;
            r.type = type;
            r.M = M;
            r.K = K;
            r.ld = ld;
            r.W = W;
            r.Ws = W_scales;
            r.N = N;
            r.offsets = offsets;
            r.experts = (int)experts;
            r.Y = Y;
            r.out_type = out_type;
            r.ldy = ldy;
            return hip_status(launch_mx_rows(r, s), "mx linear");
        }
        uint8_t* codes = static_cast<uint8_t*>(workspace);
        uint8_t* scales = codes + w.codes;
        SQ_TRY(sq_mx_quantize(X, type, 1, M, K, ld, 0, offsets, experts, codes, scales, nullptr, nullptr, stream));
        if (experts)
            return sq_mx_gemm_experts(codes, scales, M, K, offsets, experts, W, W_scales, N, Y, out_type, ldy, stream);
        return sq_mx_gemm(codes, scales, W, W_scales, M, N, K, Y, out_type, ldy, scales + w.scales, w.part, stream);
    });
}

// ---------------------------------------------------------------------------
static sq_status check_layer(const sq_mx_layer* l) {
    if (!l) return invalid("layer is NULL");
    SQ_TRY(check_type(l->type));
    if (l->experts < 0 || l->experts >= kMaxExperts) return invalid("experts is out of range");
    SQ_TRY(check_dim(l->rows, kMaxRows, "rows"));
    SQ_TRY(check_dim(l->c_in, kMaxCols, "c_in"));
    SQ_TRY(check_dim(l->c_out, kMaxCols, "c_out"));
    return l->experts ? check_segments(l->rows, l->experts) : check_inner(l->rows);
}

static sq_status check_layer_offsets(const sq_mx_layer* l, const int32_t* offsets) {
    if (l->experts) return check_experts(offsets, l->experts);
    if (offsets) return invalid("offsets without experts");
    return SQ_OK;
}

// the products dX [rows, c_in] = dY W and dW [c_out, c_in] = dY^T X, their K splits' partials one after the other
static void backward_args(const sq_mx_layer* l, MxGemmArgs& x, MxGemmArgs& w) {
    x = dense_args(l->rows, l->c_in, l->c_out);
    x.mode = l->experts ? kExpertRows : kDense;
    x.experts = (int)l->experts;
    w = dense_args(l->c_out, l->c_in, l->experts ? mx_segment_cols(l->rows, l->experts) : l->rows);
    w.mode = l->experts ? kExpertInner : kDense;
    w.experts = (int)l->experts;
    w.rows = l->rows;
}

static size_t layer_workspace(const sq_mx_layer* l) {
    if (l->experts || l->c_in == 0 || l->c_out == 0) return 0;
    MxGemmArgs x, w;
    backward_args(l, x, w);
    return std::max(l->rows ? part_bytes(dense_args(l->rows, l->c_out, l->c_in)) : 0,
                    (l->rows ? part_bytes(x) : 0) + part_bytes(w));
}

sq_status sq_mx_layer_workspace_size(const sq_mx_layer* layer, size_t* bytes) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_layer(layer));
        if (!bytes) return invalid("bytes is NULL");
        *bytes = layer_workspace(layer);
        return SQ_OK;
    });
}

sq_status sq_mx_layer_weight(const sq_mx_layer* layer, const void* W, int64_t ld, int64_t stride, void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_layer(layer));
        const sq_mx_layer& l = *layer;
        return sq_mx_quantize(W, l.type, l.experts ? l.experts : 1, l.c_out, l.c_in, ld, stride, nullptr, 0, l.w, l.w_scales,
                              l.w_t, l.w_t_scales, stream);
    });
}

sq_status sq_mx_layer_forward(const sq_mx_layer* layer, const void* X, int64_t ld, const int32_t* offsets, void* Y, int64_t ldy,
                              void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_layer(layer));
        const sq_mx_layer& l = *layer;
        SQ_TRY(check_layer_offsets(layer, offsets));
        if (l.experts && l.offsets && !aligned(l.offsets, 4)) return invalid("the layer's offsets are misaligned");
        SQ_TRY(check_product(l.rows, l.c_out, l.c_in, l.experts));
        if (l.rows > 0 && l.c_out > 0) {
            SQ_TRY(check_values(Y, l.type, ldy, l.c_out, "Y"));
            if (l.c_in > 0) {
                SQ_TRY(check_mx(l.w, l.w_scales, "w"));
                SQ_TRY(check_mx(l.x, l.x_scales, "x"));
            }
        }
        SQ_TRY(check_workspace(l.workspace, l.workspace_bytes, layer_workspace(layer)));
        // No offsets are kept where there is nothing to quantize: no result of the backward depends on them then.
        SQ_TRY(quantize(X, l.type, 1, l.rows, l.c_in, ld, 0, offsets, l.experts, l.x, l.x_scales, l.x_t, l.x_t_scales,
                        l.experts ? l.offsets : nullptr, stream));
        if (l.experts)
            return sq_mx_gemm_experts(l.x, l.x_scales, l.rows, l.c_in, offsets, l.experts, l.w, l.w_scales, l.c_out, Y, l.type,
                                      ldy, stream);
        return sq_mx_gemm(l.x, l.x_scales, l.w, l.w_scales, l.rows, l.c_out, l.c_in, Y, l.type, ldy, l.workspace,
                          l.workspace_bytes, stream);
    });
}

sq_status sq_mx_layer_backward(const sq_mx_layer* layer, const void* dY, int64_t ld, const int32_t* offsets, void* dX,
                               int64_t ld_dx, float* dW, int64_t ld_dw, void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_layer(layer));
        const sq_mx_layer& l = *layer;
        if (!offsets && l.experts) offsets = l.offsets;
        SQ_TRY(check_layer_offsets(layer, offsets));
        SQ_TRY(check_product(l.rows, l.c_in, l.c_out, l.experts));
        SQ_TRY(check_blocks(l.c_out, 16, l.c_in, 16, 0, std::max<int64_t>(l.experts, 1)));
        if (l.rows > 0 && l.c_in > 0) {
            SQ_TRY(check_values(dX, l.type, ld_dx, l.c_in, "dX"));
            if (l.c_out > 0) {
                SQ_TRY(check_mx(l.w_t, l.w_t_scales, "w_t"));
                SQ_TRY(check_mx(l.dy, l.dy_scales, "dy"));
            }
        }
        if (l.c_out > 0 && l.c_in > 0) {
            SQ_TRY(check_values(dW, SQ_TYPE_F32, ld_dw, l.c_in, "dW"));
            if (l.rows > 0) {
                SQ_TRY(check_mx(l.x_t, l.x_t_scales, "x_t"));
                SQ_TRY(check_mx(l.dy_t, l.dy_t_scales, "dy_t"));
            }
        }
        SQ_TRY(check_workspace(l.workspace, l.workspace_bytes, layer_workspace(layer)));
        SQ_TRY(sq_mx_quantize(dY, l.type, 1, l.rows, l.c_out, ld, 0, offsets, l.experts, l.dy, l.dy_scales, l.dy_t,
                              l.dy_t_scales, stream));
        MxGemmArgs x, w;
        backward_args(layer, x, w);
        x.A = l.dy;
        x.As = l.dy_scales;
        x.B = l.w_t;
        x.Bs = l.w_t_scales;
        x.offsets = offsets;
        x.C = dX;
        x.type = l.type;
        x.ldc = ld_dx;
        x.part = static_cast<float*>(l.workspace);
        w.A = l.dy_t;
        w.As = l.dy_t_scales;
        w.B = l.x_t;
        w.Bs = l.x_t_scales;
        w.offsets = offsets;
        w.C = dW;
        w.type = SQ_TYPE_F32;
        w.ldc = ld_dw;
        w.part = x.part + (l.experts || l.rows == 0 ? 0 : part_bytes(x) / sizeof(float));
        return hip_status(launch_mx_gemm_pair(x, w, static_cast<hipStream_t>(stream)), "mx gradients");
    });
}

// ---------------------------------------------------------------------------
static sq_status check_act(int32_t type, int32_t kind, int32_t gated, int64_t M, int64_t F, int64_t ld_x, int64_t ld_h) {
    SQ_TRY(check_type(type));
    if (kind != SQ_ACT_SILU && kind != SQ_ACT_GELU) return invalid("kind must be SQ_ACT_SILU or SQ_ACT_GELU");
    if (gated != 0 && gated != 1) return invalid("gated must be 0 or 1");
    SQ_TRY(check_dim(M, kMaxRows, "M"));
    SQ_TRY(check_dim(F, kMaxCols, "F"));
    if (M == 0 || F == 0) return SQ_OK;
    if (ld_x < F * (gated ? 2 : 1)) return invalid("the row stride of X or dX is smaller than its row");
    if (ld_h < F) return invalid("the row stride of H or dH is smaller than its row");
    return SQ_OK;
}

static sq_status check_copy(const int8_t* codes, const uint8_t* scales) {
    if (!codes || !scales) return invalid("codes or scales are NULL");
    if (!aligned(codes, 16)) return invalid("codes must be 16-byte aligned");
    return SQ_OK;
}

sq_status sq_act_size(int64_t M, int64_t F, int32_t gated, size_t* code_bytes, size_t* scale_bytes) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_dim(M, kMaxRows, "M"));
        SQ_TRY(check_dim(F, kMaxCols, "F"));
        if (gated != 0 && gated != 1) return invalid("gated must be 0 or 1");
        if (!code_bytes || !scale_bytes) return invalid("a size output is NULL");
        *code_bytes = (size_t)(M * round_up(F, 32) * (gated ? 2 : 1));
        *scale_bytes = *code_bytes / 32;
        return SQ_OK;
    });
}

sq_status sq_act_forward(const void* X, int32_t type, int32_t kind, int32_t gated, int64_t M, int64_t F, int64_t ld_x, void* H,
                         int64_t ld_h, int8_t* codes, uint8_t* scales, void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_act(type, kind, gated, M, F, ld_x, ld_h));
        if (M == 0 || F == 0) return SQ_OK;
        SQ_TRY(check_values(X, type, ld_x, F, "X"));
        SQ_TRY(check_values(H, type, ld_h, F, "H"));
        SQ_TRY(check_copy(codes, scales));
        ActArgs a{};
        a.kind = kind;
        a.gated = gated;
        a.type = type;
        a.M = M;
        a.F = F;
        a.ld_x = ld_x;
        a.ld_h = ld_h;
        a.x = X;
        a.h = H;
        a.codes = codes;
        a.scales = scales;
        return hip_status(launch_act_forward(a, static_cast<hipStream_t>(stream)), "activation forward");
    });
}

sq_status sq_act_backward(const void* dH, int32_t type, int32_t kind, int32_t gated, int64_t M, int64_t F, int64_t ld_h,
                          const int8_t* codes, const uint8_t* scales, void* dX, int64_t ld_x, void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_act(type, kind, gated, M, F, ld_x, ld_h));
        if (M == 0 || F == 0) return SQ_OK;
        SQ_TRY(check_values(dH, type, ld_h, F, "dH"));
        SQ_TRY(check_values(dX, type, ld_x, F, "dX"));
        SQ_TRY(check_copy(codes, scales));
        ActArgs a{};
        a.kind = kind;
        a.gated = gated;
        a.type = type;
        a.M = M;
        a.F = F;
        a.ld_x = ld_x;
        a.ld_h = ld_h;
        a.h = const_cast<void*>(dH);
        a.dx = dX;
        a.codes = const_cast<int8_t*>(codes);
        a.scales = const_cast<uint8_t*>(scales);
        return hip_status(launch_act_backward(a, static_cast<hipStream_t>(stream)), "activation backward");
    });
}

}  // extern "C"
