// extern "C" entry points of the dense layers in 8-bit floating point: synchronous
// argument checks, then the launches.  The semantics of every call are documented
// in include/shiftquant.h.
#include <algorithm>
#include <cstdint>
#include <string>

#include "sq_checks.h"
#include "sq_f8.h"

namespace {

using namespace sq;

constexpr int64_t kF8MaxInner = (int64_t)1 << 22;   // a tile's 16 groups, 16 bytes an element, in 30 bits

sq_status check_f8_inner(int64_t k) {
    if (k >= kF8MaxInner) return fail(SQ_ERR_UNSUPPORTED, "the inner axis has 2^22 elements or more");
    return SQ_OK;
}

size_t f8_part_bytes(int64_t M, int64_t N, int64_t K, int32_t type) {
    const int64_t s = M && N ? f8_gemm_splits(M, N, K, type) : 1;
    return s > 1 ? (size_t)round_up(s * M * N * 4, 256) : 0;
}

sq_status check_f8_product(int64_t M, int64_t N, int64_t K) {
    SQ_TRY(check_dim(M, kMaxRows, "M"));
    SQ_TRY(check_dim(N, kMaxRows, "N"));
    SQ_TRY(check_dim(K, kMaxRows, "K"));
    SQ_TRY(check_f8_inner(K));
    return check_blocks(M, 64, N, 64, 0, 256);
}

// of a product whose A is quantized on the way: N and K are columns of values too
sq_status check_f8_linear(int64_t M, int64_t N, int64_t K) {
    SQ_TRY(check_f8_product(M, N, K));
    SQ_TRY(check_dim(N, kMaxCols, "N"));
    return M == 0 || N == 0 ? SQ_OK : check_dim(K, kMaxCols, "K");
}

// codes and scales of X between the quantizer and the product
struct F8Workspace {
    size_t codes = 0, scales = 0, part = 0;
    size_t bytes() const { return codes + scales + part; }
};
F8Workspace f8_workspace(int64_t M, int64_t K, int64_t N, int32_t type, int32_t out_type) {
    F8Workspace w;
    if (M == 0 || N == 0 || f8_rows_ok(M, K, N, type)) return w;
    w.codes = (size_t)round_up(f8_code_bytes(M, K), 256);
    w.scales = (size_t)round_up(f8_scale_bytes(M, K), 256);
    w.part = f8_part_bytes(M, N, K, out_type);
    return w;
}

F8GemmArgs product_args(const uint8_t* A, const uint8_t* As, const uint8_t* B, const uint8_t* Bs, int64_t M, int64_t N, int64_t K,
                        void* C, int32_t type, int64_t ldc, void* part) {
    F8GemmArgs a{};
    a.M = M;
    a.N = N;
    a.K = K;
    a.A = A;
    a.As = As;
    a.B = B;
    a.Bs = Bs;
    a.C = C;
    a.type = type;
    a.ldc = ldc;
    a.part = static_cast<float*>(part);
    return a;
}

sq_status check_f8_layer(const sq_f8_layer* l) {
    if (!l) return invalid("layer is NULL");
    SQ_TRY(check_type(l->type));
    SQ_TRY(check_dim(l->rows, kMaxRows, "rows"));
    SQ_TRY(check_dim(l->c_in, kMaxCols, "c_in"));
    SQ_TRY(check_dim(l->c_out, kMaxCols, "c_out"));
    return check_f8_inner(l->rows);
}

size_t f8_layer_workspace(const sq_f8_layer* l) {
    return std::max(f8_part_bytes(l->rows, l->c_out, l->c_in, l->type),
                    f8_part_bytes(l->rows, l->c_in, l->c_out, l->type) + f8_part_bytes(l->c_out, l->c_in, l->rows, SQ_TYPE_F32));
}

}  // namespace

extern "C" {

sq_status sq_f8_size(int64_t rows, int64_t cols, size_t* code_bytes, size_t* scale_bytes) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_dim(rows, kMaxRows, "rows"));
        SQ_TRY(check_dim(cols, kMaxRows, "cols"));
        if (!code_bytes || !scale_bytes) return invalid("a size output is NULL");
        *code_bytes = (size_t)f8_code_bytes(rows, cols);
        *scale_bytes = (size_t)f8_scale_bytes(rows, cols);
        return SQ_OK;
    });
}

sq_status sq_f8_quantize(const void* X, int32_t type, int64_t rows, int64_t cols, int64_t ld, int32_t square, uint8_t* codes,
                         uint8_t* scales, uint8_t* codes_t, uint8_t* scales_t, void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_type(type));
        SQ_TRY(check_dim(rows, kMaxRows, "rows"));
        SQ_TRY(check_dim(cols, kMaxCols, "cols"));
        if (square != 0 && square != 1) return invalid("square must be 0 or 1");
        if (rows == 0 || cols == 0) return SQ_OK;
        if (!codes && !codes_t) return invalid("codes and codes_t are both NULL");
        if (codes || scales) SQ_TRY(check_mx(codes, scales, "codes"));
        if (codes_t || scales_t) {
            SQ_TRY(check_mx(codes_t, scales_t, "codes_t"));
            SQ_TRY(check_f8_inner(rows));
        }
        SQ_TRY(check_values(X, type, ld, cols, "X"));
        SQ_TRY(check_blocks(rows, 128, cols, 128, 0, 512));
        F8QuantArgs a{};
        a.x = X;
        a.type = type;
        a.rows = rows;
        a.cols = cols;
        a.ld = ld;
        a.square = square;
        a.codes = codes;
        a.scales = scales;
        a.codes_t = codes_t;
        a.scales_t = scales_t;
        return hip_status(launch_f8_quantize(a, static_cast<hipStream_t>(stream)), "f8 quantize");
    });
}

sq_status sq_f8_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* out, int32_t type,
                           int64_t ld, void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_type(type));
        SQ_TRY(check_dim(rows, kMaxRows, "rows"));
        SQ_TRY(check_dim(cols, kMaxRows, "cols"));
        if (rows == 0 || cols == 0) return SQ_OK;
        SQ_TRY(check_mx(codes, scales, "codes"));
        SQ_TRY(check_values(out, type, ld, cols, "out"));
        SQ_TRY(check_blocks(rows, 1, cols, 16, 0, 1));
        return hip_status(launch_f8_dequantize(codes, scales, rows, cols, out, type, ld, static_cast<hipStream_t>(stream)),
                          "f8 dequantize");
    });
}

sq_status sq_f8_gemm_workspace_size(int64_t M, int64_t N, int64_t K, size_t* bytes) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_f8_product(M, N, K));
        if (!bytes) return invalid("bytes is NULL");
        *bytes = std::max(f8_part_bytes(M, N, K, SQ_TYPE_F32), f8_part_bytes(M, N, K, SQ_TYPE_BF16));
        return SQ_OK;
    });
}

sq_status sq_f8_gemm(const uint8_t* A, const uint8_t* A_scales, const uint8_t* B, const uint8_t* B_scales, int64_t M, int64_t N,
                     int64_t K, void* C, int32_t type, int64_t ldc, void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_type(type));
        SQ_TRY(check_f8_product(M, N, K));
        if (M == 0 || N == 0) return SQ_OK;
        if (K > 0) {
            SQ_TRY(check_mx(A, A_scales, "A"));
            SQ_TRY(check_mx(B, B_scales, "B"));
        }
        SQ_TRY(check_values(C, type, ldc, N, "C"));
        SQ_TRY(check_workspace(workspace, workspace_bytes, f8_part_bytes(M, N, K, type)));
        return hip_status(launch_f8_gemm(product_args(A, A_scales, B, B_scales, M, N, K, C, type, ldc, workspace),
                                         static_cast<hipStream_t>(stream)), "f8 gemm");
    });
}

sq_status sq_f8_linear_workspace_size(int64_t M, int64_t K, int64_t N, size_t* bytes) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_f8_linear(M, N, K));
        if (!bytes) return invalid("bytes is NULL");
        *bytes = 0;
        for (const int32_t type : {SQ_TYPE_F32, SQ_TYPE_BF16})
            for (const int32_t out_type : {SQ_TYPE_F32, SQ_TYPE_BF16})
                *bytes = std::max(*bytes, f8_workspace(M, K, N, type, out_type).bytes());
        return SQ_OK;
    });
}

sq_status sq_f8_linear(const void* X, int32_t type, int64_t M, int64_t K, int64_t ld, const uint8_t* W, const uint8_t* W_scales,
                       int64_t N, void* Y, int32_t out_type, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_type(type));
        SQ_TRY(check_type(out_type));
        SQ_TRY(check_f8_linear(M, N, K));
        if (M == 0 || N == 0) return SQ_OK;
        if (K > 0) {
            SQ_TRY(check_values(X, type, ld, K, "X"));
            SQ_TRY(check_mx(W, W_scales, "W"));
        }
        SQ_TRY(check_values(Y, out_type, ldy, N, "Y"));
        const F8Workspace w = f8_workspace(M, K, N, type, out_type);
        SQ_TRY(check_workspace(workspace, workspace_bytes, w.bytes()));
        hipStream_t s = static_cast<hipStream_t>(stream);
        if (f8_rows_ok(M, K, N, type)) {
            F8RowsArgs r{};
            r.x = X;
            r.type = type;
            r.M = M;
            r.K = K;
            r.ld = ld;
            r.W = W;
            r.Ws = W_scales;
            r.N = N;
            r.Y = Y;
            r.out_type = out_type;
            r.ldy = ldy;
            return hip_status(launch_f8_rows(r, s), "f8 linear");
        }
        uint8_t* codes = static_cast<uint8_t*>(workspace);
        uint8_t* scales = codes + w.codes;
        SQ_TRY(sq_f8_quantize(X, type, M, K, ld, 0, codes, scales, nullptr, nullptr, stream));
        return sq_f8_gemm(codes, scales, W, W_scales, M, N, K, Y, out_type, ldy, scales + w.scales, w.part, stream);
    });
}

// ---------------------------------------------------------------------------
sq_status sq_f8_layer_workspace_size(const sq_f8_layer* layer, size_t* bytes) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_f8_layer(layer));
        if (!bytes) return invalid("bytes is NULL");
        *bytes = f8_layer_workspace(layer);
        return SQ_OK;
    });
}

sq_status sq_f8_layer_weight(const sq_f8_layer* layer, const void* W, int64_t ld, void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_f8_layer(layer));
        const sq_f8_layer& l = *layer;
        return sq_f8_quantize(W, l.type, l.c_out, l.c_in, ld, 1, l.w, l.w_scales, l.w_t, l.w_t_scales, stream);
    });
}

sq_status sq_f8_layer_forward(const sq_f8_layer* layer, const void* X, int64_t ld, void* Y, int64_t ldy, void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_f8_layer(layer));
        const sq_f8_layer& l = *layer;
        SQ_TRY(check_f8_product(l.rows, l.c_out, l.c_in));
        if (l.rows > 0 && l.c_out > 0) {
            SQ_TRY(check_values(Y, l.type, ldy, l.c_out, "Y"));
            if (l.c_in > 0) {
                SQ_TRY(check_mx(l.w, l.w_scales, "w"));
                SQ_TRY(check_mx(l.x, l.x_scales, "x"));
            }
        }
        SQ_TRY(check_workspace(l.workspace, l.workspace_bytes, f8_layer_workspace(layer)));
        SQ_TRY(sq_f8_quantize(X, l.type, l.rows, l.c_in, ld, 0, l.x, l.x_scales, l.x_t, l.x_t_scales, stream));
        return sq_f8_gemm(l.x, l.x_scales, l.w, l.w_scales, l.rows, l.c_out, l.c_in, Y, l.type, ldy, l.workspace, l.workspace_bytes,
                          stream);
    });
}

sq_status sq_f8_layer_backward(const sq_f8_layer* layer, const void* dY, int64_t ld, void* dX, int64_t ld_dx, float* dW,
                               int64_t ld_dw, void* stream) {
    return guarded([&]() -> sq_status {
        SQ_TRY(check_f8_layer(layer));
        const sq_f8_layer& l = *layer;
        SQ_TRY(check_f8_product(l.rows, l.c_in, l.c_out));
        SQ_TRY(check_f8_product(l.c_out, l.c_in, l.rows));
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
        SQ_TRY(check_workspace(l.workspace, l.workspace_bytes, f8_layer_workspace(layer)));
        SQ_TRY(sq_f8_quantize(dY, l.type, l.rows, l.c_out, ld, 0, l.dy, l.dy_scales, l.dy_t, l.dy_t_scales, stream));
        const size_t part = f8_part_bytes(l.rows, l.c_in, l.c_out, l.type);
        const F8GemmArgs x = product_args(l.dy, l.dy_scales, l.w_t, l.w_t_scales, l.rows, l.c_in, l.c_out, dX, l.type, ld_dx,
                                          l.workspace),
                         w = product_args(l.dy_t, l.dy_t_scales, l.x_t, l.x_t_scales, l.c_out, l.c_in, l.rows, dW, SQ_TYPE_F32,
                                          ld_dw, static_cast<uint8_t*>(l.workspace) + part);
        return hip_status(launch_f8_gemm_pair(x, w, static_cast<hipStream_t>(stream)), "f8 gradients");
    });
}

}  // extern "C"
