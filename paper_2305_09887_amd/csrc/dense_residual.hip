// Dense layers that add to what goes past them:  Z = X W + 1 b^T,  Y = act(Z) + R,  and their backward pass
//     dZ = dY (.) act'(Z),  dW = X^T dZ,  dbias = 1^T dZ,  dX = dZ W^T + R   (R: the gradient that went past; dY itself goes to the forward call's R).
// Bias, activation and addition happen where the product's sums are (wide_gemm.hpp); backward: see wide_layers.hpp.
#include "wide_layers.hpp"

namespace tma {

template <typename T>
static int residual_fwd(const char *fn, int64_t n, const void *X, int64_t ldx, int32_t F_in, const float *W, const float *bias, int32_t F_out, int32_t act, const void *R,
                        int64_t ldr, void *Z, int64_t ldz, void *Y, int64_t ldy, void *ws, hipStream_t s)
{
    T *z = static_cast<T *>(Z), *y = static_cast<T *>(Y);
    const T *r = static_cast<const T *>(R);
    auto make = [&](auto streamed) {
        return ResidualEpilogue<T, decltype(streamed)::value>{z, y, r, ldz, ldy, ldr, n, bias, F_out, act, whole_rows(y, ldy) && (!z || whole_rows(z, ldz)),
                                                              r && whole_rows(r, ldr), bias_pieces(bias, F_out)};
    };
    if (n <= kFewMost) return launch_few<T, 1>(fn, sizeof(T) == 2 ? "residual_few_bf16" : "residual_few", n, X, ldx, W, nullptr, F_in, F_out, make(std::false_type{}), ws, s);
    const ForwardPlan p = plan_forward<T>(n, F_in, F_out, 1, r != nullptr, ws);
    const float *const one[2] = {W, nullptr};
    auto go = [&](auto streamed) {
        return forward_product<T>(fn, sizeof(T) == 2 ? "residual_fwd_bf16" : "residual_fwd", n, static_cast<const T *>(X), ldx, F_in, one, F_out, p, make(streamed), s);
    };
    return past_caches(n, F_out, sizeof(T) * (z ? 2 : 1)) ? go(std::true_type{}) : go(std::false_type{});
}

template <typename T>
static int residual_bwd(const char *fn, int64_t n, const void *X, int64_t ldx, const void *Z, int64_t ldz, const void *dY, int64_t ldy, const float *W_, int32_t F_in,
                        int32_t F_out, int32_t act, float *dW_, float *dbias, void *dX, int64_t ld_dx, const void *R, int64_t ldr, void *ws, hipStream_t s)
{
    GradCall<T> g{static_cast<const T *>(Z), nullptr, static_cast<const T *>(dY), ldz, ldy, n, F_out, act};
    g.wz = Z && whole_rows(g.Z, ldz);
    g.wy = whole_rows(g.dY, ldy);
    const float *const W[2] = {W_, nullptr};
    float *const dW[2] = {dW_, nullptr}, *const db[2] = {dbias, nullptr};
    return wide_backward<T, 1>(fn, "residual", n, static_cast<const T *>(X), ldx, g, W, F_in, dW, db, static_cast<T *>(dX), ld_dx, static_cast<const T *>(R), ldr, ws, s);
}

}  // namespace tma

extern "C" size_t tma_dense_residual_fwd_workspace_bytes(int64_t n, int32_t F_in, int32_t F_out, int32_t dtype)
{
    return tma::forward_workspace(n, F_in, F_out, 1, dtype, false);
}

extern "C" size_t tma_dense_residual_fwd_workspace_bytes_at16(int64_t n, int32_t F_in, int32_t F_out, int32_t dtype)
{
    return tma::forward_workspace(n, F_in, F_out, 1, dtype, true);
}

extern "C" int tma_dense_residual_fwd(int64_t n, const void *X, int64_t ldx, int32_t F_in, const float *W, const float *bias, int32_t F_out, int32_t act, int32_t dtype,
                                      const void *R, int64_t ldr, void *Z_out, int64_t ldz, void *Y_out, int64_t ldy, void *ws, size_t ws_bytes, tma_stream_t stream)
{
    using namespace tma;
    const char *fn = "tma_dense_residual_fwd";
    if (int rc = check_wide(fn, n, F_in, F_out, act, dtype, ws, ws_bytes, forward_workspace(n, F_in, F_out, 1, dtype, rows_at16(X, ldx)))) return rc;
    if (n == 0) return TMA_OK;
    TMA_REQUIRE(X && W && Y_out, TMA_ERR_INVALID_ARG, "%s: NULL argument", fn);
    TMA_REQUIRE(Y_out != X && Z_out != X && Z_out != Y_out && (!Z_out || Z_out != R), TMA_ERR_INVALID_ARG, "%s: Z_out is one of X, R, Y_out, or Y_out is X", fn);
    TMA_REQUIRE(ldx >= F_in && ldy >= F_out && (!Z_out || ldz >= F_out) && (!R || ldr >= F_out), TMA_ERR_BAD_SHAPE, "%s: a leading dimension is below its width", fn);
    TMA_REQUIRE(R != Y_out || ldr == ldy, TMA_ERR_BAD_SHAPE, "%s: R in place has Y_out's leading dimension", fn);
    hipStream_t s = as_stream(stream);
    return dtype == TMA_BF16 ? residual_fwd<uint16_t>(fn, n, X, ldx, F_in, W, bias, F_out, act, R, ldr, Z_out, ldz, Y_out, ldy, ws, s)
                             : residual_fwd<float>(fn, n, X, ldx, F_in, W, bias, F_out, act, R, ldr, Z_out, ldz, Y_out, ldy, ws, s);
}

extern "C" size_t tma_dense_residual_bwd_workspace_bytes(int64_t n, int32_t F_in, int32_t F_out, int32_t act, int32_t dtype, int32_t need_dX)
{
    using namespace tma;
    if (!wide_sizes_ok(n, F_in, F_out)) return 0;
    const bool exact = act == TMA_ACT_NONE;
    return (dtype == TMA_BF16 ? plan_backward<uint16_t>(n, F_in, F_out, 1, exact, need_dX != 0, false, nullptr)
                              : plan_backward<float>(n, F_in, F_out, 1, exact, need_dX != 0, false, nullptr)).bytes;
}

extern "C" int tma_dense_residual_bwd(int64_t n, const void *X, int64_t ldx, const void *Z, int64_t ldz, const void *dY, int64_t ldy, const float *W, int32_t F_in,
                                      int32_t F_out, int32_t act, int32_t dtype, float *dW, float *dbias, void *dX_out, int64_t ld_dx, const void *R, int64_t ldr,
                                      void *ws, size_t ws_bytes, tma_stream_t stream)
{
    using namespace tma;
    const char *fn = "tma_dense_residual_bwd";
    if (int rc = check_wide(fn, n, F_in, F_out, act, dtype, ws, ws_bytes, tma_dense_residual_bwd_workspace_bytes(n, F_in, F_out, act, dtype, dX_out != nullptr))) return rc;
    TMA_REQUIRE(dW && dW != W, TMA_ERR_INVALID_ARG, "%s: dW is NULL, or W", fn);
    if (n > 0) {
        TMA_REQUIRE(X && dY && (!dX_out || W), TMA_ERR_INVALID_ARG, "%s: NULL argument", fn);
        TMA_REQUIRE(act == TMA_ACT_NONE || Z, TMA_ERR_INVALID_ARG, "%s: Z is required with an activation", fn);
        TMA_REQUIRE(ldx >= F_in && ldy >= F_out && (act == TMA_ACT_NONE || ldz >= F_out) && (!dX_out || (ld_dx >= F_in && (!R || ldr >= F_in))), TMA_ERR_BAD_SHAPE,
                    "%s: a leading dimension is below its width", fn);
        TMA_REQUIRE(!dX_out || (dX_out != X && dX_out != Z && (dX_out != dY || R == dY)), TMA_ERR_INVALID_ARG, "%s: dX_out is one of X, Z, or dY without being R", fn);
        TMA_REQUIRE(!dX_out || dX_out != R || ld_dx == ldr, TMA_ERR_BAD_SHAPE, "%s: R in place has dX_out's leading dimension", fn);
    }
    hipStream_t s = as_stream(stream);
    return dtype == TMA_BF16 ? residual_bwd<uint16_t>(fn, n, X, ldx, Z, ldz, dY, ldy, W, F_in, F_out, act, dW, dbias, n > 0 ? dX_out : nullptr, ld_dx, R, ldr, ws, s)
                             : residual_bwd<float>(fn, n, X, ldx, Z, ldz, dY, ldy, W, F_in, F_out, act, dW, dbias, n > 0 ? dX_out : nullptr, ld_dx, R, ldr, ws, s);
}
