// Gated dense layers:  G = X W_gate + b_gate,  U = X W_up + b_up,  H = act(G) (.) U,  and their backward pass
//     dG = dH (.) U (.) act'(G),  dU = dH (.) act(G),
//     dW_gate = X^T dG,  dW_up = X^T dU,  db_gate = 1^T dG,  db_up = 1^T dU,  dX = dG W_gate^T + dU W_up^T + R.
// Forward: one product whose columns are the two weights' in turn, 32 of the one and 32 of the other, so that a lane ends with G and U of the same places
// and H is written without either having been in memory (wide_gemm.hpp).  Backward: see wide_layers.hpp.
#include "wide_layers.hpp"

namespace tma {

template <typename T>
static int gated_fwd(const char *fn, int64_t n, const void *X, int64_t ldx, int32_t F_in, const float *W_gate, const float *W_up, const float *b_gate, const float *b_up,
                     int32_t F_out, int32_t act, void *G, void *U, int64_t ldg, void *H, int64_t ldh, void *ws, hipStream_t s)
{
    T *g = static_cast<T *>(G), *u = static_cast<T *>(U), *h = static_cast<T *>(H);
    auto make = [&](auto streamed) {
        return GatedEpilogue<T, decltype(streamed)::value>{g, u, h, ldg, ldh, n, b_gate, b_up, F_out, act, whole_rows(h, ldh) && (!g || (whole_rows(g, ldg) && whole_rows(u, ldg))),
                                                           bias_pieces(b_gate, F_out) && bias_pieces(b_up, F_out)};
    };
    if (n <= kFewMost)
        return launch_few<T, 2>(fn, sizeof(T) == 2 ? "gated_few_bf16" : "gated_few", n, X, ldx, W_gate, W_up, F_in, F_out, make(std::false_type{}), ws, s);
    const ForwardPlan p = plan_forward<T>(n, F_in, F_out, 2, false, ws);
    const float *const W[2] = {W_gate, W_up};
    auto go = [&](auto streamed) {
        return forward_product<T>(fn, sizeof(T) == 2 ? "gated_fwd_bf16" : "gated_fwd", n, static_cast<const T *>(X), ldx, F_in, W, F_out, p, make(streamed), s);
    };
    return past_caches(n, F_out, sizeof(T) * (g ? 3 : 1)) ? go(std::true_type{}) : go(std::false_type{});
}

template <typename T>
static int gated_bwd(const char *fn, int64_t n, const void *X, int64_t ldx, const void *G, const void *U, int64_t ldg, const void *dH, int64_t ldh, const float *W_gate,
                     const float *W_up, int32_t F_in, int32_t F_out, int32_t act, float *dW_gate, float *dW_up, float *db_gate, float *db_up, void *dX, int64_t ld_dx,
                     const void *R, int64_t ldr, void *ws, hipStream_t s)
{
    GradCall<T> g{static_cast<const T *>(G), static_cast<const T *>(U), static_cast<const T *>(dH), ldg, ldh, n, F_out, act};
    g.wz = whole_rows(g.Z, ldg) && whole_rows(g.U, ldg);
    g.wy = whole_rows(g.dY, ldh);
    const float *const W[2] = {W_gate, W_up};
    float *const dW[2] = {dW_gate, dW_up}, *const db[2] = {db_gate, db_up};
    return wide_backward<T, 2>(fn, "gated", n, static_cast<const T *>(X), ldx, g, W, F_in, dW, db, static_cast<T *>(dX), ld_dx, static_cast<const T *>(R), ldr, ws, s);
}

}  // namespace tma

extern "C" size_t tma_gated_dense_fwd_workspace_bytes(int64_t n, int32_t F_in, int32_t F_out, int32_t dtype)
{
    return tma::forward_workspace(n, F_in, F_out, 2, dtype, false);
}

extern "C" size_t tma_gated_dense_fwd_workspace_bytes_at16(int64_t n, int32_t F_in, int32_t F_out, int32_t dtype)
{
    return tma::forward_workspace(n, F_in, F_out, 2, dtype, true);
}

extern "C" int tma_gated_dense_fwd(int64_t n, const void *X, int64_t ldx, int32_t F_in, const float *W_gate, const float *W_up, const float *b_gate, const float *b_up,
                                   int32_t F_out, int32_t act, int32_t dtype, void *G_out, void *U_out, int64_t ldg, void *H_out, int64_t ldh, void *ws, size_t ws_bytes,
                                   tma_stream_t stream)
{
    using namespace tma;
    const char *fn = "tma_gated_dense_fwd";
    if (int rc = check_wide(fn, n, F_in, F_out, act, dtype, ws, ws_bytes, forward_workspace(n, F_in, F_out, 2, dtype, rows_at16(X, ldx)))) return rc;
    TMA_REQUIRE(!G_out == !U_out, TMA_ERR_INVALID_ARG, "%s: G_out and U_out go together", fn);
    if (n == 0) return TMA_OK;
    TMA_REQUIRE(X && W_gate && W_up && H_out, TMA_ERR_INVALID_ARG, "%s: NULL argument", fn);
    TMA_REQUIRE(H_out != X && G_out != X && U_out != X && H_out != G_out && H_out != U_out && (!G_out || G_out != U_out), TMA_ERR_INVALID_ARG,
                "%s: two of X, G_out, U_out and H_out are one", fn);
    TMA_REQUIRE(ldx >= F_in && ldh >= F_out && (!G_out || ldg >= F_out), TMA_ERR_BAD_SHAPE, "%s: a leading dimension is below its width", fn);
    hipStream_t s = as_stream(stream);
    return dtype == TMA_BF16 ? gated_fwd<uint16_t>(fn, n, X, ldx, F_in, W_gate, W_up, b_gate, b_up, F_out, act, G_out, U_out, ldg, H_out, ldh, ws, s)
                             : gated_fwd<float>(fn, n, X, ldx, F_in, W_gate, W_up, b_gate, b_up, F_out, act, G_out, U_out, ldg, H_out, ldh, ws, s);
}

extern "C" size_t tma_gated_dense_bwd_workspace_bytes(int64_t n, int32_t F_in, int32_t F_out, int32_t dtype, int32_t need_dX)
{
    using namespace tma;
    if (!wide_sizes_ok(n, F_in, F_out)) return 0;
    return (dtype == TMA_BF16 ? plan_backward<uint16_t>(n, F_in, F_out, 2, false, need_dX != 0, false, nullptr)
                              : plan_backward<float>(n, F_in, F_out, 2, false, need_dX != 0, false, nullptr)).bytes;
}

extern "C" int tma_gated_dense_bwd(int64_t n, const void *X, int64_t ldx, const void *G, const void *U, int64_t ldg, const void *dH, int64_t ldh, const float *W_gate,
                                   const float *W_up, int32_t F_in, int32_t F_out, int32_t act, int32_t dtype, float *dW_gate, float *dW_up, float *db_gate,
                                   float *db_up, void *dX_out, int64_t ld_dx, const void *R, int64_t ldr, void *ws, size_t ws_bytes, tma_stream_t stream)
{
    using namespace tma;
    const char *fn = "tma_gated_dense_bwd";
    if (int rc = check_wide(fn, n, F_in, F_out, act, dtype, ws, ws_bytes, tma_gated_dense_bwd_workspace_bytes(n, F_in, F_out, dtype, dX_out != nullptr))) return rc;
    TMA_REQUIRE(dW_gate && dW_up && dW_gate != dW_up, TMA_ERR_INVALID_ARG, "%s: dW_gate or dW_up is NULL, or they are one", fn);
    TMA_REQUIRE(!db_gate == !db_up && (!db_gate || db_gate != db_up), TMA_ERR_INVALID_ARG, "%s: db_gate and db_up go together", fn);
    for (const float *w : {W_gate, W_up}) TMA_REQUIRE(w != dW_gate && w != dW_up, TMA_ERR_INVALID_ARG, "%s: a weight is its gradient", fn);
    if (n > 0) {
        TMA_REQUIRE(X && G && U && dH && (!dX_out || (W_gate && W_up)), TMA_ERR_INVALID_ARG, "%s: NULL argument", fn);
        TMA_REQUIRE(ldx >= F_in && ldg >= F_out && ldh >= F_out && (!dX_out || (ld_dx >= F_in && (!R || ldr >= F_in))), TMA_ERR_BAD_SHAPE,
                    "%s: a leading dimension is below its width", fn);
        TMA_REQUIRE(!dX_out || (dX_out != X && dX_out != G && dX_out != U && dX_out != dH), TMA_ERR_INVALID_ARG, "%s: dX_out is one of X, G, U, dH", fn);
        TMA_REQUIRE(!dX_out || dX_out != R || ld_dx == ldr, TMA_ERR_BAD_SHAPE, "%s: R in place has dX_out's leading dimension", fn);
    }
    hipStream_t s = as_stream(stream);
    return dtype == TMA_BF16 ? gated_bwd<uint16_t>(fn, n, X, ldx, G, U, ldg, dH, ldh, W_gate, W_up, F_in, F_out, act, dW_gate, dW_up, db_gate, db_up,
                                                   n > 0 ? dX_out : nullptr, ld_dx, R, ldr, ws, s)
                             : gated_bwd<float>(fn, n, X, ldx, G, U, ldg, dH, ldh, W_gate, W_up, F_in, F_out, act, dW_gate, dW_up, db_gate, db_up,
                                                n > 0 ? dX_out : nullptr, ld_dx, R, ldr, ws, s);
}
