// What the gated layers and the dense layers with a residual share beside their products (wide_gemm.hpp): activations, what becomes of a product, the
// gradients of the pre-activations, and the host's plans.
#pragma once
#include "wide_few.hpp"
#include "wide_gemm.hpp"
#include "wide_split.hpp"

namespace tma {

// ---- activations ---------------------------------------------------------------
// silu z = z s(z), s = 1 / (1 + e^-z); gelu z = z Phi(z), Phi(-|z|) = erfc(|z| / sqrt 2) / 2.
__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }
// Phi(z), from e = e^(-z^2 / 2).  erfc(x) = e^(-x^2) t Q(t), t = 1 / (1 + x / 2): Q of degree 8 is a fit of erfcx(x) / t over 0 <= x <= 12 by weighted least
// squares, relative error 4.4e-8; in fp32 3.4e-7 at most and 8e-8 in the mean over 0 <= x <= 9.  What callers pass for e is e^(-z^2 / 2) (1 + d), |d| up to
// 2^-24 z^2: the exponent is rounded when it is squared and when it is multiplied by log2 e.  So the tail is off by 1.9e-6 of itself at z = -6 and 7e-6 at -12.5
// (SiLU's by 4e-6 at -87), Phi by 1.6e-7 at most, absolute; an exponent in two parts would take six instructions more.  (The library's erfc takes some five times
// the instructions: 8,192 rows 2048 -> 8192 gated 577 us, with silu 483.)
__device__ __forceinline__ float normal_below(float z, float e)
{
    const float t = __builtin_amdgcn_rcpf(fmaf(0.35355339f, fabsf(z), 1.0f));
    float q = -0.05936308f;
    q = fmaf(q, t, 0.28601065f);
    q = fmaf(q, t, -0.49017346f);
    q = fmaf(q, t, 0.28146902f);
    q = fmaf(q, t, -0.028968235f);
    q = fmaf(q, t, 0.2036771f);
    q = fmaf(q, t, 0.24285392f);
    q = fmaf(q, t, 0.28240955f);
    q = fmaf(q, t, 0.28208447f);
    const float tail = 0.5f * e * (t * q);
    return z > 0.0f ? 1.0f - tail : tail;
}

template <int N>
__device__ __forceinline__ void activate(int act, float (&v)[N])
{
    if (act == TMA_ACT_SILU) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] *= logistic(v[j]);
    } else if (act == TMA_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] *= normal_below(v[j], __expf(-0.5f * v[j] * v[j]));
    } else if (act == TMA_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = v[j] > 0.0f ? v[j] : 0.0f;
    }
}
// act(z) and act'(z)
template <int N>
__device__ __forceinline__ void activate_both(int act, const float (&z)[N], float (&value)[N], float (&slope)[N])
{
    if (act == TMA_ACT_SILU) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float t = logistic(z[j]);
            value[j] = z[j] * t;
            slope[j] = t * (1.0f + z[j] * (1.0f - t));
        }
    } else if (act == TMA_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float e = __expf(-0.5f * z[j] * z[j]), p = normal_below(z[j], e);
            value[j] = z[j] * p;
            slope[j] = p + z[j] * (0.39894228f * e);
        }
    } else if (act == TMA_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            value[j] = z[j] > 0.0f ? z[j] : 0.0f;
            slope[j] = z[j] > 0.0f ? 1.0f : 0.0f;
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            value[j] = z[j];
            slope[j] = 1.0f;
        }
    }
}

// ---- what becomes of a product -------------------------------------------------
// E = 16 / sizeof(T) neighbours of a row, of which those before `cols` exist; whole: all do, and lie at a multiple of 16 bytes.
// kStreamed: past the caches (a flag of the type: of two stores behind a condition the compiler makes one ordinary one).  Results that those would not hold anyway are stored faster so (125,237 rows 128 -> 2 x 256 in fp32 with its backward pass 611 and 566 us, 1,000,003
// rows 256 -> 256 in bf16 499 and 485); smaller ones are read from there by the next call (a block of 4,096 rows, 1024 and 4096 wide, 625 us, so 635).
typedef uint32_t Words __attribute__((ext_vector_type(4)));
template <bool kStreamed>
__device__ __forceinline__ void store_words(void *p, const Words &w)
{
    if constexpr (kStreamed) __builtin_nontemporal_store(w, static_cast<Words *>(p));
    else *static_cast<Words *>(p) = w;
}
template <bool kStreamed = false, int E>
__device__ __forceinline__ void store_some(float *p, int c, int cols, bool whole, const float (&v)[E])
{
    if (whole) {
        const Words w = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
        store_words<kStreamed>(p + c, w);
    } else {
#pragma unroll
        for (int j = 0; j < E; ++j)
            if (c + j < cols) p[c + j] = v[j];
    }
}
template <bool kStreamed = false, int E>
__device__ __forceinline__ void store_some(uint16_t *p, int c, int cols, bool whole, const float (&v)[E])
{
    if (whole) {
        const Words w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
        store_words<kStreamed>(p + c, w);
    } else {
#pragma unroll
        for (int j = 0; j < E; ++j)
            if (c + j < cols) p[c + j] = f32_to_bf16(v[j]);
    }
}
__device__ __forceinline__ void narrow(float *p, float v) { *p = v; }
__device__ __forceinline__ void narrow(uint16_t *p, float v) { *p = f32_to_bf16(v); }

// (every load without a condition of its own: each of those was waited for before the next, 100 us of 8,192 rows 2048 -> 8192)
template <int E>
__device__ __forceinline__ void bias_of(const float *bias, int c, int cols, bool pieces, float (&v)[E])
{
    if (!bias) {
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = 0.0f;
    } else if (pieces) {      // at a multiple of 16 bytes, and cols a multiple of eight
        const float4 *from = reinterpret_cast<const float4 *>(bias + (c < cols ? c : 0));
#pragma unroll
        for (int p = 0; p < E / 4; ++p) {
            const float4 x = from[p];
            v[4 * p] = x.x;
            v[4 * p + 1] = x.y;
            v[4 * p + 2] = x.z;
            v[4 * p + 3] = x.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = bias[c + j < cols ? c + j : cols - 1];
    }
}
inline bool past_caches(int64_t rows, int64_t cols, int64_t bytes) { return rows * cols * bytes > int64_t(256) << 20; }
inline bool bias_pieces(const float *bias, int cols) { return aligned(bias, 16) && cols % 8 == 0; }

// What an epilogue does with a stage of sums: a lane has E neighbours of each kRows-th row, kLanes of them make one.
template <typename T, int kSides, class St>
struct Lanes {
    static constexpr int E = 16 / sizeof(T), kLanes = St::kCols / kSides / E, kRows = 64 / kLanes, kSteps = St::kRows / kRows;
};

// H = act(G) (.) U, G and U kept where asked for
template <typename T, bool kStreamed = false>
struct GatedEpilogue {
    static constexpr int kSides = 2, kStores = sizeof(T) == 2 ? 1 : 2, E = 16 / sizeof(T);
    static constexpr bool kPast = false;
    template <int TN>
    using StageOf = std::conditional_t<sizeof(T) == 2 && TN % 4 == 0, Stage<16, 128>, Stage<32, 64>>;
    T *G, *U, *H;                 // G, U: NULL together
    int64_t ldg, ldh, M;
    const float *b_gate, *b_up;   // may be NULL
    int N, act;
    bool whole16, pieces;         // rows of G, U and H begin at 16 bytes; the biases come in such pieces
    struct Past {};
    template <class St>
    struct Cols {
        float g[E], u[E];
        __device__ __forceinline__ void wait()
        {
#pragma unroll
            for (int j = 0; j < E; ++j) {
                arrived(g[j]);
                arrived(u[j]);
            }
        }
    };
    template <class St>
    __device__ __forceinline__ void columns(int col, int lane, Cols<St> &k) const
    {
        const int c = col + lane % Lanes<T, 2, St>::kLanes * E;
        bias_of(b_gate, c, N, pieces, k.g);
        bias_of(b_up, c, N, pieces, k.u);
    }
    __device__ __forceinline__ void past(int64_t, int, int, Past &) const {}
    template <class St>
    __device__ __forceinline__ void emit(const St &t, int64_t row0, int col, int, const Cols<St> &of, Past &) const
    {
        typedef Lanes<T, 2, St> L;
        const int in = t.lane % L::kLanes * E, c = col + in, r0 = t.lane / L::kLanes, at = in / 32 * 64 + in % 32;
        if (c >= N) return;
        const bool all = whole16 && c + E <= N;
#pragma unroll
        for (int k = 0; k < L::kSteps; ++k) {
            const int64_t row = row0 + r0 + k * L::kRows;
            float g[E], u[E];
            t.get(r0 + k * L::kRows, at, g);
            t.get(r0 + k * L::kRows, at + 32, u);
            if (row >= M) continue;
#pragma unroll
            for (int j = 0; j < E; ++j) {
                g[j] += of.g[j];
                u[j] += of.u[j];
            }
            if (G) {
                store_some<kStreamed>(G + row * ldg, c, N, all, g);
                store_some<kStreamed>(U + row * ldg, c, N, all, u);
            }
            activate(act, g);
#pragma unroll
            for (int j = 0; j < E; ++j) g[j] *= u[j];
            store_some<kStreamed>(H + row * ldh, c, N, all, g);
        }
    }
    __device__ __forceinline__ bool whole(int64_t m_end, int n_end) const { return whole16 && m_end <= M && n_end <= N; }
    // of one place
    __device__ __forceinline__ void one(int64_t row, int c, float g, float u) const
    {
        if (b_gate) g += b_gate[c];
        if (b_up) u += b_up[c];
        if (G) {
            narrow(G + row * ldg + c, g);
            narrow(U + row * ldg + c, u);
        }
        float v[1] = {g};
        activate(act, v);
        narrow(H + row * ldh + c, v[0] * u);
    }
};

// Y = act(Z) + R, Z = product + bias kept where asked for.  R is on its way before the sums that it is added to are in LDS.
template <typename T, bool kStreamed = false>
struct ResidualEpilogue {
    template <int TN>
    using StageOf = Stage<32, 64>;
    typedef Lanes<T, 1, Stage<32, 64>> L;
    static constexpr int kSides = 1, kStores = sizeof(T) == 2 ? 2 : 4;
    static constexpr bool kPast = true;
    T *Z, *Y;                     // Z may be NULL
    const T *R;                   // may be NULL, may be Y
    int64_t ldz, ldy, ldr, M;
    const float *bias;            // may be NULL
    int N, act;
    bool whole16, past16, pieces; // rows of Z and Y, of R, begin at 16 bytes; the bias comes in such pieces
    struct Past {
        uint4 v[L::kSteps];
    };
    template <class St>
    struct Cols {
        float b[L::E];
        __device__ __forceinline__ void wait()
        {
#pragma unroll
            for (int j = 0; j < L::E; ++j) arrived(b[j]);
        }
    };
    template <class St>
    __device__ __forceinline__ void columns(int col, int lane, Cols<St> &k) const { bias_of(bias, col + lane % L::kLanes * L::E, N, pieces, k.b); }
    __device__ __forceinline__ void past(int64_t row0, int col, int lane, Past &p) const
    {
        if (!R) return;
        const int c = col + lane % L::kLanes * L::E;
#pragma unroll
        for (int k = 0; k < L::kSteps; ++k) {
            const int64_t row = row0 + lane / L::kLanes + k * L::kRows;
            if (row >= M || c >= N) continue;
            const T *from = R + row * ldr + c;
            if (past16 && c + L::E <= N) {
                const Words *words = reinterpret_cast<const Words *>(from);
                Words w;
                if constexpr (kStreamed) w = __builtin_nontemporal_load(words);
                else w = *words;
                p.v[k] = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
                T one[L::E];
#pragma unroll
                for (int j = 0; j < L::E; ++j) one[j] = c + j < N ? from[j] : T(0);
                __builtin_memcpy(&p.v[k], one, 16);
            }
        }
    }
    template <class St>
    __device__ __forceinline__ void emit(const St &t, int64_t row0, int col, int, const Cols<St> &of, Past &p) const
    {
        constexpr int E = L::E;
#pragma unroll
        for (int k = 0; k < L::kSteps; ++k) arrived(p.v[k]);
        const int in = t.lane % L::kLanes * E, c = col + in, r0 = t.lane / L::kLanes;
        if (c >= N) return;
        const bool all = whole16 && c + E <= N;
#pragma unroll
        for (int k = 0; k < L::kSteps; ++k) {
            const int64_t row = row0 + r0 + k * L::kRows;
            float z[E];
            t.get(r0 + k * L::kRows, in, z);
            if (row >= M) continue;
#pragma unroll
            for (int j = 0; j < E; ++j) z[j] += of.b[j];
            if (Z) store_some<kStreamed>(Z + row * ldz, c, N, all, z);
            activate(act, z);
            if (R) {
                float r[E];
                Chunk<T>::widen(p.v[k], r);
#pragma unroll
                for (int j = 0; j < E; ++j) z[j] += r[j];
            }
            store_some<kStreamed>(Y + row * ldy, c, N, all, z);
        }
    }
    __device__ __forceinline__ bool whole(int64_t m_end, int n_end) const { return whole16 && m_end <= M && n_end <= N; }
    __device__ __forceinline__ void one(int64_t row, int c, float z, float) const
    {
        if (bias) z += bias[c];
        if (Z) narrow(Z + row * ldz + c, z);
        float v[1] = {z};
        activate(act, v);
        if (R) v[0] += widen1(R[row * ldr + c]);
        narrow(Y + row * ldy + c, v[0]);
    }
};

// a weight gradient, or a range's share of it: the columns of `sides` matrices behind each other, each padded to whole units
struct WeightEpilogue {
    template <int TN>
    using StageOf = Stage<32, 64>;
    typedef Lanes<float, 1, Stage<32, 64>> L;
    static constexpr int kSides = 1, kStores = 4;
    static constexpr bool kPast = false;
    float *out[2];
    int64_t split_stride, M;
    int N, padded, sides;
    bool whole16;
    struct Past {};
    template <class St>
    struct Cols {
        __device__ __forceinline__ void wait() {}
    };
    template <class St>
    __device__ __forceinline__ void columns(int, int, Cols<St> &) const {}
    __device__ __forceinline__ void past(int64_t, int, int, Past &) const {}
    template <class St>
    __device__ __forceinline__ void emit(const St &t, int64_t row0, int col, int split, const Cols<St> &, Past &) const
    {
        const int in = t.lane % L::kLanes * 4, r0 = t.lane / L::kLanes;
        const int side = sides == 2 && col + in >= padded ? 1 : 0, c = col + in - side * padded;     // (tiles may reach past the last side)
        if (c >= N) return;
        const bool all = whole16 && c + 4 <= N;
        float *to = out[side] + split * split_stride;
#pragma unroll
        for (int k = 0; k < L::kSteps; ++k) {
            const int64_t row = row0 + r0 + k * L::kRows;
            float v[4];
            t.get(r0 + k * L::kRows, in, v);
            if (row < M) store_some(to + row * N, c, N, all, v);
        }
    }
    __device__ __forceinline__ bool whole(int64_t m_end, int n_end) const { return whole16 && m_end <= M && N == padded && n_end <= sides * padded; }
};

// ---- gradients of pre-activations ----------------------------------------------
// Gated: dG = dH U act'(G), dU = dH act(G).  One-sided: dZ = dY act'(Z).  Computed once, in fp32, and laid out once, the columns as a unit's rows: along k for
// dW = X^T [dG | dU], along its rows for dX = [dG | dU] [W_gate | W_up]^T.  In two bf16 parts of bf16 rows' gradients: dW is fp32, and its error from the parts
// is 2.8e-6 (2^-17 a value; sums of 8,192 products in fp32 have 1.6e-6; a third part would make dW half as dear again), dX, which is rounded to bf16, takes the first alone.
// The columns' sums go along: a block keeps them over its rows.  (Laid out for each of the two products they took a third more: 8,192 rows of 2 x 8192 in bf16
// 230 us, 125,237 of 2 x 256 in fp32 225, five TB/s.)
template <typename T>
struct GradCall {
    const T *Z, *U, *dY;          // Z: the gate's pre-activations; Z may be NULL without an activation
    int64_t ldz, ldy, n;
    int N, act;
    bool wz, wy;
    Packed by_cols;
    float *sums;                  // [blocks along the rows][sides * padded], or NULL
    int row_blocks;
};
template <int kSides>
struct GradTile {
    float tile[kSides][32][65], joined[kSides][4][64];
};
template <typename T, int kSides, int kParts>
__device__ __forceinline__ void grad_pack(const GradCall<T> &q, int block, GradTile<kSides> &lds)
{
    auto &tile = lds.tile;
    auto &joined = lds.joined;
    const int t = threadIdx.x, r = t / 8, piece = t % 8, col_in = t % 64, quarter = t / 64;
    const int strips = (q.N + 63) / 64, strip = block % strips, rows_at = block / strips;
    const int c0 = strip * 64, padded = (q.N + 31) / 32 * 32, c = c0 + piece * 8;
    const int64_t tiles = (q.n + 31) / 32;
    float sum[kSides] = {};
    for (int64_t i = rows_at; i < tiles; i += q.row_blocks) {
        const int64_t row = i * 32 + r;
        float d[kSides][8] = {};
        if (row < q.n && c < q.N) {
            float dy[8];
            load_eight(q.dY + row * q.ldy, c, q.N, q.wy, dy);
            if constexpr (kSides == 1) {
                float z[8], value[8], slope[8];
                if (q.act != TMA_ACT_NONE) load_eight(q.Z + row * q.ldz, c, q.N, q.wz, z);
                else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) z[j] = 0.0f;
                }
                activate_both(q.act, z, value, slope);
#pragma unroll
                for (int j = 0; j < 8; ++j) d[0][j] = q.act == TMA_ACT_NONE ? dy[j] : dy[j] * slope[j];
            } else {
                float g[8], u[8], value[8], slope[8];
                load_eight(q.Z + row * q.ldz, c, q.N, q.wz, g);
                load_eight(q.U + row * q.ldz, c, q.N, q.wz, u);
                activate_both(q.act, g, value, slope);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    d[0][j] = dy[j] * u[j] * slope[j];
                    d[kSides - 1][j] = dy[j] * value[j];
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int side = 0; side < kSides; ++side)
#pragma unroll
            for (int j = 0; j < 8; ++j) tile[side][r][piece * 8 + j] = d[side][j];
        __syncthreads();
        if (c0 + col_in < padded) {
#pragma unroll
            for (int side = 0; side < kSides; ++side) {
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = tile[side][quarter * 8 + j][col_in];
                uint4 parts[kParts];
                pack_eight<kParts>(v, parts);
                const int rb = side * (padded / kUnitRows) + (c0 + col_in) / kUnitRows;
                const int64_t kg = i * 2 + quarter / 2;
                const int slot = weights_place(fragment_row(col_in % 32), quarter % 2, quarter / 2);
#pragma unroll
                for (int p = 0; p < kParts; ++p)
                    *reinterpret_cast<uint4 *>(q.by_cols.at + p * q.by_cols.plane() + q.by_cols.unit(rb, kg) + slot * 16) = parts[p];
                sum[side] += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
            }
        }
    }
    if (!q.sums) return;
#pragma unroll
    for (int side = 0; side < kSides; ++side) joined[side][quarter][col_in] = sum[side];
    __syncthreads();
    if (t < 64 && c0 + t < padded) {
#pragma unroll
        for (int side = 0; side < kSides; ++side)
            q.sums[(int64_t(rows_at) * kSides + side) * padded + c0 + t] = (joined[side][0][t] + joined[side][1][t]) + (joined[side][2][t] + joined[side][3][t]);
    }
}

// Backward: the gradients of the pre-activations in the first `grads` blocks, the rows by columns in the next `cols`, the weights by rows in what blocks there are
// beyond.  One launch: a call of a few hundred rows is launches above all.
template <typename T, int kSides, int kParts>
__global__ __launch_bounds__(256) void backward_layouts_kernel(GradCall<T> g, ColsPack x, RowsPack w, int grads, int cols)
{
    constexpr int kP = sizeof(T) == 2 ? 1 : 3;
    __shared__ __attribute__((aligned(16))) union {
        GradTile<kSides> gradients;
        RowsTile<kP> rows;
    } lds;
    const int block = int(blockIdx.x);
    if (block < grads) grad_pack<T, kSides, kParts>(g, block, lds.gradients);
    else if (block < grads + cols) pack_cols<T, kP>(x, block - grads, cols);
    else pack_rows<float, kP>(w, block - grads - cols, int(gridDim.x) - grads - cols, lds.rows);
}

// What the ranges and the blocks of the layouts left: out[side][i] = the ranges' shares added up in their order, in the first sides * range_blocks blocks; then
// sums_out[side][i] = the blocks' sums of column i, 16 columns a block, 64 threads a column, each every 64th of them, joined in a fixed order.
struct JoinCall {
    const float *partial;
    int ranges, range_blocks, sides;
    int64_t range_stride, side_stride, count;
    float *out[2];
    const float *sums;
    int sum_blocks, padded, N;
    float *sums_out[2];
};
static __global__ __launch_bounds__(1024) void join_kernel(JoinCall q)
{
    __shared__ float part[64][17];
    const int block = int(blockIdx.x), of_ranges = q.sides * q.range_blocks;
    if (block < of_ranges) {
        const int side = block / q.range_blocks;
        const float *in = q.partial + side * q.side_stride;
        float *out = side ? q.out[1] : q.out[0];
        for (int64_t i = int64_t(block % q.range_blocks) * 1024 + threadIdx.x; i < q.count; i += int64_t(q.range_blocks) * 1024) {
            float sum = 0.0f;
#pragma unroll 4
            for (int p = 0; p < q.ranges; ++p) sum += in[p * q.range_stride + i];
            out[i] = sum;
        }
        return;
    }
    const int strips = (q.N + 15) / 16, at = block - of_ranges, side = at / strips;
    const int c = threadIdx.x % 16, g = threadIdx.x / 16, col = at % strips * 16 + c;
    float sum = 0.0f;
    if (col < q.N) {
#pragma unroll 8
        for (int p = g; p < q.sum_blocks; p += 64) sum += q.sums[(int64_t(p) * q.sides + side) * q.padded + col];
    }
    part[g][c] = sum;
    for (int half = 32; half; half >>= 1) {
        __syncthreads();
        if (g < half) part[g][c] += part[g + half][c];
    }
    if (g == 0 && col < q.N) (side ? q.sums_out[1] : q.sums_out[0])[col] = part[0][c];
}
// partial NULL and ranges 1: the product has stored its results itself; sums_out NULL: not wanted
static int launch_join(const char *fn, JoinCall q, hipStream_t s)
{
    const int64_t wide = ceil_div(q.count, 1024);
    q.range_blocks = q.ranges == 1 ? 0 : int(wide < 1 ? 1 : wide > 1024 ? 1024 : wide);
    const int64_t blocks = int64_t(q.sides) * (q.range_blocks + (q.sums_out[0] ? ceil_div(q.N, 16) : 0));
    if (blocks == 0) return TMA_OK;
    TMA_TIMED("wide_join", s);
    hipLaunchKernelGGL(join_kernel, dim3(unsigned(blocks)), dim3(1024), 0, s, q);
    return check_launch(fn);
}

// ---- plans ---------------------------------------------------------------------
constexpr int kCus = 256;
struct WidePlan {
    bool big;                     // tiles of 256 x 256 results, else of 128 x 128
    int splits, split_slabs;
};
inline int64_t wide_tiles(int m_units, int n_units, bool big) { return ceil_div(m_units, big ? 8 : 4) * ceil_div(n_units, big ? 8 : 4); }
// whether tiles of 256 x 256 multiply hardly more than there is (128 of 256 columns fill half of one: weight gradients of 128 x 512, 125,237 rows in fp32
// 230 us so)
inline bool fills_big(int m_units, int n_units) { return wide_tiles(m_units, n_units, true) * 4 * 10 <= wide_tiles(m_units, n_units, false) * 11; }
// Products of rows.  A large tile is multiplied 7 % faster (8192 -> 2048, 8,192 rows 267 and 287 us) but is alone on its unit, which does
// nothing else while results are written: where a product is short beside them, and first of all where they are added to something that has to be
// read, two small ones a unit are faster (256 -> 256 with a residual, 1,000,003 rows in bf16, eight slabs: 719 and 490 us).
// Where the tiles are few and long, ranges of k go to more blocks, and a second kernel joins their shares: as many as make least what a range's slabs take one after the
// other, 0.3 us each (fp32 1.1), with 3 us for the second kernel and the shares' way to memory and back.  (One range, then those chosen: 128 rows 4096 -> 4096 in bf16 with a
// residual 59 and 36 us; 100 rows 4096 -> 2 x 1024 in fp32 159 and 42; input gradient and all else backward of 128 rows 2048 -> 2 x 5632 in bf16 186 and 90.)
inline WidePlan plan_rows(int64_t n, const Packed &b, bool reads, bool fp32)
{
    const int slabs = b.kgs / 2, row_units = int(ceil_div(n, kUnitRows));
    const int64_t tiles = wide_tiles(row_units, b.rbs, false);
    int ranges = 1;       // of the sizes alone: the workspace is asked for without `reads`
    float least = 1e30f;
    for (int r = 1; r == 1 || (r <= 16 && r * tiles <= 2 * kCus && r * 4 <= slabs); ++r) {
        const float t = float(ceil_div(slabs, r)) * (fp32 ? 1.1f : 0.3f) + (r > 1 ? 3.0f + float(r) * float(n) * float(b.rbs) * (32 * 8 / 3e6f) : 0.0f);
        if (t < least) {
            least = t;
            ranges = r;
        }
    }
    if (ranges == 1)
        return {!fp32 && wide_tiles(row_units, b.rbs, true) >= kCus * 3 / 4 && fills_big(row_units, b.rbs) && slabs >= (reads ? 64 : 16), 1, slabs};
    const int per = int(ceil_div(slabs, ranges));
    return {false, int(ceil_div(slabs, per)), per};
}
inline size_t row_shares(const WidePlan &p, int64_t n, const Packed &b) { return p.splits > 1 ? size_t(p.splits) * size_t(n) * size_t(b.rbs) * (kUnitRows * 4) : 0; }
// ranges of k until the tiles fill the chip, 512 rows each at least; fp32 has small tiles only (two ranges a
// unit: three were no faster and wrote more, 125,237 rows of 128 x 512 141 and 144 us with their sums)
inline WidePlan plan_weight(const Packed &a, const Packed &b, bool fp32)
{
    const int slabs = a.kgs / 2, most = slabs / 16 > 1 ? slabs / 16 : 1;
    for (bool big : {true, false}) {
        const int64_t tiles = wide_tiles(a.rbs, b.rbs, big), slots = big ? kCus : 2 * kCus;
        int64_t want = slots / tiles;
        want = want < 1 ? 1 : want > most ? most : want;
        if (big && (fp32 || tiles * want < kCus / 2 || !fills_big(a.rbs, b.rbs))) continue;
        const int per = int(ceil_div(slabs, want));
        return {big, int(ceil_div(slabs, per)), per};
    }
    return {false, 1, slabs};
}

template <RowsAs kRows, bool kSmall, class Epi>
static int launch_wide_as(const char *name, WideCall q, const WidePlan &p, const Epi &e, hipStream_t s)
{
    const int units = p.big ? 8 : 4, per_cu = p.big ? 1 : 2;
    q.m_tiles = int(ceil_div(q.row_units, units));
    q.n_tiles = int(ceil_div(q.b.rbs, units));
    if (q.panel > q.n_tiles) q.panel = q.n_tiles;
    const int64_t total = int64_t(q.m_tiles) * q.n_tiles * q.splits;
    int64_t per_die = ceil_div(total, kWideDies);
    if (per_die > 32 * per_cu) per_die = 32 * per_cu;
    TMA_TIMED(name, s);
    const dim3 grid(unsigned(per_die * kWideDies)), block(256);
    if constexpr (!kSmall)
        if (p.big) {
            hipLaunchKernelGGL((wide_gemm_kernel<8, 8, 2, 2, 4, kRows, Epi>), grid, block, 0, s, q, e);
            return check_launch(name);
        }
    hipLaunchKernelGGL((wide_gemm_kernel<4, 4, 2, 2, 3, kRows, Epi>), grid, block, 0, s, q, e);
    return check_launch(name);
}
// operands of type T laid out: of bf16 in one part, on the weights' side in two where q says so, of fp32 in three; kSmall: the plan has small tiles
template <typename T, RowsAs kRows, bool kSmall = false, class Epi>
static int launch_wide(const char *name, WideCall q, const WidePlan &p, const Epi &e, hipStream_t s)
{
    if constexpr (sizeof(T) == 2) {
        return launch_wide_as<kRows, kSmall>(name, q, p, e, s);
    } else {
        q.m_tiles = int(ceil_div(q.row_units, 4));
        q.n_tiles = int(ceil_div(q.b.rbs, 4));
        if (q.panel > q.n_tiles) q.panel = q.n_tiles;
        const int64_t blocks = ceil_div(int64_t(q.m_tiles) * q.n_tiles * q.splits, kWideDies) * kWideDies;
        if (blocks > INT32_MAX) return fail(TMA_ERR_BAD_SHAPE, "%s: too many tiles", name);
        TMA_TIMED(name, s);
        hipLaunchKernelGGL((wide_split_kernel<kRows == kTurned, Epi>), dim3(unsigned(blocks)), dim3(256), 0, s, q, e);
        return check_launch(name);
    }
}

// A product of rows, in ranges of k where the plan says so: their shares [range][row][packed column], and what becomes of the sums
template <int kSides, class Out>
static __global__ __launch_bounds__(256) void join_rows_kernel(const float *__restrict__ shares, int ranges, int64_t n, int N, int pitch, Out out)
{
    const int64_t cells = n * N, stride = n * pitch;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < cells; i += int64_t(gridDim.x) * 256) {
        const int64_t row = i / N;
        const int c = int(i - row * N);
        const float *from = shares + row * pitch + (kSides == 2 ? c / 32 * 64 + c % 32 : c);
        float sum[kSides] = {};
#pragma unroll 4
        for (int p = 0; p < ranges; ++p)
#pragma unroll
            for (int s = 0; s < kSides; ++s) sum[s] += from[p * stride + s * 32];
        out.one(row, c, sum[0], sum[kSides - 1]);
    }
}
template <typename T, RowsAs kRows, class Epi>
static int launch_rows(const char *name, WideCall q, const WidePlan &p, float *shares, int64_t n, int N, const Epi &e, hipStream_t s)
{
    q.planes = planes_of(1);
    q.panel = 8;
    q.splits = p.splits;
    q.split_slabs = p.split_slabs;
    q.row_units = int(ceil_div(n, kUnitRows));
    if (p.splits == 1) return launch_wide<T, kRows>(name, q, p, e, s);
    const int pitch = q.b.rbs * kUnitRows;
    const WeightEpilogue share{{shares, nullptr}, n * pitch, n, pitch, pitch, 1, true};
    if (int rc = launch_wide<T, kRows, true>(name, q, p, share, s)) return rc;
    TMA_TIMED("wide_join_rows", s);
    int64_t blocks = ceil_div(n * N, 256);
    if (blocks > 8192) blocks = 8192;
    hipLaunchKernelGGL((join_rows_kernel<Epi::kSides, Epi>), dim3(unsigned(blocks)), dim3(256), 0, s, shares, p.splits, n, N, pitch, e);
    return check_launch(name);
}

// Parts that an operand is laid out in.  With rows in bf16 one: fp32 weights are rounded to bf16, as in the library's other bf16 products, which makes the error of a result that
// is itself rounded to bf16 0.0020 for 0.0017 (of a gated layer, two weights, 0.0029; relative norm against 64 bits).  A second part of the weights would be twice the
// matrix work, 450 us more of the 517 of 8,192 rows 2048 -> 2 x 8192.  Up to 64 rows, where the matrix units have time, the weights are taken whole (wide_few.hpp).
template <typename T>
constexpr int kPartsOf = sizeof(T) == 2 ? 1 : 3;

// the workspace, cut piece by piece
struct Cutter {
    char *at;
    size_t used = 0;
    void *take(size_t bytes)
    {
        void *p = at ? at + used : nullptr;
        used += round_up(bytes, 256);
        return p;
    }
    void take(Packed &p, int parts) { p.at = static_cast<char *>(take(p.bytes(parts))); }
};

// forward: weights laid out, and rows; lying: bytes of all but the rows, the last, where a call reads those where they lie
struct ForwardPlan {
    Packed a, b;
    WidePlan rows;
    float *shares;
    size_t lying, bytes;
};
// Rows that a product takes where they lie (see WideCall).  (A tile's rows are within 32 bits of each other.)  That takes their pass off and a tenth more time, for
// half lines of memory: 1,000,003 rows 256 -> 256 690 -> 500 us, 8,192 rows 8192 -> 2048 290 -> 280, 2048 -> 2 x 8192 530 -> 565.
template <typename T>
inline bool direct_sizes(int32_t F_in, int n_units) { return sizeof(T) == 2 && F_in % 32 == 0 && n_units <= 128; }
template <typename T>
inline bool direct_rows(const T *X, int64_t ldx, int32_t F_in, int n_units)
{
    return direct_sizes<T>(F_in, n_units) && whole_rows(X, ldx) && ldx <= (1 << 22);
}

// the product of weights, laid out here, and of rows, laid out where they have to be
template <typename T, class Epi>
static int forward_product(const char *fn, const char *name, int64_t n, const T *X, int64_t ldx, int32_t F_in, const float *const (&W)[2], int32_t F_out, const ForwardPlan &p,
                           const Epi &e, hipStream_t s)
{
    constexpr int kP = kPartsOf<T>;
    const ColsPack w = cols_pack<float>(W[0], W[1], F_out, F_in, F_out, true, p.b);
    const RowsPack x = rows_pack<T>(X, nullptr, ldx, n, F_in, false, p.a);
    const bool direct = direct_rows(X, ldx, F_in, p.b.rbs);
    {
        const int cols = blocks_of(w);
        TMA_TIMED("wide_layouts", s);
        hipLaunchKernelGGL((forward_layouts_kernel<T, kP>), dim3(unsigned(cols + (direct ? 0 : blocks_of(x)))), dim3(kPackThreads), 0, s, w, x, cols);
        if (int rc = check_launch(fn)) return rc;
    }
    WideCall q{};
    q.a = p.a;
    q.b = p.b;
    if constexpr (sizeof(T) == 2)
        if (direct) {
            q.a.at = const_cast<char *>(reinterpret_cast<const char *>(X));
            q.lda = ldx;
            q.rows = n;
            return launch_rows<T, kLying>(name, q, p.rows, p.shares, n, F_out, e, s);
        }
    return launch_rows<T, kUnits_>(name, q, p.rows, p.shares, n, F_out, e, s);
}

template <typename T>
inline ForwardPlan plan_forward(int64_t n, int32_t F_in, int32_t F_out, int sides, bool reads, void *ws)
{
    ForwardPlan p{};
    if (n <= kFewMost) {      // nothing is laid out
        p.bytes = p.lying = round_up(plan_few(n, F_in, F_out, sides, sizeof(T)).bytes, 256);
        return p;
    }
    p.a = packed_shape(n, F_in);
    p.b = packed_shape(F_out, F_in);
    p.b.rbs *= sides;
    Cutter cut{static_cast<char *>(ws)};
    cut.take(p.b, kPartsOf<T>);
    p.rows = plan_rows(n, p.b, reads, sizeof(T) == 4);
    p.shares = static_cast<float *>(cut.take(row_shares(p.rows, n, p.b)));
    p.lying = cut.used;
    cut.take(p.a, kPartsOf<T>);
    p.bytes = cut.used;
    return p;
}

struct BackwardPlan {
    Packed d_cols, x_cols, w_rows;
    int padded, row_blocks, parts_c;
    WidePlan weight, data;
    float *sums, *partial, *shares;
    size_t bytes;
};
// exact: the gradients of the pre-activations are bf16 as they come (no activation on bf16 rows); reads: something is added to dX (no matter for the sizes:
// only tiles enough for large ones, which have no ranges, depend on it)
template <typename T>
inline BackwardPlan plan_backward(int64_t n, int32_t F_in, int32_t F_out, int sides, bool exact, bool need_dX, bool reads, void *ws)
{
    BackwardPlan p;
    p.padded = int(round_up(size_t(F_out), 32));
    p.parts_c = sizeof(T) == 4 ? 3 : exact ? 1 : 2;
    p.d_cols = packed_shape(int64_t(sides) * p.padded, n);
    p.x_cols = packed_shape(F_in, n);
    p.w_rows = packed_shape(F_in, int64_t(sides) * p.padded);
    p.weight = plan_weight(p.x_cols, p.d_cols, sizeof(T) == 4);
    const int strips = int(ceil_div(F_out, 64));
    int64_t blocks = ceil_div(4096, strips);
    if (blocks > ceil_div(n > 0 ? n : 1, 32)) blocks = ceil_div(n > 0 ? n : 1, 32);
    p.row_blocks = int(blocks);
    Cutter cut{static_cast<char *>(ws)};
    cut.take(p.d_cols, p.parts_c);
    cut.take(p.x_cols, kPartsOf<T>);
    p.sums = static_cast<float *>(cut.take(size_t(p.row_blocks) * size_t(sides) * size_t(p.padded) * 4));
    p.partial = p.weight.splits > 1 ? static_cast<float *>(cut.take(size_t(p.weight.splits) * size_t(sides) * size_t(F_in) * size_t(F_out) * 4)) : nullptr;
    p.shares = nullptr;
    if (need_dX) {
        cut.take(p.w_rows, kPartsOf<T>);
        p.data = plan_rows(n, p.w_rows, reads, sizeof(T) == 4);
        p.shares = static_cast<float *>(cut.take(row_shares(p.data, n, p.w_rows)));
    }
    p.bytes = cut.used;
    return p;
}

// dW, db of one matrix or two, and dX + R
template <typename T, int kSides>
static int wide_backward(const char *fn, const char *what, int64_t n, const T *X, int64_t ldx, GradCall<T> g, const float *const (&W)[2], int32_t F_in, float *const (&dW)[2],
                         float *const (&db)[2], T *dX, int64_t ld_dx, const T *R, int64_t ldr, void *ws, hipStream_t s)
{
    const int32_t N = g.N;
    const int64_t cells = int64_t(F_in) * N;
    JoinCall join{nullptr, 0, 0, kSides, 0, 0, cells, {dW[0], dW[1]}, nullptr, 0, 0, N, {db[0], db[1]}};
    if (n == 0) return launch_join(fn, join, s);      // (no ranges: zeros)
    const bool exact = kSides == 1 && g.act == TMA_ACT_NONE;
    const BackwardPlan p = plan_backward<T>(n, F_in, N, kSides, exact, dX != nullptr, R != nullptr, ws);
    g.by_cols = p.d_cols;
    g.sums = db[0] ? p.sums : nullptr;
    g.row_blocks = p.row_blocks;
    {
        const ColsPack x = cols_pack<T>(X, nullptr, ldx, n, F_in, false, p.x_cols);
        const RowsPack w = rows_pack<float>(W[0], kSides == 2 ? W[1] : nullptr, N, F_in, N, true, p.w_rows);
        const int grads = int(ceil_div(N, 64)) * p.row_blocks, cols = blocks_of(x);
        TMA_TIMED("wide_layouts", s);
        const dim3 grid(unsigned(grads + cols + (dX ? blocks_of(w) : 0))), block(256);
        if constexpr (sizeof(T) == 4) hipLaunchKernelGGL((backward_layouts_kernel<T, kSides, 3>), grid, block, 0, s, g, x, w, grads, cols);
        else if constexpr (kSides == 2) hipLaunchKernelGGL((backward_layouts_kernel<T, kSides, 2>), grid, block, 0, s, g, x, w, grads, cols);
        else if (exact) hipLaunchKernelGGL((backward_layouts_kernel<T, kSides, 1>), grid, block, 0, s, g, x, w, grads, cols);
        else hipLaunchKernelGGL((backward_layouts_kernel<T, kSides, 2>), grid, block, 0, s, g, x, w, grads, cols);
        if (int rc = check_launch(fn)) return rc;
    }
    const bool split = p.weight.splits > 1;
    WeightEpilogue we{{split ? p.partial : dW[0], split ? p.partial + cells : dW[1]}, cells * kSides, F_in, N, p.padded, kSides, false};
    we.whole16 = N % 4 == 0 && aligned(we.out[0], 16) && (kSides == 1 || aligned(we.out[1], 16));
    char name[64];
    snprintf(name, sizeof(name), "%s_bwd_weight%s", what, sizeof(T) == 2 ? "_bf16" : "");
    const WideCall weight{p.x_cols, p.d_cols, planes_of(p.parts_c), 0, 0, 8, p.weight.splits, p.weight.split_slabs, 0, 0, p.x_cols.rbs};
    if (int rc = launch_wide<T, kUnits_>(name, weight, p.weight, we, s)) return rc;
    join.partial = p.partial;
    join.ranges = p.weight.splits;
    join.range_stride = cells * kSides;
    join.side_stride = cells;
    join.sums = p.sums;
    join.sum_blocks = p.row_blocks;
    join.padded = p.padded;
    if (int rc = launch_join(fn, join, s)) return rc;
    if (!dX) return TMA_OK;
    snprintf(name, sizeof(name), "%s_bwd_data%s", what, sizeof(T) == 2 ? "_bf16" : "");
    WideCall data{};
    data.a = p.d_cols;
    data.b = p.w_rows;
    auto go = [&](auto streamed) {
        const ResidualEpilogue<T, decltype(streamed)::value> re{nullptr, dX, R, 0, ld_dx, ldr, n, nullptr, F_in, TMA_ACT_NONE, whole_rows(dX, ld_dx), R && whole_rows(R, ldr), false};
        return launch_rows<T, kTurned>(name, data, p.data, p.shares, n, F_in, re, s);
    };
    return past_caches(n, F_in, sizeof(T)) ? go(std::true_type{}) : go(std::false_type{});
}

// every number of a call that asks for a workspace, too
inline bool wide_sizes_ok(int64_t n, int32_t F_in, int32_t F_out) { return n >= 0 && n <= INT32_MAX && F_in >= 1 && F_out >= 1 && F_in <= (1 << 16) && F_out <= (1 << 16); }
// of a forward call; at16: of one whose rows begin at 16 bytes, 2^22 elements apart at most
template <typename T>
inline size_t forward_bytes(int64_t n, int32_t F_in, int32_t F_out, int sides, bool at16)
{
    const ForwardPlan p = plan_forward<T>(n, F_in, F_out, sides, true, nullptr);
    return at16 && direct_sizes<T>(F_in, p.b.rbs) ? p.lying : p.bytes;
}
inline size_t forward_workspace(int64_t n, int32_t F_in, int32_t F_out, int sides, int32_t dtype, bool at16)
{
    if (!wide_sizes_ok(n, F_in, F_out)) return 0;
    return dtype == TMA_BF16 ? forward_bytes<uint16_t>(n, F_in, F_out, sides, at16) : forward_bytes<float>(n, F_in, F_out, sides, at16);
}
inline bool rows_at16(const void *X, int64_t ldx) { return whole_rows(static_cast<const uint16_t *>(X), ldx) && ldx <= (1 << 22); }      // (of bf16: fp32 rows are laid out)
inline bool wide_act_ok(int32_t act) { return act == TMA_ACT_NONE || act == TMA_ACT_RELU || act == TMA_ACT_SILU || act == TMA_ACT_GELU; }
inline int check_wide(const char *fn, int64_t n, int32_t F_in, int32_t F_out, int32_t act, int32_t dtype, const void *ws, size_t ws_bytes, size_t need)
{
    TMA_REQUIRE(n >= 0 && n <= INT32_MAX, TMA_ERR_INVALID_ARG, "%s: n outside [0, 2^31)", fn);
    TMA_REQUIRE(F_in >= 1 && F_out >= 1 && F_in <= (1 << 16) && F_out <= (1 << 16), TMA_ERR_BAD_SHAPE, "%s: F_in=%d F_out=%d", fn, F_in, F_out);
    TMA_REQUIRE(wide_act_ok(act), TMA_ERR_INVALID_ARG, "%s: act %d", fn, act);
    TMA_REQUIRE(dtype == TMA_F32 || dtype == TMA_BF16, TMA_ERR_UNSUPPORTED_DTYPE, "%s: dtype %d", fn, dtype);
    TMA_REQUIRE(!need || (ws && aligned(ws, 256)), TMA_ERR_INVALID_ARG, "%s: workspace NULL or not 256-byte aligned", fn);
    TMA_REQUIRE(ws_bytes >= need, TMA_ERR_WORKSPACE_TOO_SMALL, "%s: workspace %zu < %zu", fn, ws_bytes, need);
    return TMA_OK;
}

}  // namespace tma
