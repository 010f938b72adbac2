// Dropout from the library's counter-based generator (SplitMix64, the one of tma_partition): the mask is a function of a
// seed and an element's place, so nothing of it is stored, and backward makes it again.
//   unit(v, c) = (first_row + v) * ceil(F / 4) + c / 4,  z = SplitMix64(s, unit),  field = bits [16 (c % 4), + 16) of z
//   out = field >= T ? x * 65536 / (65536 - T) : 0,      T = floor(65536 p + 1/2)
// One number serves four elements: its two 64-bit products are 20-odd of a wavefront's vector cycles, which at one number
// per element would be dearer than the memory (8 or 4 bytes an element; 256 units x 64 lanes x 2.4 GHz at 5 TB/s: 60 or 30
// vector instructions an element).  Sixteen bits resolve p to 2^-17; the scale is that of the probability as it is taken, so
// that the mean is kept exactly.  An element that is dropped is zero whatever it was (selected, not multiplied).  2,400,000 rows of 256 in
// bf16 528 us (2.46 GB, 4.65 TB/s), 120,011 of 150 in fp32 32 us (144 MB, 4.5 TB/s): what a copy reaches.
#include "common.hpp"

#include <type_traits>

namespace tma {

constexpr int kDropThreads = 256;
constexpr int kDropRows = 4;           // rows of a thread whose loads are in flight together
constexpr int kDropBlocks = 256 * 8;   // persistent: eight blocks of four wavefronts fill a compute unit

struct DropRule {
    uint64_t seed;
    const int64_t *step;    // NULL, or device memory: the stream of this step is SplitMix64(seed, *step)
    int64_t first_row;
    uint32_t limit;         // T
    float scale;
};

__device__ __forceinline__ float keep_field(float x, uint32_t field, const DropRule &r) { return field >= r.limit ? x * r.scale : 0.0f; }

typedef uint32_t Words4 __attribute__((ext_vector_type(4), aligned(4)));      // 16 bytes at a 4-byte-aligned address

// A thread keeps its piece of columns (16 bytes; without kWords four elements) and walks down the rows, `lanes` threads share a row.  The end of a row
// that is no whole piece is read as one too (what follows is the row's padding or the next row) and stored element by element; in the last
// row it is read so as well.
template <typename T, bool kWords>
__global__ __launch_bounds__(kDropThreads) void dropout_kernel(int64_t n, int F, const T *X, int64_t ldx, DropRule rule, T *Y, int64_t ldy, int lanes)
{
    constexpr int E = kWords ? Chunk<T>::kElems : 4;
    const int units = (F + 3) / 4, pieces = (F + E - 1) / E;
    const int rows_per_block = kDropThreads / lanes;
    const int piece = int(blockIdx.y) * lanes + int(threadIdx.x) % lanes, slot = int(threadIdx.x) / lanes;
    if (piece >= pieces || slot >= rows_per_block) return;
    const uint64_t seed = rule.step ? splitmix64_at(rule.seed, uint64_t(*rule.step)) : rule.seed;
    const int c0 = piece * E, valid = F - c0 < E ? F - c0 : E;
    const int64_t stride = int64_t(gridDim.x) * rows_per_block, extent = (n - 1) * ldx + F;
    // rows in which 16 bytes from the piece on lie in the matrix: all, or all but the last few
    int64_t whole_rows = 0;
    if (kWords && extent - c0 >= E) whole_rows = (extent - c0 - E) / ldx + 1 < n ? (extent - c0 - E) / ldx + 1 : n;

    auto drop = [&](int64_t v, const float (&x)[E], float (&y)[E]) {
#pragma unroll
        for (int u = 0; u < E / 4; ++u) {
            const uint64_t z = splitmix64_at(seed, uint64_t(rule.first_row + v) * uint64_t(units) + uint64_t(c0 / 4 + u));
#pragma unroll
            for (int i = 0; i < 4; ++i) y[4 * u + i] = keep_field(x[4 * u + i], uint32_t(z >> (16 * i)) & 0xFFFFu, rule);
        }
    };
    auto store = [&](int64_t v, const float (&y)[E]) {
        T *out = Y + v * ldy + c0;
        if constexpr (kWords) {
            if (valid == E) {
                Words4 w;
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = sizeof(T) == 4 ? __float_as_uint(y[i]) : pack_bf16(y[2 * i % E], y[(2 * i + 1) % E]);
                *reinterpret_cast<Words4 *>(out) = w;
                return;
            }
        }
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (i < valid) {
                if constexpr (sizeof(T) == 4) out[i] = y[i];
                else out[i] = f32_to_bf16(y[i]);
            }
    };
    int64_t v = int64_t(blockIdx.x) * rows_per_block + slot;
    if constexpr (kWords) {
        for (; v < whole_rows; v += kDropRows * stride) {
            Words4 raw[kDropRows];
#pragma unroll
            for (int j = 0; j < kDropRows; ++j)
                if (v + j * stride < whole_rows) raw[j] = *reinterpret_cast<const Words4 *>(X + (v + j * stride) * ldx + c0);
#pragma unroll
            for (int j = 0; j < kDropRows; ++j)
                if (v + j * stride < whole_rows) {
                    float x[E], y[E];
                    Chunk<T>::widen(make_uint4(raw[j].x, raw[j].y, raw[j].z, raw[j].w), x);
                    drop(v + j * stride, x, y);
                    store(v + j * stride, y);
                }
        }
        // the first of this thread's rows that are left
        const int64_t first = int64_t(blockIdx.x) * rows_per_block + slot;
        v = whole_rows > first ? first + (whole_rows - first + stride - 1) / stride * stride : first;
    }
    for (; v < n; v += stride) {
        float x[E], y[E];
#pragma unroll
        for (int i = 0; i < E; ++i) {
            x[i] = 0.0f;
            if (i < valid) {
                if constexpr (sizeof(T) == 4) x[i] = X[v * ldx + c0 + i];
                else x[i] = bf16_to_f32(X[v * ldx + c0 + i]);
            }
        }
        drop(v, x, y);
        store(v, y);
    }
}

template <typename T>
static int launch_dropout(const char *fn, const char *name, int64_t n, int32_t F, const void *X, int64_t ldx, const DropRule &rule, void *Y,
                          int64_t ldy, hipStream_t s)
{
    const bool words = sizeof(T) == 4 || (aligned(X, 4) && aligned(Y, 4) && ldx % 2 == 0 && ldy % 2 == 0);
    const int E = words ? Chunk<T>::kElems : 4;
    const int pieces = int(ceil_div(F, E)), lanes = pieces < kDropThreads ? pieces : kDropThreads;
    int64_t blocks = ceil_div(n, kDropThreads / lanes);
    if (blocks > kDropBlocks) blocks = kDropBlocks;
    const dim3 grid(unsigned(blocks), unsigned(ceil_div(pieces, lanes)));
    TMA_TIMED(name, s);
    if (words) hipLaunchKernelGGL((dropout_kernel<T, true>), grid, dim3(kDropThreads), 0, s, n, F, static_cast<const T *>(X), ldx, rule, static_cast<T *>(Y), ldy, lanes);
    else hipLaunchKernelGGL((dropout_kernel<T, false>), grid, dim3(kDropThreads), 0, s, n, F, static_cast<const T *>(X), ldx, rule, static_cast<T *>(Y), ldy, lanes);
    return check_launch(fn);
}

static int dropout_run(const char *fn, int64_t n, int32_t F, const void *X, int64_t ldx, double p, uint64_t seed, const int64_t *d_step,
                       int64_t first_row, int32_t dtype, void *Y, int64_t ldy, tma_stream_t stream)
{
    TMA_REQUIRE(n >= 0 && n <= INT32_MAX, TMA_ERR_INVALID_ARG, "%s: n outside [0, 2^31)", fn);
    TMA_REQUIRE(F >= 1 && F <= (1 << 20), TMA_ERR_BAD_SHAPE, "%s: F=%d", fn, F);
    TMA_REQUIRE(p >= 0.0 && p <= 1.0, TMA_ERR_INVALID_ARG, "%s: p outside [0, 1]", fn);
    TMA_REQUIRE(first_row >= 0, TMA_ERR_INVALID_ARG, "%s: first_row < 0", fn);
    TMA_REQUIRE(dtype == TMA_F32 || dtype == TMA_BF16, TMA_ERR_UNSUPPORTED_DTYPE, "%s: dtype %d", fn, dtype);
    TMA_REQUIRE(aligned(d_step, 8), TMA_ERR_INVALID_ARG, "%s: d_step is not 8-byte aligned", fn);
    if (n == 0) return TMA_OK;
    TMA_REQUIRE(X && Y, TMA_ERR_INVALID_ARG, "%s: NULL argument", fn);
    TMA_REQUIRE(ldx >= F && ldy >= F, TMA_ERR_BAD_SHAPE, "%s: a leading dimension is below F", fn);
    TMA_REQUIRE(X != Y || ldx == ldy, TMA_ERR_BAD_SHAPE, "%s: in place the leading dimensions are equal", fn);
    DropRule rule{seed, d_step, first_row, uint32_t(p * 65536.0 + 0.5), 0.0f};
    if (rule.limit < 65536u) rule.scale = float(65536.0 / double(65536u - rule.limit));
    hipStream_t s = as_stream(stream);
    if (dtype == TMA_F32) return launch_dropout<float>(fn, "dropout_f32", n, F, X, ldx, rule, Y, ldy, s);
    return launch_dropout<uint16_t>(fn, "dropout_bf16", n, F, X, ldx, rule, Y, ldy, s);
}

}  // namespace tma

extern "C" int tma_dropout_fwd(int64_t n, int32_t F, const void *X, int64_t ldx, double p, uint64_t seed, const int64_t *d_step,
                               int64_t first_row, int32_t dtype, void *Y_out, int64_t ldy, tma_stream_t stream)
{
    return tma::dropout_run("tma_dropout_fwd", n, F, X, ldx, p, seed, d_step, first_row, dtype, Y_out, ldy, stream);
}

extern "C" int tma_dropout_bwd(int64_t n, int32_t F, const void *dY, int64_t ldy, double p, uint64_t seed, const int64_t *d_step,
                               int64_t first_row, int32_t dtype, void *dX_out, int64_t ldx, tma_stream_t stream)
{
    return tma::dropout_run("tma_dropout_bwd", n, F, dY, ldy, p, seed, d_step, first_row, dtype, dX_out, ldx, stream);
}
