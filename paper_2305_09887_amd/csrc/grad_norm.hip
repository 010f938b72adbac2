// The global norm of a model's gradients, many tensors at once, and clipping by it:
//     norm = sqrt(sum over all tensors of g^2),  out = g * c,  c = norm > max_norm ? max_norm / norm : 1.
// A list of tensors goes to the kernels as their arguments, kListed at a time: no table in device memory, no copy of one, nothing that a captured graph
// could find changed.  A tensor is cut into chunks, blocks take every grid-th chunk of the list and keep its squares' sum in 64 bits: the squares of
// fp32 values are exact there and neither overflow nor vanish, and the vector units have the time (two instructions for four bytes).  Sums are joined in a
// fixed order; clipping's second kernel does so in every block, and takes a list's chunks from the last to the first, since the last were just read and a
// cache may still have them.  Lists go first to last both times: of 400 M bf16 values in three the second pass reads from memory what the first did (counted: 828 MB
// and 817).  Bound by memory: a gradient is read once, and once more and written where it is clipped.  400 M bf16 values in one tensor 443 us, 5.4 TB/s; 200 tensors
// that begin at whole lines, two lists, 483; 290 of odd lengths, three lists, whose pieces of 1 KB lie across lines, 530.
#include "kernels.hpp"

#include <algorithm>
#include <cstdlib>

namespace tma {

constexpr int kListed = 128, kNormBlocks = 2048, kNormThreads = 256;
template <typename T>
constexpr int kChunk = (1 << 16) / sizeof(T);      // 64 KB: the search for its tensor takes a microsecond

struct GradTensors {
    const void *in[kListed];
    int64_t size[kListed];
    int first[kListed];        // chunks before it
    int count, chunks;
};
struct GradOutputs {
    void *out[kListed];
};

// the tensor that chunk c is of: the last that begins at or before it
__device__ __forceinline__ int tensor_of(const GradTensors &q, int c)
{
    const int lane = threadIdx.x & 63;
    const uint64_t low = __ballot(lane < q.count && q.first[lane] <= c), high = __ballot(lane + 64 < q.count && q.first[lane + 64] <= c);
    return __popcll(low) + __popcll(high) - 1;
}

template <typename T>
__device__ __forceinline__ void add_squares(const T *p, int64_t n, double (&sum)[4])
{
    constexpr int E = 16 / sizeof(T);
    const int t = threadIdx.x;
    int64_t head = (-reinterpret_cast<intptr_t>(p) & 15) / int64_t(sizeof(T));
    head = head < n ? head : n;
    auto one = [&](int64_t i) {
        const double x = std::is_same<T, float>::value ? double(p[i]) : double(__uint_as_float(uint32_t(p[i]) << 16));
        sum[0] = fma(x, x, sum[0]);
    };
    if (t < head) one(t);
    const int64_t pieces = (n - head) / E, tail = head + pieces * E;
    const uint4 *v = reinterpret_cast<const uint4 *>(p + head);
    auto add = [&](const uint4 &w) {
        float x[E];
        Chunk<T>::widen(w, x);
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const double d = x[j];
            sum[j % 4] = fma(d, d, sum[j % 4]);
        }
    };
    int64_t i = t;
    for (; i + 3 * kNormThreads < pieces; i += 4 * kNormThreads) {
        const uint4 a = v[i], b = v[i + kNormThreads], c = v[i + 2 * kNormThreads], d = v[i + 3 * kNormThreads];
        add(a);
        add(b);
        add(c);
        add(d);
    }
    for (; i < pieces; i += kNormThreads) add(v[i]);
    if (tail + t < n) one(tail + t);
}

// the sum over the block's threads, in a fixed order; thread 0 has it
__device__ __forceinline__ double block_sum(double s)
{
    __shared__ double waves[kNormThreads / kWave];
    for (int d = kWave / 2; d; d >>= 1) s += __shfl_down(s, d, kWave);
    if (threadIdx.x % kWave == 0) waves[threadIdx.x / kWave] = s;
    __syncthreads();
    return (waves[0] + waves[1]) + (waves[2] + waves[3]);
}

// partial[block] = its chunks' squares
template <typename T>
__global__ __launch_bounds__(kNormThreads) void grad_squares_kernel(GradTensors q, double *partial)
{
    double sum[4] = {0, 0, 0, 0};
    for (int c = blockIdx.x; c < q.chunks; c += gridDim.x) {
        const int i = __builtin_amdgcn_readfirstlane(tensor_of(q, c));
        const int64_t at = int64_t(c - q.first[i]) * kChunk<T>, left = q.size[i] - at;
        add_squares(static_cast<const T *>(q.in[i]) + at, left < kChunk<T> ? left : kChunk<T>, sum);
    }
    const double all = block_sum((sum[0] + sum[1]) + (sum[2] + sum[3]));
    if (threadIdx.x == 0) partial[blockIdx.x] = all;
}

__device__ __forceinline__ double norm_of(const double *partial, int count)
{
    double s = 0.0;
    for (int i = threadIdx.x; i < count; i += kNormThreads) s += partial[i];
    return sqrt(block_sum(s));
}

__global__ __launch_bounds__(kNormThreads) void grad_norm_kernel(const double *partial, int count, float *norm_out)
{
    const double norm = norm_of(partial, count);
    if (threadIdx.x == 0) *norm_out = float(norm);
}

// In 64 bits: the factor of gradients that exploded, or of a tiny bound, is no normal fp32 number, while its products are.
__device__ __forceinline__ float scaled(float g, double c)
{
    float v = float(double(g) * c);
    asm("" : "+v"(v));      // (of a single value the compiler would round 64 bits to bf16 at once, of a pair it does not: one value, two results)
    return v;
}
template <typename T>
__device__ __forceinline__ void scale_piece(const uint4 &piece, T *out, double c)
{
    float v[16 / sizeof(T)];
    Chunk<T>::widen(piece, v);
#pragma unroll
    for (size_t j = 0; j < 16 / sizeof(T); ++j) v[j] = scaled(v[j], c);
    Chunk<T>::store(out, v);
}
__device__ __forceinline__ void scale_one(const float *in, float *out, double c) { *out = scaled(*in, c); }
__device__ __forceinline__ void scale_one(const uint16_t *in, uint16_t *out, double c) { *out = f32_to_bf16(scaled(bf16_to_f32(*in), c)); }

// first: this launch writes norm_out.  Where the factor is 1 nothing is written in place.
template <typename T>
__global__ __launch_bounds__(kNormThreads) void grad_scale_kernel(GradTensors q, GradOutputs o, const double *partial, int count, double max_norm, bool first,
                                                                  float *norm_out)
{
    constexpr int E = 16 / sizeof(T);
    const double norm = norm_of(partial, count);
    if (first && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = float(norm);
    // (a norm that is NaN makes every gradient NaN)
    const double factor = norm <= max_norm ? 1.0 : max_norm / norm;
    const int t = threadIdx.x;
    for (int b = blockIdx.x; b < q.chunks; b += gridDim.x) {
        const int c = q.chunks - 1 - b;
        const int i = __builtin_amdgcn_readfirstlane(tensor_of(q, c));
        const int64_t at = int64_t(c - q.first[i]) * kChunk<T>, left = q.size[i] - at, n = left < kChunk<T> ? left : kChunk<T>;
        const T *in = static_cast<const T *>(q.in[i]) + at;
        T *out = static_cast<T *>(o.out[i]) + at;
        if (in == out && factor == 1.0) continue;
        int64_t head = 0, pieces = 0;
        if (((reinterpret_cast<intptr_t>(in) ^ reinterpret_cast<intptr_t>(out)) & 15) == 0) {
            head = (-reinterpret_cast<intptr_t>(in) & 15) / int64_t(sizeof(T));
            head = head < n ? head : n;
            pieces = (n - head) / E;
        }
        const uint4 *from = reinterpret_cast<const uint4 *>(in + head);
        T *to = out + head;
        int64_t j = t;
        for (; j + 3 * kNormThreads < pieces; j += 4 * kNormThreads) {
            uint4 w[4];
#pragma unroll
            for (int p = 0; p < 4; ++p) w[p] = from[j + p * kNormThreads];
#pragma unroll
            for (int p = 0; p < 4; ++p) scale_piece(w[p], to + (j + p * kNormThreads) * E, factor);
        }
        for (; j < pieces; j += kNormThreads) scale_piece(from[j], to + j * E, factor);
        for (int64_t i = t; i < n - pieces * E; i += kNormThreads) {
            const int64_t k = i < head ? i : i + pieces * E;
            scale_one(in + k, out + k, factor);
        }
    }
}

// the next of the list's tensors, from `begin` on, as arguments; empty ones are left out.  Returns where the rest begins.
template <typename T>
static int list_tensors(int begin, int n_tensors, const void *const *h_grads, void *const *h_outs, const int64_t *h_sizes, GradTensors &q, GradOutputs &o)
{
    q.count = q.chunks = 0;
    int i = begin;
    for (; i < n_tensors && q.count < kListed; ++i) {
        if (h_sizes[i] == 0) continue;
        const int64_t more = ceil_div(h_sizes[i], kChunk<T>);
        if (q.chunks + more > INT32_MAX / 2) break;     // (one tensor alone is below this: see the checks)
        q.in[q.count] = h_grads[i];
        o.out[q.count] = h_outs ? h_outs[i] : const_cast<void *>(h_grads[i]);
        q.size[q.count] = h_sizes[i];
        q.first[q.count] = q.chunks;
        q.chunks += int(more);
        ++q.count;
    }
    return i;
}

constexpr int kMaxLists = 1 << 10;     // of kListed tensors each, at least
static size_t norm_workspace(int32_t n_tensors) { return round_up(size_t(ceil_div(n_tensors > 0 ? n_tensors : 1, kListed) + 1) * kNormBlocks * sizeof(double), 256); }

template <typename T>
static int grad_norm(const char *fn, int32_t n_tensors, const void *const *h_grads, void *const *h_outs, const int64_t *h_sizes, bool clip, double max_norm, float *norm_out,
                     double *partial, size_t room, hipStream_t s)
{
    GradTensors q;
    GradOutputs o;
    int count = 0;
    for (int at = 0; at < n_tensors;) {
        at = list_tensors<T>(at, n_tensors, h_grads, h_outs, h_sizes, q, o);
        if (!q.count) break;
        const int blocks = q.chunks < kNormBlocks ? q.chunks : kNormBlocks;
        TMA_REQUIRE(size_t(count + blocks) * sizeof(double) <= room, TMA_ERR_WORKSPACE_TOO_SMALL, "%s: workspace for %d sums", fn, count + blocks);
        TMA_TIMED(sizeof(T) == 2 ? "grad_squares_bf16" : "grad_squares", s);
        hipLaunchKernelGGL(grad_squares_kernel<T>, dim3(unsigned(blocks)), dim3(kNormThreads), 0, s, q, partial + count);
        if (int rc = check_launch(fn)) return rc;
        count += blocks;
    }
    if (!clip || count == 0) {
        TMA_TIMED("grad_norm", s);
        hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(kNormThreads), 0, s, partial, count, norm_out);
        return check_launch(fn);
    }
    bool first = true;
    for (int at = 0; at < n_tensors;) {
        at = list_tensors<T>(at, n_tensors, h_grads, h_outs, h_sizes, q, o);
        if (!q.count) break;
        const int blocks = q.chunks < kNormBlocks ? q.chunks : kNormBlocks;
        TMA_TIMED(sizeof(T) == 2 ? "grad_scale_bf16" : "grad_scale", s);
        hipLaunchKernelGGL(grad_scale_kernel<T>, dim3(unsigned(blocks)), dim3(kNormThreads), 0, s, q, o, partial, count, max_norm, first, norm_out);
        if (int rc = check_launch(fn)) return rc;
        first = false;
    }
    return TMA_OK;
}

static int check_grads(const char *fn, int32_t n_tensors, const void *const *h_grads, const void *const *h_outs, const int64_t *h_sizes, int32_t dtype, const float *norm_out,
                       const void *ws, size_t ws_bytes)
{
    TMA_REQUIRE(n_tensors >= 0 && n_tensors <= kMaxLists * kListed, TMA_ERR_INVALID_ARG, "%s: n_tensors=%d outside [0, %d]", fn, n_tensors, kMaxLists * kListed);
    TMA_REQUIRE(dtype == TMA_F32 || dtype == TMA_BF16, TMA_ERR_UNSUPPORTED_DTYPE, "%s: dtype %d", fn, dtype);
    TMA_REQUIRE(norm_out && (n_tensors == 0 || (h_grads && h_sizes)), TMA_ERR_INVALID_ARG, "%s: NULL argument", fn);
    TMA_REQUIRE(ws && aligned(ws, 256), TMA_ERR_INVALID_ARG, "%s: workspace NULL or not 256-byte aligned", fn);
    TMA_REQUIRE(ws_bytes >= norm_workspace(n_tensors), TMA_ERR_WORKSPACE_TOO_SMALL, "%s: workspace %zu < %zu", fn, ws_bytes, norm_workspace(n_tensors));
    const size_t size = dtype == TMA_BF16 ? 2 : 4;
    for (int i = 0; i < n_tensors; ++i) {
        TMA_REQUIRE(h_sizes[i] >= 0 && h_sizes[i] < (int64_t(1) << 43), TMA_ERR_BAD_SHAPE, "%s: size of tensor %d", fn, i);
        if (h_sizes[i] == 0) continue;
        TMA_REQUIRE(h_grads[i] && aligned(h_grads[i], size) && (!h_outs || (h_outs[i] && aligned(h_outs[i], size))), TMA_ERR_INVALID_ARG,
                    "%s: tensor %d is NULL or not aligned to its type", fn, i);
    }
    return TMA_OK;
}

// What is written may share memory with nothing else that the call reads or writes, but a result with its own gradient, in place: results are written while other
// blocks still read gradients (one given twice would be scaled twice, or in part).  Lists in the order of their addresses, as a flat buffer's parts are, and
// apart from the others' need no sorting.
struct Range {
    uintptr_t from, to;
    bool operator<(const Range &b) const { return from < b.from; }
    bool meets(const Range &b) const { return from < b.to && b.from < to; }
};
static int check_apart(const char *fn, int32_t n_tensors, const void *const *h_grads, const void *const *h_outs, const int64_t *h_sizes, size_t size, const float *norm_out)
{
    auto range = [&](const void *const *list, int i) {
        return Range{reinterpret_cast<uintptr_t>(list[i]), reinterpret_cast<uintptr_t>(list[i]) + uintptr_t(h_sizes[i]) * size};
    };
    const void *const *outs = h_outs ? h_outs : h_grads;
    const Range norm{reinterpret_cast<uintptr_t>(norm_out), reinterpret_cast<uintptr_t>(norm_out) + sizeof(float)};
    Range written{UINTPTR_MAX, 0}, read{UINTPTR_MAX, 0};      // by results that are not in place, as gradients
    uintptr_t end = 0, g_end = 0;
    bool ordered = true, on_norm = false;
    for (int i = 0; i < n_tensors; ++i) {
        if (h_sizes[i] == 0) continue;
        const Range r = range(outs, i), g = range(h_grads, i);
        ordered = ordered && r.from >= end && g.from >= g_end;
        end = r.to;
        g_end = g.to;
        on_norm = on_norm || r.meets(norm) || g.meets(norm);
        read = {std::min(read.from, g.from), std::max(read.to, g.to)};
        if (r.from != g.from) written = {std::min(written.from, r.from), std::max(written.to, r.to)};
    }
    TMA_REQUIRE(!on_norm, TMA_ERR_INVALID_ARG, "%s: norm_out overlaps a gradient or a result", fn);
    if (ordered && !(written.from < written.to && written.meets(read))) return TMA_OK;
    Range few[256], *all = n_tensors <= 256 ? few : static_cast<Range *>(malloc(size_t(n_tensors) * sizeof(Range)));
    TMA_REQUIRE(all, TMA_ERR_INVALID_ARG, "%s: no host memory for %d tensors", fn, n_tensors);
    int count = 0;
    for (int i = 0; i < n_tensors; ++i)
        if (h_sizes[i]) all[count++] = range(outs, i);
    std::sort(all, all + count);
    bool apart = true, clear = true;
    for (int i = 1; i < count; ++i) apart = apart && all[i].from >= all[i - 1].to;
    // results that are apart: of those that meet a gradient the first is its own, which then is the only one, or an overlap
    for (int i = 0; apart && clear && i < n_tensors; ++i) {
        if (h_sizes[i] == 0) continue;
        const Range g = range(h_grads, i);
        const Range *first = std::lower_bound(all, all + count, g.from, [](const Range &r, uintptr_t at) { return r.to <= at; });
        clear = first == all + count || !first->meets(g) || (outs[i] == h_grads[i] && first->from == g.from);
    }
    if (all != few) free(all);
    TMA_REQUIRE(apart, TMA_ERR_INVALID_ARG, "%s: two of the results overlap", fn);
    TMA_REQUIRE(clear, TMA_ERR_INVALID_ARG, "%s: a result overlaps a gradient that is not its own, or its own at another place", fn);
    return TMA_OK;
}

}  // namespace tma

extern "C" size_t tma_grad_norm_workspace_bytes(int32_t n_tensors)
{
    using namespace tma;
    return n_tensors < 0 || n_tensors > kMaxLists * kListed ? 0 : norm_workspace(n_tensors);
}

extern "C" int tma_grad_norm(int32_t n_tensors, const void *const *h_grads, const int64_t *h_sizes, int32_t dtype, float *norm_out, void *ws, size_t ws_bytes,
                             tma_stream_t stream)
{
    using namespace tma;
    const char *fn = "tma_grad_norm";
    if (int rc = check_grads(fn, n_tensors, h_grads, nullptr, h_sizes, dtype, norm_out, ws, ws_bytes)) return rc;
    hipStream_t s = as_stream(stream);
    double *partial = static_cast<double *>(ws);
    return dtype == TMA_BF16 ? grad_norm<uint16_t>(fn, n_tensors, h_grads, nullptr, h_sizes, false, 0.0, norm_out, partial, ws_bytes, s)
                             : grad_norm<float>(fn, n_tensors, h_grads, nullptr, h_sizes, false, 0.0, norm_out, partial, ws_bytes, s);
}

extern "C" int tma_grad_clip(int32_t n_tensors, const void *const *h_grads, void *const *h_outs, const int64_t *h_sizes, int32_t dtype, double max_norm, float *norm_out,
                             void *ws, size_t ws_bytes, tma_stream_t stream)
{
    using namespace tma;
    const char *fn = "tma_grad_clip";
    if (int rc = check_grads(fn, n_tensors, h_grads, h_outs, h_sizes, dtype, norm_out, ws, ws_bytes)) return rc;
    TMA_REQUIRE(max_norm >= 0.0, TMA_ERR_INVALID_ARG, "%s: max_norm below 0, or NaN", fn);
    if (int rc = check_apart(fn, n_tensors, h_grads, h_outs, h_sizes, dtype == TMA_BF16 ? 2 : 4, norm_out)) return rc;
    hipStream_t s = as_stream(stream);
    double *partial = static_cast<double *>(ws);
    return dtype == TMA_BF16 ? grad_norm<uint16_t>(fn, n_tensors, h_grads, h_outs, h_sizes, true, max_norm, norm_out, partial, ws_bytes, s)
                             : grad_norm<float>(fn, n_tensors, h_grads, h_outs, h_sizes, true, max_norm, norm_out, partial, ws_bytes, s);
}
