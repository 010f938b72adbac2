// Group norm, channels last, with an activation: the F channels of a row in G groups of cg = F / G neighbours; statistics per
// (segment of rows, group), in fp32:
//     xh = (x - mean) rstd,  rstd = 1 / sqrt(var + eps),  y = gamma xh + beta,  out = act(y)
//     dz = dout act'(y),  dgamma = sum dz xh,  dbeta = sum dz,  dslope = sum over y <= 0 of dout y
//     dx = rstd (gamma dz - m1 - xh m2),   m1, m2 = means over the (segment, group) of gamma dz and gamma dz xh
// A segment is a row by itself, a run of R rows, or a range of given offsets.  HBM bound: a few operations an element.
//
// Lanes.  W lanes (a power of two, so that sums over a group are xor-shuffles) share a group's channels in pieces of E elements, the widest
// load that channels, pitches and addresses allow (two groups of four bf16 channels: 8 bytes), neighbouring groups in neighbouring
// lanes: G W lanes cover a row, a wavefront reads whole lines, and a lane keeps its columns, gamma, beta and the sums of dgamma
// and dbeta in registers.  No group takes lanes from another, so that any number of channels goes (up to 1024 a group).
//
// Rows by themselves: one pass, several rows of a lane in flight.  1,000,000 rows of 256 channels in 32 groups, bf16, with PReLU 209 us (1.02 GB, 4.9 TB/s);
// backward of 604,000 with SiLU 187 us (928 MB, 5.0 TB/s): what a copy reaches.
// Longer segments: a tile is a run of rows that the lanes walk down, segment after segment.  First pass: count, mean and sum of
// squares about it of every (tile, segment) pair, whose number tile + segment is its own; a second, small kernel joins them per
// segment in order (Chan, Golub, LeVeque: updating formulas for pairs of samples; sums of squares of raw values would lose the
// variance of data far from zero); third pass: the result.  No length of a segment makes a block's work: one segment of all
// rows and 100,000 of a few rows run alike.  Nothing is an atomic: the same bits every time.  Four passes over X in a forward and backward (statistics
// need the whole segment first): 125,237 rows of 128 in 8 groups, fp32, 1,200 segments, us: moments 24, apply 32, sums 38, backward 39 (64, 128, 128 and
// 192 MB moved: 2.7 to 5 TB/s; a tile's search of its segment and two chunks of loads follow each other), joins 5 to 6 each.
#include "kernels.hpp"

#include <type_traits>

namespace tma {

constexpr int kGnThreads = 256;
constexpr int kGnMaxChannels = 1024;          // of a group
constexpr int kGnBlocks = 256 * 8;            // forward: eight blocks fill a compute unit
constexpr int kGnBwdBlocks = 1024;            // backward: as many partial rows of dgamma and dbeta
constexpr int64_t kGnLanes = 256 * 1024;      // lanes that a pass over tiles should have (twice as many, in us as above: 26, 31, 40, 39)
constexpr int kGnChunk = 8;                   // rows of a lane in flight in the first pass

template <int kBytes>
struct RawBits;
template <>
struct RawBits<16> { typedef uint4 type; };
template <>
struct RawBits<8> { typedef uint2 type; };
template <>
struct RawBits<4> { typedef uint32_t type; };
template <>
struct RawBits<2> { typedef uint16_t type; };

// E elements of storage type T with one access
template <typename T, int E>
struct Piece {
    typedef typename RawBits<E * sizeof(T)>::type Raw;
    static __device__ __forceinline__ Raw load(const T *p) { return *reinterpret_cast<const Raw *>(p); }
    static __device__ __forceinline__ void widen(const Raw &r, float (&x)[E])
    {
        if constexpr (sizeof(T) == 2 && E == 1) x[0] = bf16_to_f32(r);
        else {
            uint32_t w[sizeof(Raw) / 4];
            __builtin_memcpy(w, &r, sizeof(Raw));
#pragma unroll
            for (int i = 0; i < int(sizeof(Raw) / 4); ++i) {
                if constexpr (sizeof(T) == 4) x[i] = __uint_as_float(w[i]);
                else {
                    x[2 * i] = __uint_as_float(w[i] << 16);
                    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
                }
            }
        }
    }
    static __device__ __forceinline__ void store(T *p, const float (&x)[E])
    {
        if constexpr (sizeof(T) == 2 && E == 1) *p = f32_to_bf16(x[0]);
        else {
            uint32_t w[sizeof(Raw) / 4];
#pragma unroll
            for (int i = 0; i < int(sizeof(Raw) / 4); ++i) {
                if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(x[i]);
                else w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
            }
            Raw r;
            __builtin_memcpy(&r, w, sizeof(Raw));
            *reinterpret_cast<Raw *>(p) = r;
        }
    }
};

struct GnShape {
    int64_t n;
    int F, G, cg;
    int W;                    // lanes of a group
    int lanes, parts, tpb;    // lanes of a row in a block, blocks that a row takes, rows (or tiles) side by side in a block
    float eps;
    int act;
};

struct GnSegments {
    const int32_t *offsets;   // NULL: runs of `rows` rows
    int64_t rows, count, n;
    int64_t tile_rows, tiles;
    __device__ __forceinline__ int64_t start(int64_t s) const
    {
        if (!offsets) return s * rows;
        const int64_t o = offsets[s];
        return o < 0 ? 0 : o < n ? o : n;
    }
    // the segment of a row, the last that begins at or before it (-1: none); all threads of a block call this with one row, and each
    // step tries as many places as it has threads
    __device__ __forceinline__ int64_t of_block(int64_t row) const
    {
        if (!offsets) return row / rows;
        int64_t lo = -1, hi = count;
        while (hi - lo > 1) {
            const int64_t step = (hi - lo - 1 + kGnThreads - 1) / kGnThreads, p = lo + 1 + int64_t(threadIdx.x) * step;
            const int c = __syncthreads_count(p < hi && start(p) <= row);
            const int64_t first = lo + 1 + (c - 1) * step, next = lo + 1 + c * step;
            if (c > 0) lo = first;
            hi = next < hi ? next : hi;
        }
        return lo;
    }
    // the segment of a row at or behind one that begins at or before it
    __device__ __forceinline__ int64_t of(int64_t row, int64_t s) const
    {
        if (!offsets) return row / rows;
        int64_t d = 1;
        for (; s + d < count && start(s + d) <= row; d *= 2) s += d;
        for (d /= 2; d > 0; d /= 2)
            if (s + d < count && start(s + d) <= row) s += d;
        return s;
    }
};

// A lane's place: its group, its columns, which of the block's rows or tiles.
template <int E, int CPL>
struct GnLane {
    int g, sub, slot, c0;
    bool live;
    bool in[CPL];
    __device__ __forceinline__ GnLane(const GnShape &sh)
    {
        slot = int(threadIdx.x) / sh.lanes;
        const int r = int(blockIdx.y) * kGnThreads + int(threadIdx.x) % sh.lanes;   // (lanes < 256: blockIdx.y = 0)
        g = r / sh.W;
        sub = r % sh.W;
        live = slot < sh.tpb && g < sh.G;
        c0 = g * sh.cg + sub * E;
#pragma unroll
        for (int c = 0; c < CPL; ++c) in[c] = live && (sub + c * sh.W) * E < sh.cg;
    }
    __device__ __forceinline__ int col(const GnShape &sh, int c) const { return c0 + c * sh.W * E; }
    // where a piece is loaded from: a lane without one takes its group's first, so that no branch stands between loads (each would be waited for)
    __device__ __forceinline__ int from(const GnShape &sh, int c) const { return in[c] ? col(sh, c) : g * sh.cg; }
    __device__ __forceinline__ int columns() const
    {
        int k = 0;
#pragma unroll
        for (int c = 0; c < CPL; ++c) k += in[c] ? E : 0;
        return k;
    }
};

__device__ __forceinline__ float lanes_sum(float v, int W)
{
    for (int d = W / 2; d >= 1; d >>= 1) v += __shfl_xor(v, d, kWave);
    return v;
}

// the activation and its derivative at y.  Away from SiLU: y where y > 0, slope y elsewhere (ReLU: zero whatever y is, none: slope 1)
template <bool kSilu, bool kExact>
struct GnAct {
    float slope;
    bool zero;
    __device__ __forceinline__ GnAct(int act, const float *slope_p)
        : slope(act == TMA_ACT_PRELU ? *slope_p : act == TMA_ACT_RELU ? 0.0f : 1.0f), zero(act == TMA_ACT_RELU)
    {
    }
    // kExact (fp32 storage): the library's exponential and division; else the instructions, off by some (2 |y| + 8) 2^-23 of themselves, which bf16 does not
    // hold.  In the sums of dgamma and dbeta, fp32 also for bf16 storage, that is what an element's share may be off by: 2 10^-6 for y of three, where the
    // rounding of the bf16 inputs is 4 10^-3
    static __device__ __forceinline__ float sigmoid(float y)
    {
        if constexpr (kExact) return 1.0f / (1.0f + expf(-y));
        else return __builtin_amdgcn_rcpf(1.0f + __expf(-y));
    }
    __device__ __forceinline__ float value(float y) const
    {
        if constexpr (kSilu) return y * sigmoid(y);
        else return y > 0.0f ? y : zero ? 0.0f : slope * y;
    }
    // g act'(y); what the negative side adds to dslope
    __device__ __forceinline__ float back(float y, float g, float &dslope) const
    {
        if constexpr (kSilu) {
            const float t = sigmoid(y);
            return g * (t * (1.0f + y * (1.0f - t)));
        } else {
            const bool open = y > 0.0f;
            if (!open) dslope += g * y;
            return open ? g : zero ? 0.0f : slope * g;
        }
    }
};

template <int E, int CPL>
__device__ __forceinline__ void load_vector(const float *v, const GnShape &sh, const GnLane<E, CPL> &ln, float (&out)[CPL][E])
{
#pragma unroll
    for (int c = 0; c < CPL; ++c)
#pragma unroll
        for (int i = 0; i < E; ++i) out[c][i] = ln.in[c] ? v[ln.col(sh, c) + i] : 0.0f;
}

// ---- rows by themselves ------------------------------------------------------
// mean and 1 / sqrt(var + eps) of the group spread over W lanes (two passes over registers, as the definition reads)
template <int E, int CPL>
__device__ __forceinline__ void group_stats(const float (&x)[CPL][E], const GnLane<E, CPL> &ln, const GnShape &sh, float inv, float &mu, float &rstd)
{
    float s = 0.0f;
#pragma unroll
    for (int c = 0; c < CPL; ++c)
#pragma unroll
        for (int i = 0; i < E; ++i) s += ln.in[c] ? x[c][i] : 0.0f;
    mu = lanes_sum(s, sh.W) * inv;
    float q = 0.0f;
#pragma unroll
    for (int c = 0; c < CPL; ++c)
#pragma unroll
        for (int i = 0; i < E; ++i) q += ln.in[c] ? (x[c][i] - mu) * (x[c][i] - mu) : 0.0f;
    rstd = 1.0f / sqrtf(lanes_sum(q, sh.W) * inv + sh.eps);
}

template <typename T, int E, int CPL, bool kSilu>
__global__ __launch_bounds__(kGnThreads) void gn_rows_fwd_kernel(GnShape sh, const T *__restrict__ X, int64_t ldx, const float *__restrict__ gamma,
                                                                 const float *__restrict__ beta, const float *__restrict__ slope_p,
                                                                 T *__restrict__ Y, int64_t ldy)
{
    typedef Piece<T, E> P;
    constexpr int U = CPL == 1 ? 4 : 1;      // rows in flight
    const GnLane<E, CPL> ln(sh);
    if (!ln.live) return;
    const GnAct<kSilu, sizeof(T) == 4> act(sh.act, slope_p);
    float ga[CPL][E], be[CPL][E];
    load_vector<E, CPL>(gamma, sh, ln, ga);
    load_vector<E, CPL>(beta, sh, ln, be);
    const float inv = 1.0f / float(sh.cg);
    const int64_t stride = int64_t(gridDim.x) * sh.tpb;
    for (int64_t v0 = int64_t(blockIdx.x) * sh.tpb + ln.slot; v0 < sh.n; v0 += U * stride) {
        typename P::Raw raw[U][CPL];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int c = 0; c < CPL; ++c)
                raw[u][c] = P::load(X + (v0 + u * stride < sh.n ? v0 + u * stride : v0) * ldx + ln.from(sh, c));
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t v = v0 + u * stride;
            if (v >= sh.n) break;
            float x[CPL][E], mu, rstd;
#pragma unroll
            for (int c = 0; c < CPL; ++c) P::widen(raw[u][c], x[c]);
            group_stats<E, CPL>(x, ln, sh, inv, mu, rstd);
#pragma unroll
            for (int c = 0; c < CPL; ++c) {
#pragma unroll
                for (int i = 0; i < E; ++i) x[c][i] = act.value(ga[c][i] * ((x[c][i] - mu) * rstd) + be[c][i]);
                if (ln.in[c]) P::store(Y + v * ldy + ln.col(sh, c), x[c]);
            }
        }
    }
}

// The sums of dgamma, dbeta and dslope of a block, its rows or tiles side by side added in order, into row blockIdx.x of
// partial: [0, F) dgamma, [F, 2F) dbeta, then dslope of each of the row's blocks.
template <int E, int CPL>
__device__ __forceinline__ void store_sums(const GnShape &sh, const GnLane<E, CPL> &ln, const float (&dga)[CPL][E], const float (&dbe)[CPL][E],
                                           float dsl, float *__restrict__ partial)
{
    constexpr int PER = E * CPL;
    __shared__ float red[2 * kGnThreads * PER];
    __shared__ float red_slope[kGnThreads / kWave];
#pragma unroll
    for (int c = 0; c < CPL; ++c)
#pragma unroll
        for (int i = 0; i < E; ++i) {
            red[(2 * (c * E + i)) * kGnThreads + threadIdx.x] = dga[c][i];
            red[(2 * (c * E + i) + 1) * kGnThreads + threadIdx.x] = dbe[c][i];
        }
    dsl = lanes_sum(ln.live ? dsl : 0.0f, kWave);
    if (threadIdx.x % kWave == 0) red_slope[threadIdx.x / kWave] = dsl;
    __syncthreads();
    float *mine = partial + int64_t(blockIdx.x) * (2 * int64_t(sh.F) + sh.parts);
    if (ln.slot == 0) {
#pragma unroll
        for (int c = 0; c < CPL; ++c)
            if (ln.in[c]) {
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    float a = 0.0f, b = 0.0f;
                    for (int t = 0; t < sh.tpb; ++t) {
                        a += red[(2 * (c * E + i)) * kGnThreads + t * sh.lanes + threadIdx.x];
                        b += red[(2 * (c * E + i) + 1) * kGnThreads + t * sh.lanes + threadIdx.x];
                    }
                    mine[ln.col(sh, c) + i] = a;
                    mine[sh.F + ln.col(sh, c) + i] = b;
                }
            }
    }
    if (threadIdx.x == 0) {
        float s = 0.0f;
        for (int w = 0; w < kGnThreads / kWave; ++w) s += red_slope[w];
        mine[2 * int64_t(sh.F) + blockIdx.y] = s;
    }
}

template <typename T, int E, int CPL, bool kSilu>
__global__ __launch_bounds__(kGnThreads) void gn_rows_bwd_kernel(GnShape sh, const T *__restrict__ X, int64_t ldx, const T *dY, int64_t ldd,   // may alias dX
                                                                 const float *__restrict__ gamma, const float *__restrict__ beta,
                                                                 const float *__restrict__ slope_p, T *dX, int64_t ldo, float *__restrict__ partial)
{
    typedef Piece<T, E> P;
    constexpr int U = CPL == 1 ? 2 : 1;
    const GnLane<E, CPL> ln(sh);
    const GnAct<kSilu, sizeof(T) == 4> act(sh.act, slope_p);
    float ga[CPL][E], be[CPL][E], dga[CPL][E], dbe[CPL][E], dsl = 0.0f;
    load_vector<E, CPL>(gamma, sh, ln, ga);
    load_vector<E, CPL>(beta, sh, ln, be);
#pragma unroll
    for (int c = 0; c < CPL; ++c)
#pragma unroll
        for (int i = 0; i < E; ++i) dga[c][i] = dbe[c][i] = 0.0f;
    const float inv = 1.0f / float(sh.cg);
    const int64_t stride = int64_t(gridDim.x) * sh.tpb;
    const int64_t end = ln.live ? sh.n : 0;
    for (int64_t v0 = int64_t(blockIdx.x) * sh.tpb + ln.slot; v0 < end; v0 += U * stride) {
        typename P::Raw rx[U][CPL], rg[U][CPL];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int c = 0; c < CPL; ++c) {
                const int64_t v = v0 + u * stride < end ? v0 + u * stride : v0;
                rx[u][c] = P::load(X + v * ldx + ln.from(sh, c));
                rg[u][c] = P::load(dY + v * ldd + ln.from(sh, c));
            }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t v = v0 + u * stride;
            if (v >= end) break;
            float x[CPL][E], g[CPL][E], mu, rstd;
#pragma unroll
            for (int c = 0; c < CPL; ++c) {
                P::widen(rx[u][c], x[c]);
                P::widen(rg[u][c], g[c]);
            }
            group_stats<E, CPL>(x, ln, sh, inv, mu, rstd);
            float m1 = 0.0f, m2 = 0.0f;
#pragma unroll
            for (int c = 0; c < CPL; ++c)
                if (ln.in[c]) {
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        const float xh = (x[c][i] - mu) * rstd;
                        const float dz = act.back(ga[c][i] * xh + be[c][i], g[c][i], dsl);
                        dga[c][i] += dz * xh;
                        dbe[c][i] += dz;
                        const float dxh = dz * ga[c][i];
                        m1 += dxh;
                        m2 += dxh * xh;
                        x[c][i] = xh;
                        g[c][i] = dxh;
                    }
                }
            m1 = lanes_sum(m1, sh.W) * inv;
            m2 = lanes_sum(m2, sh.W) * inv;
#pragma unroll
            for (int c = 0; c < CPL; ++c) {
#pragma unroll
                for (int i = 0; i < E; ++i) x[c][i] = (g[c][i] - m1 - x[c][i] * m2) * rstd;
                if (ln.in[c]) P::store(dX + v * ldo + ln.col(sh, c), x[c]);
            }
        }
    }
    store_sums<E, CPL>(sh, ln, dga, dbe, dsl, partial);
}

// ---- longer segments -----------------------------------------------------------
// The tiles of a block, U rows of a lane at a time: load(row, end) fetches the rows [row, end) of a chunk, on their way while the segments
// are looked up; use(s, from, to) is what segment s has of them, counted from the chunk's first row; done(tile, s) follows the last of a segment's rows
// in a tile.  By all threads of the block (`live`: those that have columns).
template <int U, class Load, class Use, class Done>
__device__ __forceinline__ void walk_tiles(const GnShape &sh, const GnSegments &sg, int slot, bool live, Load &&load, Use &&use, Done &&done)
{
    for (int64_t t0 = int64_t(blockIdx.x) * sh.tpb; t0 < sg.tiles; t0 += int64_t(gridDim.x) * sh.tpb) {
        const int64_t tile = t0 + slot, first = tile * sg.tile_rows;
        const bool mine = live && tile < sg.tiles;
        const int64_t last = !mine ? first : first + sg.tile_rows < sg.n ? first + sg.tile_rows : sg.n;
        if (mine) load(first, first + U < last ? first + U : last);
        int64_t s = sg.of_block(t0 * sg.tile_rows);
        if (!mine) continue;
        s = sg.of(first, s < 0 ? 0 : s);
        int64_t begin = sg.start(s), end = sg.start(s + 1);
        bool open = false;
        for (int64_t c = first; c < last; c += U) {
            const int64_t stop = c + U < last ? c + U : last;
            if (c > first) load(c, stop);
            int64_t row = c;
            while (s < sg.count && row < stop) {
                const int64_t a = begin > row ? begin : row, b = end < stop ? end : stop;
                if (a < b) {
                    use(s, int(a - c), int(b - c));
                    open = true;
                    row = b;
                } else if (begin >= stop) {
                    break;
                }
                if (end <= stop) {
                    if (open) done(tile, s);
                    open = false;
                    ++s;
                    begin = end;
                    if (s < sg.count) end = sg.start(s + 1);
                }
            }
        }
        if (open) done(tile, s);
    }
}

struct Moments {      // of a sample: its size, mean, sum of squares about it
    float n, mean, m2;
    __device__ __forceinline__ void join(float nb, float mb, float m2b)
    {
        const float both = n + nb;
        if (both > 0.0f) {
            const float d = mb - mean, part = nb / both;
            mean += d * part;
            m2 += m2b + d * d * (n * part);
            n = both;
        }
    }
    __device__ __forceinline__ void join_lanes(int W)
    {
        for (int d = W / 2; d >= 1; d >>= 1) {
            const float nb = __shfl_xor(n, d, kWave), mb = __shfl_xor(mean, d, kWave), qb = __shfl_xor(m2, d, kWave);
            join(nb, mb, qb);
        }
    }
};

// mean and sum of squares of every (tile, segment) pair's groups, at [tile + segment][G]
template <typename T, int E, int CPL>
__global__ __launch_bounds__(kGnThreads) void gn_moments_kernel(GnShape sh, GnSegments sg, const T *__restrict__ X, int64_t ldx, float2 *__restrict__ pairs)
{
    typedef Piece<T, E> P;
    constexpr int U = CPL == 1 ? kGnChunk : 1;
    const GnLane<E, CPL> ln(sh);
    const float columns = float(ln.columns());
    typename P::Raw raw[U][CPL];
    Moments all{0.0f, 0.0f, 0.0f};
    walk_tiles<U>(sh, sg, ln.slot, ln.live,
        [&](int64_t row, int64_t end) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int c = 0; c < CPL; ++c)
                    raw[u][c] = P::load(X + (row + u < end ? row + u : row) * ldx + ln.from(sh, c));
        },
        [&](int64_t, int from, int to) {
            float x[U][CPL][E], sum = 0.0f, sq = 0.0f;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int c = 0; c < CPL; ++c) {
                    P::widen(raw[u][c], x[u][c]);
#pragma unroll
                    for (int i = 0; i < E; ++i) sum += ln.in[c] && u >= from && u < to ? x[u][c][i] : 0.0f;
                }
            const float count = float(to - from) * columns, mean = count > 0.0f ? sum / count : 0.0f;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int c = 0; c < CPL; ++c)
#pragma unroll
                    for (int i = 0; i < E; ++i) sq += ln.in[c] && u >= from && u < to ? (x[u][c][i] - mean) * (x[u][c][i] - mean) : 0.0f;
            all.join(count, mean, sq);
        },
        [&](int64_t tile, int64_t s) {
            all.join_lanes(sh.W);
            if (ln.sub == 0) pairs[(tile + s) * sh.G + ln.g] = make_float2(all.mean, all.m2);
            all = Moments{0.0f, 0.0f, 0.0f};
        });
}

// L lanes per (segment, group): the pairs of its tiles joined, mean and 1 / sqrt(var + eps) out (zeros of a segment without rows)
__global__ __launch_bounds__(kGnThreads) void gn_stats_kernel(GnShape sh, GnSegments sg, const float2 *__restrict__ pairs, float2 *__restrict__ stats, int L)
{
    const int64_t cells = sg.count * sh.G;
    const int l = int(threadIdx.x) % L;
    for (int64_t cell = (int64_t(blockIdx.x) * kGnThreads + threadIdx.x) / L; cell < cells; cell += int64_t(gridDim.x) * kGnThreads / L) {
        const int64_t s = cell / sh.G, begin = sg.start(s), end = sg.start(s + 1);
        Moments all{0.0f, 0.0f, 0.0f};
        if (end > begin) {
            const int64_t last = (end - 1) / sg.tile_rows;
            for (int64_t t = begin / sg.tile_rows + l; t <= last; t += L) {
                const int64_t a = t * sg.tile_rows, b = a + sg.tile_rows;
                const int64_t rows = (b < end ? b : end) - (a > begin ? a : begin);
                const float2 p = pairs[(t + s) * sh.G + cell % sh.G];
                all.join(float(rows) * float(sh.cg), p.x, p.y);
            }
        }
        all.join_lanes(L);
        if (l == 0) stats[cell] = all.n > 0.0f ? make_float2(all.mean, 1.0f / sqrtf(all.m2 / all.n + sh.eps)) : make_float2(0.0f, 0.0f);
    }
}

template <typename T, int E, int CPL, bool kSilu>
__global__ __launch_bounds__(kGnThreads) void gn_apply_kernel(GnShape sh, GnSegments sg, const T *__restrict__ X, int64_t ldx, const float *__restrict__ gamma,
                                                              const float *__restrict__ beta, const float *__restrict__ slope_p,
                                                              const float2 *__restrict__ stats, T *__restrict__ Y, int64_t ldy)
{
    typedef Piece<T, E> P;
    constexpr int U = CPL == 1 ? 4 : 1;
    const GnLane<E, CPL> ln(sh);
    const GnAct<kSilu, sizeof(T) == 4> act(sh.act, slope_p);
    float ga[CPL][E], be[CPL][E];
    load_vector<E, CPL>(gamma, sh, ln, ga);
    load_vector<E, CPL>(beta, sh, ln, be);
    typename P::Raw raw[U][CPL];
    float2 st = make_float2(0.0f, 0.0f);
    int64_t of = -1, row0 = 0;
    walk_tiles<U>(sh, sg, ln.slot, ln.live,
        [&](int64_t row, int64_t end) {
            row0 = row;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int c = 0; c < CPL; ++c)
                    raw[u][c] = P::load(X + (row + u < end ? row + u : row) * ldx + ln.from(sh, c));
        },
        [&](int64_t s, int from, int to) {
            if (s != of) st = stats[s * sh.G + ln.g];
            of = s;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int c = 0; c < CPL; ++c)
                    if (ln.in[c] && u >= from && u < to) {
                        float x[E];
                        P::widen(raw[u][c], x);
#pragma unroll
                        for (int i = 0; i < E; ++i) x[i] = act.value(ga[c][i] * ((x[i] - st.x) * st.y) + be[c][i]);
                        P::store(Y + (row0 + u) * ldy + ln.col(sh, c), x);
                    }
        },
        [&](int64_t, int64_t) {});
}

// sums of gamma dz and gamma dz xh of every (tile, segment) pair's groups; dgamma, dbeta, dslope of the block
template <typename T, int E, int CPL, bool kSilu>
__global__ __launch_bounds__(kGnThreads) void gn_sums_kernel(GnShape sh, GnSegments sg, const T *__restrict__ X, int64_t ldx, const T *__restrict__ dY,
                                                             int64_t ldd, const float *__restrict__ gamma, const float *__restrict__ beta,
                                                             const float *__restrict__ slope_p, const float2 *__restrict__ stats,
                                                             float2 *__restrict__ pairs, float *__restrict__ partial)
{
    typedef Piece<T, E> P;
    constexpr int U = CPL == 1 ? 4 : 1;
    const GnLane<E, CPL> ln(sh);
    const GnAct<kSilu, sizeof(T) == 4> act(sh.act, slope_p);
    float ga[CPL][E], be[CPL][E], dga[CPL][E], dbe[CPL][E], dsl = 0.0f;
    load_vector<E, CPL>(gamma, sh, ln, ga);
    load_vector<E, CPL>(beta, sh, ln, be);
#pragma unroll
    for (int c = 0; c < CPL; ++c)
#pragma unroll
        for (int i = 0; i < E; ++i) dga[c][i] = dbe[c][i] = 0.0f;
    typename P::Raw rx[U][CPL], rg[U][CPL];
    float2 st = make_float2(0.0f, 0.0f);
    float s1 = 0.0f, s2 = 0.0f;
    int64_t of = -1;
    walk_tiles<U>(sh, sg, ln.slot, ln.live,
        [&](int64_t row, int64_t end) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int c = 0; c < CPL; ++c) {
                    const int64_t v = row + u < end ? row + u : row;
                    rx[u][c] = P::load(X + v * ldx + ln.from(sh, c));
                    rg[u][c] = P::load(dY + v * ldd + ln.from(sh, c));
                }
        },
        [&](int64_t s, int from, int to) {
            if (s != of) st = stats[s * sh.G + ln.g];
            of = s;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int c = 0; c < CPL; ++c)
                    if (ln.in[c] && u >= from && u < to) {
                        float x[E], g[E];
                        P::widen(rx[u][c], x);
                        P::widen(rg[u][c], g);
#pragma unroll
                        for (int i = 0; i < E; ++i) {
                            const float xh = (x[i] - st.x) * st.y;
                            const float dz = act.back(ga[c][i] * xh + be[c][i], g[i], dsl);
                            dga[c][i] += dz * xh;
                            dbe[c][i] += dz;
                            s1 += dz * ga[c][i];
                            s2 += dz * ga[c][i] * xh;
                        }
                    }
        },
        [&](int64_t tile, int64_t s) {
            s1 = lanes_sum(s1, sh.W);
            s2 = lanes_sum(s2, sh.W);
            if (ln.sub == 0) pairs[(tile + s) * sh.G + ln.g] = make_float2(s1, s2);
            s1 = s2 = 0.0f;
        });
    store_sums<E, CPL>(sh, ln, dga, dbe, dsl, partial);
}

// m1, m2 of every (segment, group)
__global__ __launch_bounds__(kGnThreads) void gn_means_kernel(GnShape sh, GnSegments sg, const float2 *__restrict__ pairs, float2 *__restrict__ means, int L)
{
    const int64_t cells = sg.count * sh.G;
    const int l = int(threadIdx.x) % L;
    for (int64_t cell = (int64_t(blockIdx.x) * kGnThreads + threadIdx.x) / L; cell < cells; cell += int64_t(gridDim.x) * kGnThreads / L) {
        const int64_t s = cell / sh.G, begin = sg.start(s), end = sg.start(s + 1);
        float a = 0.0f, b = 0.0f;
        if (end > begin) {
            const int64_t last = (end - 1) / sg.tile_rows;
            for (int64_t t = begin / sg.tile_rows + l; t <= last; t += L) {
                const float2 p = pairs[(t + s) * sh.G + cell % sh.G];
                a += p.x;
                b += p.y;
            }
        }
        a = lanes_sum(a, L);
        b = lanes_sum(b, L);
        const float count = float(end > begin ? end - begin : 1) * float(sh.cg);
        if (l == 0) means[cell] = make_float2(a / count, b / count);
    }
}

template <typename T, int E, int CPL, bool kSilu>
__global__ __launch_bounds__(kGnThreads) void gn_apply_bwd_kernel(GnShape sh, GnSegments sg, const T *__restrict__ X, int64_t ldx, const T *dY, int64_t ldd,   // may alias dX
                                                                  const float *__restrict__ gamma, const float *__restrict__ beta,
                                                                  const float *__restrict__ slope_p, const float2 *__restrict__ stats,
                                                                  const float2 *__restrict__ means, T *dX, int64_t ldo)
{
    typedef Piece<T, E> P;
    constexpr int U = CPL == 1 ? 4 : 1;
    const GnLane<E, CPL> ln(sh);
    const GnAct<kSilu, sizeof(T) == 4> act(sh.act, slope_p);
    float ga[CPL][E], be[CPL][E], unused = 0.0f;
    load_vector<E, CPL>(gamma, sh, ln, ga);
    load_vector<E, CPL>(beta, sh, ln, be);
    typename P::Raw rx[U][CPL], rg[U][CPL];
    float2 st = make_float2(0.0f, 0.0f), m = st;
    int64_t of = -1, row0 = 0;
    walk_tiles<U>(sh, sg, ln.slot, ln.live,
        [&](int64_t row, int64_t end) {
            row0 = row;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int c = 0; c < CPL; ++c) {
                    const int64_t v = row + u < end ? row + u : row;
                    rx[u][c] = P::load(X + v * ldx + ln.from(sh, c));
                    rg[u][c] = P::load(dY + v * ldd + ln.from(sh, c));
                }
        },
        [&](int64_t s, int from, int to) {
            if (s != of) {
                st = stats[s * sh.G + ln.g];
                m = means[s * sh.G + ln.g];
            }
            of = s;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int c = 0; c < CPL; ++c)
                    if (ln.in[c] && u >= from && u < to) {
                        float x[E], g[E];
                        P::widen(rx[u][c], x);
                        P::widen(rg[u][c], g);
#pragma unroll
                        for (int i = 0; i < E; ++i) {
                            const float xh = (x[i] - st.x) * st.y;
                            const float dz = act.back(ga[c][i] * xh + be[c][i], g[i], unused);
                            x[i] = (dz * ga[c][i] - m.x - xh * m.y) * st.y;
                        }
                        P::store(dX + (row0 + u) * ldo + ln.col(sh, c), x);
                    }
        },
        [&](int64_t, int64_t) {});
}

// dgamma, dbeta, dslope from the blocks' rows: 16 columns a block, 64 slices of the rows each, combined in order
constexpr int kFinCols = 16, kFinSlices = 64;

__global__ __launch_bounds__(kFinCols *kFinSlices) void gn_finish_kernel(int nb, int F, int parts, const float *__restrict__ partial, float *__restrict__ dgamma,
                                                                        float *__restrict__ dbeta, float *__restrict__ dslope)
{
    __shared__ float part[kFinSlices][kFinCols];
    const int64_t width = 2 * int64_t(F) + parts;
    const int c = threadIdx.x % kFinCols, slice = threadIdx.x / kFinCols;
    const int64_t j = int64_t(blockIdx.x) * kFinCols + c;
    const int per = (nb + kFinSlices - 1) / kFinSlices, b0 = slice * per, b1 = b0 + per < nb ? b0 + per : nb;
    const int cells = j < 2 * int64_t(F) ? 1 : j == 2 * int64_t(F) ? parts : 0;
    float s0 = 0.0f, s1 = 0.0f, s2 = 0.0f, s3 = 0.0f;
    for (int q = 0; q < cells; ++q) {
        const float *p = partial + j + q;
        int b = b0;
        for (; b + 3 < b1; b += 4) {
            s0 += p[int64_t(b) * width];
            s1 += p[int64_t(b + 1) * width];
            s2 += p[int64_t(b + 2) * width];
            s3 += p[int64_t(b + 3) * width];
        }
        for (; b < b1; ++b) s0 += p[int64_t(b) * width];
    }
    part[slice][c] = (s0 + s1) + (s2 + s3);
    __syncthreads();
    if (slice == 0 && cells > 0) {
        float s = 0.0f;
        for (int k = 0; k < kFinSlices; ++k) s += part[k][c];
        if (j < F) dgamma[j] = s;
        else if (j < 2 * int64_t(F)) dbeta[j - F] = s;
        else if (dslope) *dslope = s;
    }
}

// ---- host ----------------------------------------------------------------------
static int pow2_at_least(int64_t v, int most)
{
    int p = 1;
    while (p < v && p < most) p *= 2;
    return p;
}

// E: the widest piece that channels, pitches and addresses allow
static int piece_elements(int cg, size_t elem, std::initializer_list<const void *> ptrs, std::initializer_list<int64_t> pitches)
{
    int E = int(16 / elem);
    for (; E > 1; E /= 2) {
        bool ok = cg % E == 0;
        for (const void *p : ptrs) ok = ok && aligned(p, size_t(E) * elem);
        for (int64_t ld : pitches) ok = ok && ld % E == 0;
        if (ok) break;
    }
    return E;
}

static GnShape make_shape(int64_t n, int F, int G, int E, float eps, int act)
{
    GnShape sh;
    sh.n = n;
    sh.F = F;
    sh.G = G;
    sh.cg = F / G;
    sh.W = pow2_at_least(sh.cg / E, kWave);
    const int64_t row = int64_t(G) * sh.W;
    sh.lanes = row < kGnThreads ? int(row) : kGnThreads;
    sh.parts = int(ceil_div(row, kGnThreads));
    sh.tpb = kGnThreads / sh.lanes;
    sh.eps = eps;
    sh.act = act;
    return sh;
}

// Tiles so that a pass has about kGnLanes lanes at 16-byte pieces (at least a chunk of rows each); the same for any alignment, so
// that the workspace is a function of sizes alone.
static int64_t tile_rows(int64_t n, int F, int G, size_t elem)
{
    const int cg = F / G, E = int(16 / elem);
    const int64_t row = int64_t(G) * pow2_at_least(ceil_div(cg, E), kWave);
    const int64_t want = kGnLanes / row > 0 ? kGnLanes / row : 1;
    const int64_t rows = ceil_div(n > 0 ? n : 1, want);
    return int64_t(round_up(size_t(rows), kGnChunk));
}

static size_t pairs_bytes(int64_t n, int F, int G, int64_t S, size_t elem)
{
    return round_up(size_t(ceil_div(n > 0 ? n : 1, tile_rows(n, F, G, elem)) + S) * size_t(G) * 8, 256);
}

static size_t sums_bytes(int F)      // a row takes at most 2 F lanes (see make_shape), so ceil(2 F / 256) blocks
{
    return round_up(size_t(kGnBwdBlocks) * (2 * size_t(F) + size_t(ceil_div(2 * int64_t(F), kGnThreads))) * 4, 256);
}

// f(type, E, CPL) of the instance for this piece width and number of channels
template <typename T, class Launch>
static void dispatch_piece(int E, int cg, Launch &&f)
{
    auto go = [&](auto e) {
        constexpr int kE = decltype(e)::value;
        if (cg <= kWave * kE) f(T{}, e, std::integral_constant<int, 1>{});
        else f(T{}, e, std::integral_constant<int, kGnMaxChannels / (kWave * kE)>{});
    };
    if constexpr (sizeof(T) == 2)
        if (E == 8) return go(std::integral_constant<int, 8>{});
    if (E == 4) go(std::integral_constant<int, 4>{});
    else if (E == 2) go(std::integral_constant<int, 2>{});
    else go(std::integral_constant<int, 1>{});
}

template <class Launch>
static void dispatch_norm_instance(int32_t dtype, int E, int cg, int act, Launch &&f)
{
    auto with_act = [&](auto t, auto e, auto c) {
        if (act == TMA_ACT_SILU) f(t, e, c, std::integral_constant<bool, true>{});
        else f(t, e, c, std::integral_constant<bool, false>{});
    };
    if (dtype == TMA_F32) dispatch_piece<float>(E, cg, with_act);
    else dispatch_piece<uint16_t>(E, cg, with_act);
}

struct GnCall {
    const char *fn;
    int64_t n;
    int32_t F, G;
    int64_t n_segments;
    const int32_t *segments;
    int64_t rows_per_segment;
    const float *gamma, *beta, *slope;
    float eps;
    int32_t act, dtype;
    bool single() const { return !segments && rows_per_segment == 1; }
};

static int check_call(const GnCall &q)
{
    TMA_REQUIRE(q.n >= 0 && q.n <= INT32_MAX, TMA_ERR_INVALID_ARG, "%s: n outside [0, 2^31)", q.fn);
    TMA_REQUIRE(q.F >= 1 && q.F <= (1 << 20) && q.G >= 1 && q.F % q.G == 0, TMA_ERR_BAD_SHAPE, "%s: F=%d G=%d", q.fn, q.F, q.G);
    TMA_REQUIRE(q.F / q.G <= kGnMaxChannels, TMA_ERR_BAD_SHAPE, "%s: a group of %d channels is beyond %d", q.fn, q.F / q.G, kGnMaxChannels);
    TMA_REQUIRE(q.dtype == TMA_F32 || q.dtype == TMA_BF16, TMA_ERR_UNSUPPORTED_DTYPE, "%s: dtype %d", q.fn, q.dtype);
    TMA_REQUIRE(q.act >= TMA_ACT_NONE && q.act <= TMA_ACT_SILU, TMA_ERR_INVALID_ARG, "%s: act %d", q.fn, q.act);
    TMA_REQUIRE(q.eps >= 0.0f, TMA_ERR_INVALID_ARG, "%s: eps < 0", q.fn);
    TMA_REQUIRE(q.gamma && q.beta && (q.act != TMA_ACT_PRELU || q.slope), TMA_ERR_INVALID_ARG, "%s: gamma / beta / slope is NULL", q.fn);
    if (q.segments) {
        TMA_REQUIRE(q.n_segments >= 1 && q.n_segments <= INT32_MAX, TMA_ERR_INVALID_ARG, "%s: n_segments outside [1, 2^31)", q.fn);
    } else {
        TMA_REQUIRE(q.rows_per_segment >= 1 && q.n % q.rows_per_segment == 0, TMA_ERR_BAD_SHAPE, "%s: %lld rows are no runs of %lld", q.fn, (long long)q.n,
                    (long long)q.rows_per_segment);
    }
    return TMA_OK;
}

static int64_t segment_count(const GnCall &q) { return q.segments ? q.n_segments : q.n / q.rows_per_segment; }

static GnSegments make_segments(const GnCall &q, size_t elem)
{
    GnSegments sg;
    sg.offsets = q.segments;
    sg.rows = q.rows_per_segment;
    sg.count = segment_count(q);
    sg.n = q.n;
    sg.tile_rows = tile_rows(q.n, q.F, q.G, elem);
    sg.tiles = ceil_div(q.n, sg.tile_rows);
    return sg;
}

// Lanes that join a (segment, group): as many as its tiles on average; with given offsets at least eight, since one segment may
// be longer than all others.
static int joining_lanes(const GnSegments &sg)
{
    const int L = pow2_at_least(ceil_div(sg.tiles, sg.count), kWave);
    return sg.offsets && L < 8 ? 8 : L;
}

static unsigned joining_blocks(const GnSegments &sg, int G, int L)
{
    const int64_t want = ceil_div(sg.count * G * L, kGnThreads);
    return unsigned(want < 65536 ? want : 65536);
}

static dim3 tile_grid(const GnShape &sh, int64_t tiles, int64_t most)
{
    int64_t blocks = ceil_div(tiles, sh.tpb);
    if (blocks > most) blocks = most;
    return dim3(unsigned(blocks), unsigned(sh.parts));
}

static size_t elem_size(int32_t dtype) { return dtype == TMA_BF16 ? 2 : 4; }

}  // namespace tma

extern "C" size_t tma_groupnorm_act_fwd_workspace_bytes(int64_t n, int32_t F, int32_t G, int64_t n_segments, int32_t dtype)
{
    using namespace tma;
    if (n < 0 || n > INT32_MAX || F < 1 || F > (1 << 20) || G < 1 || F % G || n_segments < 1 || n_segments > INT32_MAX) return 0;
    return pairs_bytes(n, F, G, n_segments, elem_size(dtype)) + round_up(size_t(n_segments) * size_t(G) * 8, 256);
}

extern "C" int tma_groupnorm_act_fwd(int64_t n, int32_t F, int32_t G, int64_t n_segments, const int32_t *segments, int64_t rows_per_segment,
                                     const void *X, int64_t ldx, const float *gamma, const float *beta, const float *slope, float eps, int32_t act,
                                     int32_t dtype, void *Y_out, int64_t ldy, float *stats_out, void *ws, size_t ws_bytes, tma_stream_t stream)
{
    using namespace tma;
    const GnCall q{"tma_groupnorm_act_fwd", n, F, G, n_segments, segments, rows_per_segment, gamma, beta, slope, eps, act, dtype};
    if (int rc = check_call(q)) return rc;
    TMA_REQUIRE(aligned(stats_out, 8), TMA_ERR_INVALID_ARG, "%s: stats_out is not 8-byte aligned", q.fn);
    const int64_t S = segment_count(q);
    if (!q.single() && S > 0) {
        TMA_REQUIRE(ws && aligned(ws, 256), TMA_ERR_INVALID_ARG, "%s: workspace NULL or not 256-byte aligned", q.fn);
        TMA_REQUIRE(ws_bytes >= tma_groupnorm_act_fwd_workspace_bytes(n, F, G, S, dtype), TMA_ERR_WORKSPACE_TOO_SMALL, "%s: workspace too small", q.fn);
    }
    TMA_REQUIRE(n == 0 || (X && Y_out && X != Y_out), TMA_ERR_INVALID_ARG, "%s: X or Y_out is NULL, or they are one", q.fn);
    TMA_REQUIRE(n == 0 || (ldx >= F && ldy >= F), TMA_ERR_BAD_SHAPE, "%s: a leading dimension is below F", q.fn);
    if (S == 0 || (n == 0 && q.single())) return TMA_OK;
    const size_t elem = elem_size(dtype);
    const int E = piece_elements(F / G, elem, {X, Y_out}, {ldx, ldy});
    const GnShape sh = make_shape(n, F, G, E, eps, act);
    hipStream_t s = as_stream(stream);
    if (q.single()) {
        TMA_TIMED(dtype == TMA_BF16 ? "gn_rows_fwd_bf16" : "gn_rows_fwd_f32", s);
        dispatch_norm_instance(dtype, E, sh.cg, act, [&](auto t, auto e, auto c, auto silu) {
            typedef decltype(t) T;
            hipLaunchKernelGGL((gn_rows_fwd_kernel<T, decltype(e)::value, decltype(c)::value, decltype(silu)::value>), tile_grid(sh, n, kGnBlocks),
                               dim3(kGnThreads), 0, s, sh, static_cast<const T *>(X), ldx, gamma, beta, slope, static_cast<T *>(Y_out), ldy);
        });
        return check_launch(q.fn);
    }
    const GnSegments sg = make_segments(q, elem);
    float2 *pairs = static_cast<float2 *>(ws);
    float2 *stats = stats_out ? reinterpret_cast<float2 *>(stats_out) : reinterpret_cast<float2 *>(static_cast<char *>(ws) + pairs_bytes(n, F, G, S, elem));
    if (n > 0) {
        TMA_TIMED(dtype == TMA_BF16 ? "gn_moments_bf16" : "gn_moments_f32", s);
        auto go = [&](auto t, auto e, auto c) {
            typedef decltype(t) T;
            hipLaunchKernelGGL((gn_moments_kernel<T, decltype(e)::value, decltype(c)::value>), tile_grid(sh, sg.tiles, INT32_MAX), dim3(kGnThreads), 0, s, sh,
                               sg, static_cast<const T *>(X), ldx, pairs);
        };
        if (dtype == TMA_F32) dispatch_piece<float>(E, sh.cg, go);
        else dispatch_piece<uint16_t>(E, sh.cg, go);
        if (int rc = check_launch(q.fn)) return rc;
    }
    {
        const int L = joining_lanes(sg);
        TMA_TIMED("gn_stats", s);
        hipLaunchKernelGGL(gn_stats_kernel, dim3(joining_blocks(sg, G, L)), dim3(kGnThreads), 0, s, sh, sg, pairs, stats, L);
        if (int rc = check_launch(q.fn)) return rc;
    }
    if (n == 0) return TMA_OK;
    TMA_TIMED(dtype == TMA_BF16 ? "gn_apply_bf16" : "gn_apply_f32", s);
    dispatch_norm_instance(dtype, E, sh.cg, act, [&](auto t, auto e, auto c, auto silu) {
        typedef decltype(t) T;
        hipLaunchKernelGGL((gn_apply_kernel<T, decltype(e)::value, decltype(c)::value, decltype(silu)::value>), tile_grid(sh, sg.tiles, INT32_MAX),
                           dim3(kGnThreads), 0, s, sh, sg, static_cast<const T *>(X), ldx, gamma, beta, slope, stats, static_cast<T *>(Y_out), ldy);
    });
    return check_launch(q.fn);
}

extern "C" size_t tma_groupnorm_act_bwd_workspace_bytes(int64_t n, int32_t F, int32_t G, int64_t n_segments, int32_t dtype)
{
    using namespace tma;
    if (n < 0 || n > INT32_MAX || F < 1 || F > (1 << 20) || G < 1 || F % G || n_segments < 1 || n_segments > INT32_MAX) return 0;
    return sums_bytes(F) + pairs_bytes(n, F, G, n_segments, elem_size(dtype)) + round_up(size_t(n_segments) * size_t(G) * 8, 256);
}

extern "C" int tma_groupnorm_act_bwd(int64_t n, int32_t F, int32_t G, int64_t n_segments, const int32_t *segments, int64_t rows_per_segment,
                                     const void *X, int64_t ldx, const void *dY, int64_t ldd, const float *gamma, const float *beta, const float *slope,
                                     float eps, int32_t act, int32_t dtype, const float *stats, void *dX_out, int64_t ld_dx, float *dgamma, float *dbeta,
                                     float *dslope, void *ws, size_t ws_bytes, tma_stream_t stream)
{
    using namespace tma;
    const GnCall q{"tma_groupnorm_act_bwd", n, F, G, n_segments, segments, rows_per_segment, gamma, beta, slope, eps, act, dtype};
    if (int rc = check_call(q)) return rc;
    TMA_REQUIRE(dgamma && dbeta && (act != TMA_ACT_PRELU || dslope), TMA_ERR_INVALID_ARG, "%s: gradient output is NULL", q.fn);
    const int64_t S = segment_count(q);
    const size_t elem = elem_size(dtype);
    TMA_REQUIRE(ws && aligned(ws, 256), TMA_ERR_INVALID_ARG, "%s: workspace NULL or not 256-byte aligned", q.fn);
    const size_t need = q.single() || S == 0 ? sums_bytes(F) : tma_groupnorm_act_bwd_workspace_bytes(n, F, G, S, dtype);
    TMA_REQUIRE(ws_bytes >= need, TMA_ERR_WORKSPACE_TOO_SMALL, "%s: workspace too small", q.fn);
    TMA_REQUIRE(n == 0 || (X && dY && dX_out && dX_out != X), TMA_ERR_INVALID_ARG, "%s: X, dY or dX_out is NULL, or dX_out is X", q.fn);
    TMA_REQUIRE(n == 0 || (ldx >= F && ldd >= F && ld_dx >= F), TMA_ERR_BAD_SHAPE, "%s: a leading dimension is below F", q.fn);
    TMA_REQUIRE(dY != dX_out || ldd == ld_dx, TMA_ERR_BAD_SHAPE, "%s: in place the leading dimensions are equal", q.fn);
    TMA_REQUIRE(q.single() || S == 0 || (stats && aligned(stats, 8)), TMA_ERR_INVALID_ARG, "%s: stats is NULL or not 8-byte aligned", q.fn);
    const int E = piece_elements(F / G, elem, {X, dY, dX_out}, {ldx, ldd, ld_dx});
    const GnShape sh = make_shape(n, F, G, E, eps, act);
    hipStream_t s = as_stream(stream);
    float *partial = static_cast<float *>(ws);
    int nb = 0;
    if (n > 0 && q.single()) {
        const dim3 grid = tile_grid(sh, n, kGnBwdBlocks);
        nb = int(grid.x);
        TMA_TIMED(dtype == TMA_BF16 ? "gn_rows_bwd_bf16" : "gn_rows_bwd_f32", s);
        dispatch_norm_instance(dtype, E, sh.cg, act, [&](auto t, auto e, auto c, auto silu) {
            typedef decltype(t) T;
            hipLaunchKernelGGL((gn_rows_bwd_kernel<T, decltype(e)::value, decltype(c)::value, decltype(silu)::value>), grid, dim3(kGnThreads), 0, s, sh,
                               static_cast<const T *>(X), ldx, static_cast<const T *>(dY), ldd, gamma, beta, slope, static_cast<T *>(dX_out), ld_dx, partial);
        });
        if (int rc = check_launch(q.fn)) return rc;
    } else if (n > 0) {
        const GnSegments sg = make_segments(q, elem);
        const float2 *st = reinterpret_cast<const float2 *>(stats);
        float2 *pairs = reinterpret_cast<float2 *>(static_cast<char *>(ws) + sums_bytes(F));
        float2 *means = reinterpret_cast<float2 *>(static_cast<char *>(ws) + sums_bytes(F) + pairs_bytes(n, F, G, S, elem));
        const dim3 grid = tile_grid(sh, sg.tiles, kGnBwdBlocks);
        nb = int(grid.x);
        {
            TMA_TIMED(dtype == TMA_BF16 ? "gn_sums_bf16" : "gn_sums_f32", s);
            dispatch_norm_instance(dtype, E, sh.cg, act, [&](auto t, auto e, auto c, auto silu) {
                typedef decltype(t) T;
                hipLaunchKernelGGL((gn_sums_kernel<T, decltype(e)::value, decltype(c)::value, decltype(silu)::value>), grid, dim3(kGnThreads), 0, s, sh, sg,
                                   static_cast<const T *>(X), ldx, static_cast<const T *>(dY), ldd, gamma, beta, slope, st, pairs, partial);
            });
            if (int rc = check_launch(q.fn)) return rc;
        }
        {
            const int L = joining_lanes(sg);
            TMA_TIMED("gn_means", s);
            hipLaunchKernelGGL(gn_means_kernel, dim3(joining_blocks(sg, G, L)), dim3(kGnThreads), 0, s, sh, sg, pairs, means, L);
            if (int rc = check_launch(q.fn)) return rc;
        }
        TMA_TIMED(dtype == TMA_BF16 ? "gn_apply_bwd_bf16" : "gn_apply_bwd_f32", s);
        dispatch_norm_instance(dtype, E, sh.cg, act, [&](auto t, auto e, auto c, auto silu) {
            typedef decltype(t) T;
            hipLaunchKernelGGL((gn_apply_bwd_kernel<T, decltype(e)::value, decltype(c)::value, decltype(silu)::value>), tile_grid(sh, sg.tiles, INT32_MAX),
                               dim3(kGnThreads), 0, s, sh, sg, static_cast<const T *>(X), ldx, static_cast<const T *>(dY), ldd, gamma, beta, slope, st, means,
                               static_cast<T *>(dX_out), ld_dx);
        });
        if (int rc = check_launch(q.fn)) return rc;
    }
    TMA_TIMED("gn_finish", s);
    hipLaunchKernelGGL(gn_finish_kernel, dim3(unsigned(ceil_div(2 * int64_t(F) + 1, kFinCols))), dim3(kFinCols * kFinSlices), 0, s, nb, F, sh.parts, partial, dgamma, dbeta, dslope);
    return check_launch(q.fn);
}
