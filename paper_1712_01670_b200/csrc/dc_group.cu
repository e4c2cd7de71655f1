// Group normalisation with an activation, channels last, and its gradients.
//
//   mean, rstd over the pixels of a map and the channels of a group;  xh = (x - mean) rstd,  z = xh gamma + beta,  y = act(z)
//   with dz = dy act'(z), g = dz gamma:  dx = rstd (g - mean(g) - xh mean(g xh)),  dgamma = sum over maps and pixels dz xh,  dbeta = sum dz
//
// What bounds them: memory, one read and one write of the map (two reads and a write for the gradients).
//
// A slice is the columns of a map that a CTA works on: some whole groups, or a piece of one that is wider than a CTA.  A thread has one column (16 bytes of
// each of its rows, or one element where rows are not aligned to 16 bytes) and so one set of weights and of sums.
//
// Sums of squares: each thread takes its values' distances from the first of them, which is one of the n values themselves, so the squares around it are at most n
// times those around the mean, whatever the mean is; threads', CTAs' and chunks' means and squares are then joined by
// M2 = sum M2_i + sum n_i (mean_i - mean)^2, in a fixed order: equal calls give equal bits.
#include <atomic>

#include "dc_quantise.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kMostChunks = 64;

struct GroupArgs {
    const void *x, *dy; void* y;                    // y: the output, or dx
    size_t x_pitch, dy_pitch, y_pitch;
    const float *gamma, *beta;                      // or NULL: ones, zeros
    float *mean, *rstd;                             // [maps][groups]: out (or NULL) of the forward pass, in of the backward pass
    float eps;
    int maps, pixels, channels, groups, per;        // per: channels of a group
    int width, slices, gs, pieces, piece_items;     // columns of a slice; slices of a map; groups of a slice; slices of a group; columns of a group (with pieces)
    int by_width, by_per;                           // slices of at most 16 columns: 65536 / width and / per, rounded up; else 0
    int chunks, rows_per;                           // CTAs to the rows of a slice, and the rows of each
    float2* part;                                   // [maps][chunks * pieces][groups]: mean and squares, or the two sums of a group's gradients
    float* sums;                                    // [maps][chunks][2][channels]: sums of dz and of dz xh; or NULL: not wanted
    bool joined;                                    // (host) they have been
    float *dgamma, *dbeta;                          // of a single map that clusters hold whole: written at once
};

// The columns of a CTA.
struct Place {
    int map, chunk, piece, group0, ngroups, col0, cols, row0, rows;      // col0, cols in columns of VE channels
};
__device__ __forceinline__ int rows_of(const GroupArgs& a, int chunk) { return max(0, min(a.rows_per, a.pixels - chunk * a.rows_per)); }
__device__ __forceinline__ int cols_of(const GroupArgs& a, int piece) { return a.pieces > 1 ? min(a.width, a.piece_items - piece * a.width) : a.width; }
__device__ __forceinline__ Place place_of(const GroupArgs& a)
{
    Place p;
    const int unit = blockIdx.x / a.chunks, slice = unit % a.slices;
    p.chunk = blockIdx.x - unit * a.chunks;
    p.map = unit / a.slices;
    p.piece = a.pieces > 1 ? slice % a.pieces : 0;
    p.group0 = a.pieces > 1 ? slice / a.pieces : slice * a.gs;
    p.ngroups = a.pieces > 1 ? 1 : a.gs;
    p.col0 = a.pieces > 1 ? p.group0 * a.piece_items + p.piece * a.width : slice * a.width;
    p.cols = cols_of(a, p.piece);
    p.row0 = p.chunk * a.rows_per;
    p.rows = rows_of(a, p.chunk);
    return p;
}
__device__ __forceinline__ char* row_at(const void* p, size_t pitch, int64_t row) { return (char*)p + (uint64_t)row * pitch; }

// 1 / (1 + e^-z)
__device__ __forceinline__ float one_and_exp(float z)
{
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.4426950408889634f));
    return 1.f + e;
}
__device__ __forceinline__ float reciprocal(float v)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
// Of four values: an exponential each and, JOINT, one reciprocal for all, 1 / a = bcd / abcd (the unit for both gives 16 results a cycle); where abcd is beyond a number's
// range, or none, each has its own.  Not JOINT: a value's result depends on no other.
template <bool JOINT>
__device__ __forceinline__ void sigmoids(const float2* z, float2* p)
{
    const float2 a = make_float2(one_and_exp(z[0].x), one_and_exp(z[0].y)), c = make_float2(one_and_exp(z[1].x), one_and_exp(z[1].y));
    if (JOINT) {
        const float ab = a.x * a.y, cd = c.x * c.y, t = ab * cd;
        if (t < 1e37f) {
            const float r = reciprocal(t);
            p[0] = mul2(both<float2>(r * cd), make_float2(a.y, a.x));
            p[1] = mul2(both<float2>(r * ab), make_float2(c.y, c.x));
            return;
        }
    }
    p[0] = make_float2(reciprocal(a.x), reciprocal(a.y));
    p[1] = make_float2(reciprocal(c.x), reciprocal(c.y));
}
template <bool JOINT> __device__ __forceinline__ void sigmoids(const float* z, float* p) { p[0] = reciprocal(one_and_exp(z[0])); }

__device__ __forceinline__ float positive(float z) { asm("max.NaN.f32 %0, %0, 0f00000000;" : "+f"(z)); return z; }
__device__ __forceinline__ float2 positive(float2 z) { return make_float2(positive(z.x), positive(z.y)); }
__device__ __forceinline__ float where_positive(float dy, float z) { return z > 0.f ? dy : z != z ? z : 0.f; }
__device__ __forceinline__ float2 where_positive(float2 dy, float2 z) { return make_float2(where_positive(dy.x, z.x), where_positive(dy.y, z.y)); }
// act(z), and dy act'(z), of a column's values, in place
template <int ACT, bool JOINT, int P, typename F>
__device__ __forceinline__ void activate(F (&z)[P])
{
    constexpr int STEP = P > 1 ? 2 : 1;
#pragma unroll
    for (int k = 0; k < P; k += STEP) {
        if (ACT == DC_ACT_SILU) {
            F p[STEP];
            sigmoids<JOINT>(z + k, p);
#pragma unroll
            for (int h = 0; h < STEP; ++h) z[k + h] = mul2(z[k + h], p[h]);
        } else if (ACT == DC_ACT_RELU)
#pragma unroll
            for (int h = 0; h < STEP; ++h) z[k + h] = positive(z[k + h]);
    }
}
template <int ACT, bool JOINT, int P, typename F>
__device__ __forceinline__ void activate_back(F (&dy)[P], const F (&z)[P])
{
    constexpr int STEP = P > 1 ? 2 : 1;
#pragma unroll
    for (int k = 0; k < P; k += STEP) {
        if (ACT == DC_ACT_SILU) {
            F p[STEP];
            sigmoids<JOINT>(z + k, p);
#pragma unroll
            for (int h = 0; h < STEP; ++h) {
                const F zp = mul2(z[k + h], p[h]);                               // p (1 + z (1 - p)) = p + zp - zp p
                dy[k + h] = mul2(dy[k + h], fma2(mul2(zp, both<F>(-1.f)), p[h], add2(p[h], zp)));
            }
        } else if (ACT == DC_ACT_RELU)
#pragma unroll
            for (int h = 0; h < STEP; ++h) dy[k + h] = where_positive(dy[k + h], z[k + h]);
    }
}

__device__ __forceinline__ float lane_of(float v, int) { return v; }
__device__ __forceinline__ float lane_of(float2 v, int k) { return k ? v.y : v.x; }
template <typename F> __device__ __forceinline__ F two(float a, float b);
template <> __device__ __forceinline__ float two<float>(float a, float) { return a; }
template <> __device__ __forceinline__ float2 two<float2>(float a, float b) { return make_float2(a, b); }

// z, the same bits in both passes: each product and sum is rounded by itself, so that what the forward pass has cut off is what the backward pass leaves out.
template <typename F> __device__ __forceinline__ F hat(F x, F minus_mean, F rstd) { return rounded(add2(x, minus_mean), rstd); }
__device__ __forceinline__ float affine(float xh, float g, float b) { return __fadd_rn(__fmul_rn(xh, g), b); }
__device__ __forceinline__ float2 affine(float2 xh, float2 g, float2 b) { return add2(mul2(xh, g), b); }

// Means and squares of the items of a group, joined by a warp: item i has n(i) values; all lanes get the result.
template <typename N, typename M, typename Q>
__device__ __forceinline__ float2 join_items(int items, N n, M mean, Q squares, float total)
{
    const int lane = threadIdx.x & 31;
    float s = 0.f;
    for (int i = lane; i < items; i += 32) s = fmaf(n(i), mean(i), s);
    s = reduce_lanes<Sum>(s, 32);
    const float m = total > 0.f ? s / total : 0.f;
    float q = 0.f;
    for (int i = lane; i < items; i += 32) {
        const float w = n(i), d = mean(i) - m;
        q += w > 0.f ? fmaf(w * d, d, squares(i)) : 0.f;
    }
    return make_float2(m, reduce_lanes<Sum>(q, 32));
}

// Chunks' statistics of a map (k_group_apply's input), of a thread's columns.  ONE: a column's channels belong to one group.
template <typename T, int VE, bool ONE>
__global__ void __launch_bounds__(kThreads) k_group_stats(const GroupArgs a)
{
    typedef Vec<T, VE> V;
    typedef typename V::F F;
    constexpr int P = V::P, IT = ONE ? 1 : VE;       // items (channels or whole columns) of a column
    __shared__ float pm[kThreads * IT], pq[kThreads * IT];
    dc_pdl_wait();
    dc_pdl_release();
    const Place p = place_of(a);
    const int turns = kThreads / p.cols, col = threadIdx.x % p.cols, turn = threadIdx.x / p.cols;
    if (turn < turns) {
        const char* const x = row_at(a.x, a.x_pitch, (int64_t)p.map * a.pixels + p.row0) + (size_t)(p.col0 + col) * VE * sizeof(T);
        F s[ONE ? 1 : P], q[ONE ? 1 : P], shift[ONE ? 1 : P];
#pragma unroll
        for (int k = 0; k < (ONE ? 1 : P); ++k) s[k] = q[k] = shift[k] = both<F>(0.f);
        int n = 0;
        for (int r = turn; r < p.rows; r += 4 * turns) {
            typename V::Raw raw[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) raw[u] = r + u * turns < p.rows ? *(const typename V::Raw*)(x + (size_t)(r + u * turns) * a.x_pitch) : raw_zero<typename V::Raw>();
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (r + u * turns >= p.rows) break;
                F d[P];
                V::open(raw[u], d);
                if (n++ == 0)
#pragma unroll
                    for (int k = 0; k < (ONE ? 1 : P); ++k) shift[k] = ONE ? both<F>(-lane_of(d[0], 0)) : mul2(d[k], both<F>(-1.f));
#pragma unroll
                for (int k = 0; k < P; ++k) {
                    const int at = ONE ? 0 : k;
                    const F t = add2(d[k], shift[at]);
                    s[at] = add2(s[at], t);
                    q[at] = fma2(t, t, q[at]);
                }
            }
        }
        // the thread's items: mean and squares around it
        const float count = (float)(n * (ONE ? VE : 1));
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            const float ss = ONE ? sum_of(s[0]) : lane_of(s[ONE ? 0 : i / 2], i & 1), qq = ONE ? sum_of(q[0]) : lane_of(q[ONE ? 0 : i / 2], i & 1);
            const float m = n ? ss / count : 0.f;
            const int at = turn * p.cols * IT + col * IT + i;
            pm[at] = m - lane_of(shift[ONE ? 0 : i / 2], i & 1);
            pq[at] = fmaxf(fmaf(-m, ss, qq), 0.f) + (ss - ss);           // (a NaN or an infinity stays one)
        }
    }
    __syncthreads();
    const int items = p.cols * IT, of = a.pieces > 1 ? items : items / p.ngroups;
    for (int g = threadIdx.x >> 5; g < p.ngroups; g += kThreads / 32) {
        auto at = [&](int i) { return i / of * items + g * of + i % of; };
        auto n = [&](int i) { const int t = i / of; return (float)((p.rows > t ? (p.rows - t + turns - 1) / turns : 0) * (ONE ? VE : 1)); };
        const float2 r = join_items(turns * of, n, [&](int i) { return pm[at(i)]; }, [&](int i) { return pq[at(i)]; }, (float)p.rows * of * (ONE ? VE : 1));
        if ((threadIdx.x & 31) == 0) a.part[((size_t)p.map * a.chunks * a.pieces + p.chunk * a.pieces + p.piece) * a.groups + p.group0 + g] = r;
    }
}

// A slice's groups' mean and rstd, from the chunks'.
template <int VE>
__device__ __forceinline__ void join_chunks(const GroupArgs& a, const Place& p, float2* fin)
{
    for (int g = threadIdx.x >> 5; g < p.ngroups; g += kThreads / 32) {
        const float2* const part = a.part + (size_t)p.map * a.chunks * a.pieces * a.groups + p.group0 + g;
        auto at = [&](int i) { return __ldcg(part + (size_t)i * a.groups); };
        auto n = [&](int i) { return (float)rows_of(a, i / a.pieces) * (float)(a.pieces > 1 ? cols_of(a, i % a.pieces) * VE : a.per); };
        const float total = (float)a.pixels * (float)a.per;
        const float2 r = join_items(a.chunks * a.pieces, n, [&](int i) { return at(i).x; }, [&](int i) { return at(i).y; }, total);
        const float rstd = inverse_root(r.y / total + a.eps);
        if ((threadIdx.x & 31) == 0) {
            fin[g] = make_float2(r.x, rstd);
            if (p.chunk == 0 && p.piece == 0) {
                if (a.mean) a.mean[(size_t)p.map * a.groups + p.group0 + g] = r.x;
                if (a.rstd) a.rstd[(size_t)p.map * a.groups + p.group0 + g] = rstd;
            }
        }
    }
    __syncthreads();
}

// What a thread keeps of its column: the weights, and its groups' numbers (fin: of the slice's groups).
template <typename T, int VE, bool ONE> struct Column {
    typedef typename Vec<T, VE>::F F;
    static constexpr int P = Vec<T, VE>::P;
    F g[P], b[P], first[ONE ? 1 : P], second[ONE ? 1 : P];
    __device__ __forceinline__ void weights(const GroupArgs& a, const Place& p, int col)
    {
        const int c = (p.col0 + col) * VE;
        if constexpr (VE > 1)
            if ((((uintptr_t)a.gamma | (uintptr_t)a.beta) & 15) == 0) {
                load_weights(a.gamma, c, 1.f, g);
                load_weights(a.beta, c, 0.f, b);
                return;
            }
#pragma unroll
        for (int k = 0; k < P; ++k) {
            g[k] = two<F>(a.gamma ? dc_ld(a.gamma + c + (VE > 1 ? 2 * k : 0)) : 1.f, VE > 1 ? (a.gamma ? dc_ld(a.gamma + c + 2 * k + 1) : 1.f) : 0.f);
            b[k] = two<F>(a.beta ? dc_ld(a.beta + c + (VE > 1 ? 2 * k : 0)) : 0.f, VE > 1 ? (a.beta ? dc_ld(a.beta + c + 2 * k + 1) : 0.f) : 0.f);
        }
    }
    template <typename R>
    __device__ __forceinline__ void groups(const GroupArgs& a, const Place& p, int col, F* first, F* second, R read) const
    {
#pragma unroll
        for (int k = 0; k < (ONE ? 1 : P); ++k) {
            float2 v[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int channel = col * VE + (ONE || VE == 1 ? 0 : 2 * k + h);
                v[h] = read(a.by_per ? channel * a.by_per >> 16 : a.pieces > 1 ? 0 : channel / a.per);
            }
            first[k] = two<F>(v[0].x, v[1].x);
            second[k] = two<F>(v[0].y, v[1].y);
        }
    }
};

template <typename T, int VE, bool ONE, int ACT>
__global__ void __launch_bounds__(kThreads) k_group_apply(const GroupArgs a)
{
    typedef Vec<T, VE> V;
    typedef typename V::F F;
    constexpr int P = V::P;
    __shared__ float2 fin[kThreads * (ONE ? 1 : VE)];
    dc_pdl_wait();
    dc_pdl_release();
    const Place p = place_of(a);
    join_chunks<VE>(a, p, fin);
    const int turns = kThreads / p.cols, col = threadIdx.x % p.cols, turn = threadIdx.x / p.cols;
    if (turn >= turns) return;
    Column<T, VE, ONE> c;
    F mean[ONE ? 1 : P], rstd[ONE ? 1 : P];
    c.weights(a, p, col);
    c.groups(a, p, col, mean, rstd, [&](int g) { return make_float2(-fin[g].x, fin[g].y); });
    const int64_t row0 = (int64_t)p.map * a.pixels + p.row0;
    const size_t at = (size_t)(p.col0 + col) * VE * sizeof(T);
    const char* const x = row_at(a.x, a.x_pitch, row0) + at;
    char* const y = row_at(a.y, a.y_pitch, row0) + at;
    for (int r = turn; r < p.rows; r += 4 * turns) {
        typename V::Raw raw[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) raw[u] = r + u * turns < p.rows ? *(const typename V::Raw*)(x + (size_t)(r + u * turns) * a.x_pitch) : raw_zero<typename V::Raw>();
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (r + u * turns >= p.rows) break;
            F d[P];
            V::open(raw[u], d);
#pragma unroll
            for (int k = 0; k < P; ++k) d[k] = affine(hat(d[k], mean[ONE ? 0 : k], rstd[ONE ? 0 : k]), c.g[k], c.b[k]);
            activate<ACT, ONE>(d);
            *(typename V::Raw*)(y + (size_t)(r + u * turns) * a.y_pitch) = V::close(d);
        }
    }
}

// Gradients, first pass: a chunk's sums of dz and dz xh of each channel, and of each group with gamma.
template <typename T, int VE, bool ONE, int ACT>
__global__ void __launch_bounds__(kThreads) k_group_back_sums(const GroupArgs a)
{
    typedef Vec<T, VE> V;
    typedef typename V::F F;
    constexpr int P = V::P;
    __shared__ float s1[kThreads * VE], s2[kThreads * VE];
    dc_pdl_wait();
    dc_pdl_release();
    const Place p = place_of(a);
    const int turns = kThreads / p.cols, col = threadIdx.x % p.cols, turn = threadIdx.x / p.cols, wide = p.cols * VE;
    if (turn < turns) {
        Column<T, VE, ONE> c;
        F mean[ONE ? 1 : P], rstd[ONE ? 1 : P], d1[P], d2[P];
        c.weights(a, p, col);
        const size_t of = (size_t)p.map * a.groups + p.group0;
        c.groups(a, p, col, mean, rstd, [&](int g) { return make_float2(-dc_ld(a.mean + of + g), dc_ld(a.rstd + of + g)); });
#pragma unroll
        for (int k = 0; k < P; ++k) d1[k] = d2[k] = both<F>(0.f);
        const int64_t row0 = (int64_t)p.map * a.pixels + p.row0;
        const size_t at = (size_t)(p.col0 + col) * VE * sizeof(T);
        const char *const x = row_at(a.x, a.x_pitch, row0) + at, *const dy = row_at(a.dy, a.dy_pitch, row0) + at;
        for (int r = turn; r < p.rows; r += 2 * turns) {
            typename V::Raw rx[2], rd[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bool there = r + u * turns < p.rows;
                rx[u] = there ? *(const typename V::Raw*)(x + (size_t)(r + u * turns) * a.x_pitch) : raw_zero<typename V::Raw>();
                rd[u] = there ? *(const typename V::Raw*)(dy + (size_t)(r + u * turns) * a.dy_pitch) : raw_zero<typename V::Raw>();
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (r + u * turns >= p.rows) break;
                F d[P], e[P], z[P];
                V::open(rx[u], d);
                V::open(rd[u], e);
#pragma unroll
                for (int k = 0; k < P; ++k) { d[k] = hat(d[k], mean[ONE ? 0 : k], rstd[ONE ? 0 : k]); z[k] = affine(d[k], c.g[k], c.b[k]); }
                activate_back<ACT, ONE>(e, z);
#pragma unroll
                for (int k = 0; k < P; ++k) { d1[k] = add2(d1[k], e[k]); d2[k] = fma2(e[k], d[k], d2[k]); }
            }
        }
#pragma unroll
        for (int i = 0; i < VE; ++i) { s1[turn * wide + col * VE + i] = lane_of(d1[i / 2 % P], i & 1); s2[turn * wide + col * VE + i] = lane_of(d2[i / 2 % P], i & 1); }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < wide; i += kThreads) {
        float t1 = 0.f, t2 = 0.f;
        for (int t = 0; t < turns; ++t) { t1 += s1[t * wide + i]; t2 += s2[t * wide + i]; }
        s1[i] = t1; s2[i] = t2;
        const int ch = p.col0 * VE + i;
        if (a.sums) {
            float* const out = a.sums + ((size_t)p.map * a.chunks + p.chunk) * 2 * a.channels + ch;
            out[0] = t1; out[a.channels] = t2;
        }
    }
    __syncthreads();
    const int of = wide / p.ngroups;
    for (int g = threadIdx.x >> 5; g < p.ngroups; g += kThreads / 32) {
        float t1 = 0.f, t2 = 0.f;
        for (int i = g * of + (threadIdx.x & 31); i < (g + 1) * of; i += 32) {
            const float w = a.gamma ? dc_ld(a.gamma + p.col0 * VE + i) : 1.f;
            t1 = fmaf(w, s1[i], t1); t2 = fmaf(w, s2[i], t2);
        }
        t1 = reduce_lanes<Sum>(t1, 32); t2 = reduce_lanes<Sum>(t2, 32);
        if ((threadIdx.x & 31) == 0) a.part[((size_t)p.map * a.chunks * a.pieces + p.chunk * a.pieces + p.piece) * a.groups + p.group0 + g] = make_float2(t1, t2);
    }
}

// Second pass: dx.
template <typename T, int VE, bool ONE, int ACT>
__global__ void __launch_bounds__(kThreads) k_group_back_apply(const GroupArgs a)
{
    typedef Vec<T, VE> V;
    typedef typename V::F F;
    constexpr int P = V::P;
    __shared__ float2 fin[kThreads * (ONE ? 1 : VE)];
    dc_pdl_wait();
    dc_pdl_release();
    const Place p = place_of(a);
    for (int g = threadIdx.x >> 5; g < p.ngroups; g += kThreads / 32) {
        const float2* const part = a.part + (size_t)p.map * a.chunks * a.pieces * a.groups + p.group0 + g;
        float t1 = 0.f, t2 = 0.f;
        for (int i = threadIdx.x & 31; i < a.chunks * a.pieces; i += 32) { const float2 v = __ldcg(part + (size_t)i * a.groups); t1 += v.x; t2 += v.y; }
        t1 = reduce_lanes<Sum>(t1, 32); t2 = reduce_lanes<Sum>(t2, 32);
        const float total = (float)a.pixels * (float)a.per;
        if ((threadIdx.x & 31) == 0) fin[g] = make_float2(-t1 / total, -t2 / total);
    }
    __syncthreads();
    const int turns = kThreads / p.cols, col = threadIdx.x % p.cols, turn = threadIdx.x / p.cols;
    if (turn >= turns) return;
    Column<T, VE, ONE> c;
    F mean[ONE ? 1 : P], rstd[ONE ? 1 : P], m1[ONE ? 1 : P], m2[ONE ? 1 : P];
    c.weights(a, p, col);
    const size_t of = (size_t)p.map * a.groups + p.group0;
    c.groups(a, p, col, mean, rstd, [&](int g) { return make_float2(-dc_ld(a.mean + of + g), dc_ld(a.rstd + of + g)); });
    c.groups(a, p, col, m1, m2, [&](int g) { return fin[g]; });
    const int64_t row0 = (int64_t)p.map * a.pixels + p.row0;
    const size_t at = (size_t)(p.col0 + col) * VE * sizeof(T);
    const char *const x = row_at(a.x, a.x_pitch, row0) + at, *const dy = row_at(a.dy, a.dy_pitch, row0) + at;
    char* const dx = row_at(a.y, a.y_pitch, row0) + at;
    for (int r = turn; r < p.rows; r += 2 * turns) {
        typename V::Raw rx[2], rd[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const bool there = r + u * turns < p.rows;
            rx[u] = there ? *(const typename V::Raw*)(x + (size_t)(r + u * turns) * a.x_pitch) : raw_zero<typename V::Raw>();
            rd[u] = there ? *(const typename V::Raw*)(dy + (size_t)(r + u * turns) * a.dy_pitch) : raw_zero<typename V::Raw>();
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (r + u * turns >= p.rows) break;
            F d[P], e[P], z[P];
            V::open(rx[u], d);
            V::open(rd[u], e);
#pragma unroll
            for (int k = 0; k < P; ++k) { d[k] = hat(d[k], mean[ONE ? 0 : k], rstd[ONE ? 0 : k]); z[k] = affine(d[k], c.g[k], c.b[k]); }
            activate_back<ACT, ONE>(e, z);
#pragma unroll
            for (int k = 0; k < P; ++k) d[k] = mul2(fma2(d[k], m2[ONE ? 0 : k], add2(mul2(e[k], c.g[k]), m1[ONE ? 0 : k])), rstd[ONE ? 0 : k]);
            *(typename V::Raw*)(dx + (size_t)(r + u * turns) * a.y_pitch) = V::close(d);
        }
    }
}

// ---------------------------------------------------------------------------
// A slice of a map in the shared memory of a cluster: read once
// ---------------------------------------------------------------------------
constexpr int kMostResident = 256;                            // threads
constexpr int kMostCluster = 8, kMostGroups = 64;             // CTAs to a slice; groups of one

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Nothing is sent before every CTA of the cluster runs.
__device__ __forceinline__ void cluster_started(bool cluster) { if (cluster) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait(bool cluster) { if (cluster) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// To the same place in CTA `rank` of the cluster.
__device__ __forceinline__ void send(const float2* at, int rank, float2 v)
{
    uint32_t to;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"((uint32_t)__cvta_generic_to_shared(at)), "r"(rank));
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(v.x), "f"(v.y) : "memory");
}
__device__ __forceinline__ void send(const float* at, int rank, float v)
{
    uint32_t to;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"((uint32_t)__cvta_generic_to_shared(at)), "r"(rank));
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(v) : "memory");
}
// What threads of one column have to add up: within a warp first, where its lanes hold whole rows of columns.  Returns the rows of partial sums that are left.
template <int N, typename F>
__device__ __forceinline__ int fold(F (&v)[N], int cols, int turns)
{
    if (cols & (cols - 1)) return turns;
    for (int o = cols; o < 32; o <<= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = add_shuffled(v[k], o);
    return (int)blockDim.x >> 5;
}
// ... and which of them this thread leaves, or none.
__device__ __forceinline__ int fold_row(int cols, int turn, int turns)
{
    if (cols & (cols - 1)) return turn < turns ? turn : -1;
    return (threadIdx.x & 31) < cols ? (int)(threadIdx.x >> 5) : -1;
}
// A thread's place: `turns` rows of columns at once (at most 256 threads and 16 columns: one multiplication).
__device__ __forceinline__ void seat(const GroupArgs& a, int& col, int& turn, int& turns)
{
    turns = (int)blockDim.x * a.by_width >> 16;
    turn = (int)threadIdx.x * a.by_width >> 16;
    col = (int)threadIdx.x - turn * a.width;
}
// Rows of partial sums added up: a thread to each of `wide` places.
__device__ __forceinline__ float rows_of_sums(const float* part, int left, int wide, int i)
{
    float t = 0.f;
#pragma unroll 8
    for (int k = 0; k < left; ++k) t += part[k * wide + i];
    return t;
}

__device__ __forceinline__ Place resident_place(const GroupArgs& a)
{
    Place p;
    p.chunk = blockIdx.x; p.map = blockIdx.z; p.piece = 0; p.ngroups = a.gs; p.cols = a.width;
    p.group0 = blockIdx.y * a.gs; p.col0 = blockIdx.y * a.width; p.row0 = p.chunk * a.rows_per; p.rows = rows_of(a, p.chunk);
    return p;
}

// A CTA has rows_per rows of a slice; its cluster has the slice.  Each thread copies its own values into shared memory and reads them twice from there.  Distances are
// taken from the group's first value in the CTA's first row, so that threads' sums just add up.
template <typename T, int VE, bool ONE, int ACT>
__global__ void __launch_bounds__(kMostResident) k_group_resident(const GroupArgs a)
{
    typedef Vec<T, VE> V;
    typedef typename V::F F;
    constexpr int P = V::P, IT = ONE ? 1 : VE, N = ONE ? 1 : P;
    extern __shared__ uint4 kept[];                           // [rows_per][columns], then the partial sums
    __shared__ float2 exchange[kMostCluster][kMostGroups], fin[kMostGroups];
    cluster_started(a.chunks > 1);
    dc_pdl_wait();
    dc_pdl_release();
    const Place p = resident_place(a);
    int col, turn, turns;
    seat(a, col, turn, turns);
    const int64_t row0 = (int64_t)p.map * a.pixels + p.row0;
    const size_t at = (size_t)(p.col0 + col) * 16;
    const char* const x = row_at(a.x, a.x_pitch, row0) + at;
    const uint32_t mine = (uint32_t)__cvta_generic_to_shared(kept) + 16u * threadIdx.x, line = 16u * turns * p.cols;
    if (turn < turns) {
        uint32_t to = mine;
        for (int r = turn; r < p.rows; r += turns, to += line) copy16(to, x + (size_t)r * a.x_pitch);
    }
    float* const part = (float*)(kept + (size_t)a.rows_per * p.cols);     // [rows of partial sums][sums, squares][items]
    const int items = p.cols * IT;
    Column<T, VE, ONE> c;
    c.weights(a, p, col);
    F s[2 * N], first[N], unused[N];
    if (p.rows > 0)
        c.groups(a, p, col, first, unused, [&](int g) {
            float v;
            Vec<T, 1>::open(((const T*)row_at(a.x, a.x_pitch, row0))[(p.group0 + g) * a.per], &v);
            return make_float2(-v, 0.f);
        });
#pragma unroll
    for (int k = 0; k < 2 * N; ++k) s[k] = both<F>(0.f);
    copies_done();
    if (turn < turns) {
        const uint4* k4 = kept + threadIdx.x;
#pragma unroll 4
        for (int r = turn; r < p.rows; r += turns, k4 += turns * p.cols) {
            F d[P];
            V::open(*(const typename V::Raw*)k4, d);
#pragma unroll
            for (int k = 0; k < P; ++k) {
                const int i = ONE ? 0 : k;
                const F t = add2(d[k], first[i]);
                s[i] = add2(s[i], t);
                s[N + i] = fma2(t, t, s[N + i]);
            }
        }
    }
    const int left = fold(s, p.cols, turns), to = fold_row(p.cols, turn, turns);
    if (to >= 0)
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            part[to * 2 * items + col * IT + i] = ONE ? sum_of(s[0]) : lane_of(s[ONE ? 0 : i / 2], i & 1);
            part[(to * 2 + 1) * items + col * IT + i] = ONE ? sum_of(s[N]) : lane_of(s[N + (ONE ? 0 : i / 2)], i & 1);
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * items; i += blockDim.x) part[i] = rows_of_sums(part, left, 2 * items, i);       // (its own column alone)
    __syncthreads();
    cluster_wait(a.chunks > 1);
    const int of = ONE && a.gs == p.cols ? 1 : items / p.ngroups;
    for (int g = threadIdx.x >> 5; g < p.ngroups; g += blockDim.x >> 5) {
        float sum = 0.f, squares = 0.f;
        for (int i = g * of + (threadIdx.x & 31); i < (g + 1) * of; i += 32) { sum += part[i]; squares += part[items + i]; }
        if (of > 1) { sum = reduce_lanes<Sum>(sum, 32); squares = reduce_lanes<Sum>(squares, 32); }
        else { sum = __shfl_sync(0xffffffffu, sum, 0); squares = __shfl_sync(0xffffffffu, squares, 0); }
        const float n = (float)p.rows * (float)a.per;
        float2 r = make_float2(0.f, 0.f);
        if (p.rows > 0) {
            float v;
            Vec<T, 1>::open(((const T*)row_at(a.x, a.x_pitch, row0))[(p.group0 + g) * a.per], &v);
            const float m = sum / n;
            r = make_float2(m + v, fmaxf(fmaf(-m, sum, squares), 0.f) + (sum - sum));
        }
        const int rank = threadIdx.x & 31;
        if (rank < a.chunks) send(&exchange[p.chunk][g], rank, r);
    }
    if (a.chunks > 1) cluster_sync(); else __syncthreads();
    if (threadIdx.x < p.ngroups) {
        const int g = threadIdx.x;
        const float total = (float)a.pixels * (float)a.per;
        float mean = 0.f, squares = 0.f;
        for (int k = 0; k < a.chunks; ++k) mean = fmaf((float)rows_of(a, k) * (float)a.per, exchange[k][g].x, mean);
        mean /= total;
        for (int k = 0; k < a.chunks; ++k) {
            const float2 v = exchange[k][g];
            const float w = (float)rows_of(a, k) * (float)a.per, d = v.x - mean;
            if (w > 0.f) squares += fmaf(w * d, d, v.y);
        }
        const float rstd = inverse_root(squares / total + a.eps);
        fin[g] = make_float2(-mean, rstd);
        if (p.chunk == 0) {
            if (a.mean) a.mean[(size_t)p.map * a.groups + p.group0 + g] = mean;
            if (a.rstd) a.rstd[(size_t)p.map * a.groups + p.group0 + g] = rstd;
        }
    }
    __syncthreads();
    if (turn >= turns) return;
    F mean[N], rstd[N];
    c.groups(a, p, col, mean, rstd, [&](int g) { return fin[g]; });
    char* y = row_at(a.y, a.y_pitch, row0 + turn) + at;
    const uint4* k4 = kept + threadIdx.x;
#pragma unroll 4
    for (int r = turn; r < p.rows; r += turns, k4 += turns * p.cols, y += turns * a.y_pitch) {
        F d[P];
        V::open(*(const typename V::Raw*)k4, d);
#pragma unroll
        for (int k = 0; k < P; ++k) d[k] = affine(hat(d[k], mean[ONE ? 0 : k], rstd[ONE ? 0 : k]), c.g[k], c.b[k]);
        activate<ACT, ONE>(d);
        *(typename V::Raw*)y = V::close(d);
    }
}

// The gradients likewise: x and dy are kept (behind a ReLU dy or zero, which is as exact).  SiLU's derivative is worked out twice: 32 maps of 56 x 56 x 256 bf16 55 us; with dz
// kept as floats, which leaves an SM two CTAs in the place of four, 61.
template <typename T, int VE, bool ONE, int ACT>
__global__ void __launch_bounds__(kMostResident, ONE ? 4 : 2) k_group_back_resident(const GroupArgs a)
{
    typedef Vec<T, VE> V;
    typedef typename V::F F;
    constexpr int P = V::P, N = ONE ? 1 : P;
    extern __shared__ uint4 kept[];                           // [2][rows_per][columns], then the partial sums
    __shared__ float2 exchange[kMostCluster][kMostGroups], fin[kMostGroups];
    cluster_started(a.chunks > 1);
    dc_pdl_wait();
    dc_pdl_release();
    const Place p = resident_place(a);
    const int wide = p.cols * VE;
    int col, turn, turns;
    seat(a, col, turn, turns);
    const int64_t row0 = (int64_t)p.map * a.pixels + p.row0;
    const size_t at = (size_t)(p.col0 + col) * 16;
    const char *const x = row_at(a.x, a.x_pitch, row0) + at, *const dy = row_at(a.dy, a.dy_pitch, row0) + at;
    const uint32_t mine = (uint32_t)__cvta_generic_to_shared(kept) + 16u * threadIdx.x, line = 16u * turns * p.cols, other = 16u * a.rows_per * p.cols;
    if (turn < turns) {
        uint32_t to = mine;
        for (int r = turn; r < p.rows; r += turns, to += line) { copy16(to, x + (size_t)r * a.x_pitch); copy16(to + other, dy + (size_t)r * a.dy_pitch); }
    }
    float* const part = (float*)(kept + 2 * (size_t)a.rows_per * p.cols);     // [rows of partial sums][2][channels]
    Column<T, VE, ONE> c;
    c.weights(a, p, col);
    F mean[N], rstd[N], s[2 * P];
    const size_t of_map = (size_t)p.map * a.groups + p.group0;
    c.groups(a, p, col, mean, rstd, [&](int g) { return make_float2(-dc_ld(a.mean + of_map + g), dc_ld(a.rstd + of_map + g)); });
#pragma unroll
    for (int k = 0; k < 2 * P; ++k) s[k] = both<F>(0.f);
    copies_done();
    const size_t half = (size_t)a.rows_per * p.cols;
    if (turn < turns) {
        uint4* k4 = kept + threadIdx.x;
#pragma unroll 2
        for (int r = turn; r < p.rows; r += turns, k4 += turns * p.cols) {
            F d[P], e[P], z[P];
            V::open(*(const typename V::Raw*)k4, d);
            V::open(*(const typename V::Raw*)(k4 + half), e);
#pragma unroll
            for (int k = 0; k < P; ++k) { d[k] = hat(d[k], mean[ONE ? 0 : k], rstd[ONE ? 0 : k]); z[k] = affine(d[k], c.g[k], c.b[k]); }
            activate_back<ACT, ONE>(e, z);
#pragma unroll
            for (int k = 0; k < P; ++k) { s[k] = add2(s[k], e[k]); s[P + k] = fma2(e[k], d[k], s[P + k]); }
            if (ACT == DC_ACT_RELU) *(typename V::Raw*)(k4 + half) = V::close(e);           // dy or zero: as exact as it came
        }
    }
    const int left = fold(s, p.cols, turns), to = fold_row(p.cols, turn, turns);
    if (to >= 0)
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            part[to * 2 * wide + col * VE + i] = lane_of(s[i / 2], i & 1);
            part[(to * 2 + 1) * wide + col * VE + i] = lane_of(s[P + i / 2], i & 1);
        }
    float* const sums_of_all = part + (size_t)left * 2 * wide;               // [chunks][2][channels]: of a single map, in the first CTA
    __syncthreads();
    cluster_wait(a.chunks > 1);
    for (int i = threadIdx.x; i < 2 * wide; i += blockDim.x) {
        const float t = rows_of_sums(part, left, 2 * wide, i);
        part[i] = t;                                          // (its own column alone)
        if (a.dgamma || a.dbeta) send(sums_of_all + p.chunk * 2 * wide + i, 0, t);
        else if (a.sums) a.sums[((size_t)p.map * a.chunks + p.chunk) * 2 * a.channels + (i < wide ? p.col0 * VE + i : a.channels + p.col0 * VE + i - wide)] = t;
    }
    __syncthreads();
    const int of = wide / p.ngroups;
    for (int g = threadIdx.x >> 5; g < p.ngroups; g += blockDim.x >> 5) {
        float t1 = 0.f, t2 = 0.f;
        for (int i = g * of + (threadIdx.x & 31); i < (g + 1) * of; i += 32) {
            const float w = a.gamma ? dc_ld(a.gamma + p.col0 * VE + i) : 1.f;
            t1 = fmaf(w, part[i], t1); t2 = fmaf(w, part[wide + i], t2);
        }
        t1 = reduce_lanes<Sum>(t1, 32); t2 = reduce_lanes<Sum>(t2, 32);
        const int rank = threadIdx.x & 31;
        if (rank < a.chunks) send(&exchange[p.chunk][g], rank, make_float2(t1, t2));
    }
    if (a.chunks > 1) cluster_sync(); else __syncthreads();
    if ((a.dgamma || a.dbeta) && p.chunk == 0)
        for (int i = threadIdx.x; i < 2 * wide; i += blockDim.x) {
            const float t = rows_of_sums(sums_of_all, a.chunks, 2 * wide, i);
            const int ch = p.col0 * VE + (i < wide ? i : i - wide);
            if (i < wide) { if (a.dbeta) a.dbeta[ch] = t; }
            else if (a.dgamma) a.dgamma[ch] = t;
        }
    if (!a.y) return;
    if (threadIdx.x < p.ngroups) {
        float t1 = 0.f, t2 = 0.f;
        for (int k = 0; k < a.chunks; ++k) { t1 += exchange[k][threadIdx.x].x; t2 += exchange[k][threadIdx.x].y; }
        const float total = (float)a.pixels * (float)a.per;
        fin[threadIdx.x] = make_float2(-t1 / total, -t2 / total);
    }
    __syncthreads();
    if (turn >= turns) return;
    F m1[N], m2[N];
    c.groups(a, p, col, m1, m2, [&](int g) { return fin[g]; });
    char* dx = row_at(a.y, a.y_pitch, row0 + turn) + at;
    const uint4* k4 = kept + threadIdx.x;
#pragma unroll 2
    for (int r = turn; r < p.rows; r += turns, k4 += turns * p.cols, dx += turns * a.y_pitch) {
        F d[P], e[P], z[P];
        V::open(*(const typename V::Raw*)k4, d);
        V::open(*(const typename V::Raw*)(k4 + half), e);
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const int i = ONE ? 0 : k;
            d[k] = hat(d[k], mean[i], rstd[i]);
            z[k] = affine(d[k], c.g[k], c.b[k]);
        }
        if (ACT == DC_ACT_SILU) activate_back<ACT, ONE>(e, z);
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const int i = ONE ? 0 : k;
            d[k] = mul2(fma2(d[k], m2[i], add2(mul2(e[k], c.g[k]), m1[i])), rstd[i]);
        }
        *(typename V::Raw*)dx = V::close(d);
    }
}

// dgamma and dbeta: the sums of all maps and chunks, 32 threads per column, in a fixed order.
__global__ void __launch_bounds__(1024) k_group_join(const float* sums, int count, int channels, float* dgamma, float* dbeta)
{
    __shared__ float part[32][33];
    dc_pdl_wait();
    dc_pdl_release();
    const int lane = threadIdx.x & 31, turn = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (col < 2 * channels)
#pragma unroll 4
        for (int c = turn; c < count; c += 32) s += sums[(size_t)c * 2 * channels + col];
    part[turn][lane] = s;
    __syncthreads();
    s = reduce_lanes<Sum>(part[lane][turn], 32);
    const int mine = blockIdx.x * 32 + turn;
    if (lane == 0 && mine < 2 * channels) {
        if (mine < channels) { if (dbeta) dbeta[mine] = s; }
        else if (dgamma) dgamma[mine - channels] = s;
    }
}

// CTAs to the rows of a slice, where a map's rows are dealt to several: at most so many (the workspace holds as many).
int most_chunks(int64_t maps, int64_t pixels)
{
    int64_t c = (pixels + 15) / 16;
    int64_t room = maps > 0 ? (4096 + maps - 1) / maps : 1;
    if (room < kMostCluster) room = kMostCluster;
    if (c > room) c = room;
    return (int)(c > kMostChunks ? kMostChunks : c < 1 ? 1 : c);
}
int gcd(int a, int b) { while (b) { const int t = a % b; a = b; b = t; } return a; }

size_t part_bytes(int64_t maps, int chunks, int channels, int groups) { return ((size_t)maps * chunks * ((size_t)groups + channels / kThreads + 1) * sizeof(float2) + 255) / 256 * 256; }

// Columns of VE channels: whole groups to a slice, as many as a CTA has threads for; or a wide group in pieces.  False: VE does not go.
bool plan_columns(GroupArgs& a, int ve)
{
    const int least = a.per / gcd(a.per, ve);                  // columns that whole groups take at least
    a.pieces = 1;
    if (a.channels % ve) return false;
    if (least > kThreads) {
        if (a.per % ve) return false;
        a.piece_items = a.per / ve;
        a.pieces = dc_div_up(a.piece_items, kThreads);
        a.width = dc_div_up(a.piece_items, a.pieces);
        a.pieces = dc_div_up(a.piece_items, a.width);
        a.gs = 1;
        a.slices = a.groups * a.pieces;
        return true;
    }
    const int unit = least * ve / a.per;                       // groups of those
    if (a.groups % unit) return false;
    const int units = a.groups / unit;
    int best = 1;
    for (int j = 1; j <= units; ++j)
        if (units % j == 0 && j * least <= kThreads && (j == 1 || (j - 1) * least * ve < 64)) best = j;   // columns of 64 channels or so
    a.gs = best * unit; a.width = best * least; a.slices = units / best;
    return true;
}

// A slice in the shared memory of a cluster, if it fits: columns of 64 bytes a row (fewer where it does not), CTAs of up to 56 KB, four to an SM, so that some load while others compute
// and store, or as many as a cluster has, or larger ones; 256 threads, or 128 where those would have fewer than four vectors each.  32 maps of 56 x 56 x 256 bf16, SiLU, us: forward 28.9
// (columns of 32 bytes 34.2, of 128 34.6; 25 KB 30.5, 100 KB 40), gradients 55.1 (60.5, 61; 100 KB and more 80).
constexpr int kWantKept = 56 * 1024, kMostKept = 200 * 1024;
bool plan_resident(GroupArgs& a, int ve, int planes, int num_sms, int* block, size_t* smem)
{
    const int least = a.per / gcd(a.per, ve), unit = least * ve / a.per, bytes = 16 * planes;
    if (a.channels % ve || a.groups % unit || least > 16 || a.maps > 65535) return false;
    const int units = a.groups / unit;
    int best = 0;
    for (int j = 1; j <= units && j * least <= 16; ++j) {
        if (units % j || j * unit > kMostGroups) continue;
        if ((int64_t)a.pixels * j * least * bytes > (int64_t)kMostCluster * kMostKept) break;
        best = j;
        if (j * least >= 4) break;
    }
    if (!best) return false;
    a.pieces = 1; a.gs = best * unit; a.width = best * least; a.slices = units / best;
    const int64_t slice = (int64_t)a.pixels * a.width * bytes;
    int turns = kMostResident / a.width;
    a.by_width = dc_div_up(65536, a.width); a.by_per = dc_div_up(65536, a.per);
    int cs = 1;
    while (cs < kMostCluster && (slice > (int64_t)cs * kWantKept || ((int64_t)a.maps * a.slices * cs < num_sms && a.pixels >= 4 * cs * turns))) cs *= 2;
    if (cs > most_chunks(a.maps, a.pixels)) return false;
    a.rows_per = dc_div_up(a.pixels, cs);
    a.chunks = cs;
    const int threads = (int64_t)a.rows_per * a.width >= 4 * kMostResident ? kMostResident : kMostResident / 2;
    turns = threads / a.width;
    const int left = a.width & (a.width - 1) ? turns : threads / 32;
    *block = threads;
    *smem = (size_t)a.rows_per * a.width * bytes + (size_t)(left + (a.dgamma || a.dbeta ? cs : 0)) * 2 * a.width * ve * sizeof(float);
    return *smem <= (size_t)kMostKept + 16 * 1024;
}

template <typename T, int VE, bool ONE, int ACT>
cudaError_t launch_resident(const GroupArgs& a, bool back, int block, size_t smem, int device, cudaStream_t stream)
{
    auto* const kernel = back ? k_group_back_resident<T, VE, ONE, ACT> : k_group_resident<T, VE, ONE, ACT>;
    static dc_once_per_device set[2];
    const cudaError_t e = set[back].ensure(device, [=] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostKept + 16 * 1024); });
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)a.chunks; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.chunks, (unsigned)a.slices, (unsigned)a.maps); cfg.blockDim = dim3(block); cfg.dynamicSmemBytes = smem; cfg.stream = stream;
    cfg.attrs = attr; cfg.numAttrs = g_dc_pdl ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <typename T, int VE, bool ONE, int ACT>
cudaError_t launch_group(GroupArgs& a, bool back, int device, int num_sms, cudaStream_t stream)
{
    if constexpr (VE > 1) {
        GroupArgs r = a;
        size_t smem = 0;
        int block = 0;
        const int planes = back ? 2 : 1;                      // 16 bytes that are kept of a column's row: x, and dy
        if (a.maps > 1) r.dgamma = r.dbeta = nullptr;
        if (plan_resident(r, VE, planes, num_sms, &block, &smem)) {
            a.joined = r.dgamma || r.dbeta;
            a.chunks = r.chunks;                              // (for the join of the sums)
            return launch_resident<T, VE, ONE, ACT>(r, back, block, smem, device, stream);
        }
    }
    const dim3 grid((unsigned)((int64_t)a.maps * a.slices * a.chunks));
    if (!back) {
        const cudaError_t e = dc_launch_pdl(k_group_stats<T, VE, ONE>, grid, kThreads, 0, stream, a);
        return e != cudaSuccess ? e : dc_launch_pdl(k_group_apply<T, VE, ONE, ACT>, grid, kThreads, 0, stream, a);
    }
    const cudaError_t e = dc_launch_pdl(k_group_back_sums<T, VE, ONE, ACT>, grid, kThreads, 0, stream, a);
    return e != cudaSuccess || !a.y ? e : dc_launch_pdl(k_group_back_apply<T, VE, ONE, ACT>, grid, kThreads, 0, stream, a);
}
template <typename T, int VE>
cudaError_t launch_group_as(GroupArgs& a, bool back, int activation, int device, int num_sms, cudaStream_t stream)
{
#define DC_GROUP(ONE) \
    switch (activation) { \
    case DC_ACT_RELU: return launch_group<T, VE, ONE, DC_ACT_RELU>(a, back, device, num_sms, stream); \
    case DC_ACT_SILU: return launch_group<T, VE, ONE, DC_ACT_SILU>(a, back, device, num_sms, stream); \
    default: return launch_group<T, VE, ONE, DC_ACT_NONE>(a, back, device, num_sms, stream); \
    }
    if constexpr (VE > 1)
        if (a.per % VE) { DC_GROUP(false) }
    DC_GROUP(true)
#undef DC_GROUP
}

int launch(GroupArgs& a, bool back, int activation, int dtype, cudaStream_t stream)
{
    const int elt = dtype == DC_BF16 ? 2 : 4, ve = 16 / elt;
    int device = 0, sms = 0;
    const int rc = dc_current_device(&device, &sms);
    if (rc != DC_OK) return rc;
    auto aligned = [](const void* p, size_t pitch) { return (uintptr_t)p % 16 == 0 && pitch % 16 == 0; };
    const bool rows = (int64_t)a.maps * a.pixels > 1;
    const bool vec = aligned(a.x, rows ? a.x_pitch : 0) && (!a.y || aligned(a.y, rows ? a.y_pitch : 0)) && (!back || aligned(a.dy, rows ? a.dy_pitch : 0)) && plan_columns(a, ve);
    if (!vec) plan_columns(a, 1);
    const int most = most_chunks(a.maps, a.pixels), turns = kThreads / a.width;
    a.chunks = dc_div_up(a.pixels, 4 * turns);
    if (a.chunks > most) a.chunks = most;
    a.rows_per = dc_div_up(a.pixels, a.chunks);
    a.chunks = dc_div_up(a.pixels, a.rows_per);
    if ((int64_t)a.maps * a.slices * a.chunks > 0x7fffffff) return DC_ERR_LIMIT;
    if (dtype == DC_BF16) DC_CUDA(vec ? (launch_group_as<__nv_bfloat16, 8>(a, back, activation, device, sms, stream)) : (launch_group_as<__nv_bfloat16, 1>(a, back, activation, device, sms, stream)));
    else DC_CUDA(vec ? (launch_group_as<float, 4>(a, back, activation, device, sms, stream)) : (launch_group_as<float, 1>(a, back, activation, device, sms, stream)));
    return DC_OK;
}

constexpr int kMostChannels = 16384;

// What both passes ask of their arguments.
int check(int64_t maps, int64_t pixels, int32_t channels, int32_t groups, int32_t activation, int32_t dtype)
{
    if (dtype != DC_FP32 && dtype != DC_BF16) return DC_ERR_CONFIG;
    if (activation != DC_ACT_NONE && activation != DC_ACT_RELU && activation != DC_ACT_SILU) return DC_ERR_CONFIG;
    if (maps < 0 || pixels < 0 || channels < 1 || groups < 1 || channels % groups) return DC_ERR_ARG;
    if (channels > kMostChannels || maps > DC_MOST_ROWS || pixels > DC_MOST_ROWS || maps * pixels > DC_MOST_ROWS || maps * groups > (1 << 27)) return DC_ERR_LIMIT;
    return DC_OK;
}
bool floats_ok(const float* p) { return (uintptr_t)p % sizeof(float) == 0; }
bool rows_ok(const void* p, size_t pitch, int64_t rows, int channels, int elt) { return p && (uintptr_t)p % elt == 0 && pitch % elt == 0 && (rows < 2 || pitch >= (size_t)channels * elt); }

}  // namespace

extern "C" {

int dc_group_norm_workspace(int64_t maps, int64_t pixels, int32_t channels, int32_t groups, size_t* bytes)
{
    if (!bytes) return DC_ERR_ARG;
    const int rc = check(maps, pixels, channels, groups, DC_ACT_NONE, DC_FP32);
    if (rc != DC_OK) return rc;
    const int chunks = most_chunks(maps, pixels);
    *bytes = part_bytes(maps, chunks, channels, groups) + (size_t)maps * chunks * 2 * channels * sizeof(float) + 256;
    return DC_OK;
}

int dc_group_norm(const void* x_dev, size_t x_pitch, const float* gamma_dev, const float* beta_dev, int64_t maps, int64_t pixels, int32_t channels, int32_t groups, double eps,
                  int32_t activation, int32_t dtype, void* y_dev, size_t y_pitch, float* mean_dev, float* rstd_dev, void* workspace_dev, size_t workspace_bytes, void* cuda_stream)
{
    int rc = check(maps, pixels, channels, groups, activation, dtype);
    if (rc != DC_OK) return rc;
    if (!(eps >= 0.0) || !(eps < 1e30)) return DC_ERR_ARG;
    const int64_t rows = maps * pixels;
    const int elt = dtype == DC_BF16 ? 2 : 4;
    if (rows > 1 && (x_pitch | y_pitch) > 0xffffffffu) return DC_ERR_LIMIT;
    if (!floats_ok(gamma_dev) || !floats_ok(beta_dev) || !floats_ok(mean_dev) || !floats_ok(rstd_dev)) return DC_ERR_ARG;
    if (rows == 0) return DC_OK;
    size_t need = 0;
    dc_group_norm_workspace(maps, pixels, channels, groups, &need);
    if (!rows_ok(x_dev, x_pitch, rows, channels, elt) || !rows_ok(y_dev, y_pitch, rows, channels, elt) || !workspace_dev || workspace_bytes < need) return DC_ERR_ARG;
    GroupArgs a = {};
    a.x = x_dev; a.x_pitch = x_pitch; a.y = y_dev; a.y_pitch = y_pitch; a.gamma = gamma_dev; a.beta = beta_dev; a.mean = mean_dev; a.rstd = rstd_dev; a.eps = (float)eps;
    a.maps = (int)maps; a.pixels = (int)pixels; a.channels = channels; a.groups = groups; a.per = channels / groups;
    a.part = (float2*)(((uintptr_t)workspace_dev + 255) & ~(uintptr_t)255);
    return launch(a, false, activation, dtype, (cudaStream_t)cuda_stream);
}

int dc_group_norm_backward(const void* dy_dev, size_t dy_pitch, const void* x_dev, size_t x_pitch, const float* gamma_dev, const float* beta_dev, const float* mean_dev,
                           const float* rstd_dev, int64_t maps, int64_t pixels, int32_t channels, int32_t groups, int32_t activation, int32_t dtype, void* dx_dev, size_t dx_pitch,
                           float* dgamma_dev, float* dbeta_dev, void* workspace_dev, size_t workspace_bytes, void* cuda_stream)
{
    int rc = check(maps, pixels, channels, groups, activation, dtype);
    if (rc != DC_OK) return rc;
    const int64_t rows = maps * pixels;
    const int elt = dtype == DC_BF16 ? 2 : 4;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (rows > 1 && (x_pitch | dy_pitch | (dx_dev ? dx_pitch : 0)) > 0xffffffffu) return DC_ERR_LIMIT;
    if (!floats_ok(gamma_dev) || !floats_ok(beta_dev) || !floats_ok(mean_dev) || !floats_ok(rstd_dev) || !floats_ok(dgamma_dev) || !floats_ok(dbeta_dev)) return DC_ERR_ARG;
    if (rows == 0) {                    // sums of nothing
        if (dgamma_dev) DC_CUDA(cudaMemsetAsync(dgamma_dev, 0, sizeof(float) * channels, stream));
        if (dbeta_dev) DC_CUDA(cudaMemsetAsync(dbeta_dev, 0, sizeof(float) * channels, stream));
        return DC_OK;
    }
    size_t need = 0;
    dc_group_norm_workspace(maps, pixels, channels, groups, &need);
    if (!mean_dev || !rstd_dev || !rows_ok(dy_dev, dy_pitch, rows, channels, elt) || !rows_ok(x_dev, x_pitch, rows, channels, elt) || !workspace_dev || workspace_bytes < need) return DC_ERR_ARG;
    if (dx_dev && !rows_ok(dx_dev, dx_pitch, rows, channels, elt)) return DC_ERR_ARG;
    const bool weights = dgamma_dev || dbeta_dev;
    if (!dx_dev && !weights) return DC_OK;
    GroupArgs a = {};
    a.x = x_dev; a.x_pitch = x_pitch; a.dy = dy_dev; a.dy_pitch = dy_pitch; a.y = dx_dev; a.y_pitch = dx_pitch; a.gamma = gamma_dev; a.beta = beta_dev;
    a.mean = (float*)mean_dev; a.rstd = (float*)rstd_dev;
    a.maps = (int)maps; a.pixels = (int)pixels; a.channels = channels; a.groups = groups; a.per = channels / groups;
    a.part = (float2*)(((uintptr_t)workspace_dev + 255) & ~(uintptr_t)255);
    a.dgamma = dgamma_dev; a.dbeta = dbeta_dev;
    a.sums = weights ? (float*)((char*)a.part + part_bytes(maps, most_chunks(maps, pixels), channels, groups)) : nullptr;
    if ((rc = launch(a, true, activation, dtype, stream)) != DC_OK) return rc;
    if (weights && !a.joined)
        DC_CUDA(dc_launch_pdl(k_group_join, dim3((unsigned)dc_div_up(2 * channels, 32)), 1024, 0, stream, (const float*)a.sums, a.maps * a.chunks, (int)channels, dgamma_dev, dbeta_dev));
    return DC_OK;
}

}  // extern "C"
