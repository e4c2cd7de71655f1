// Group normalisation with an activation, channels last, and its gradients.
//
//   mean, rstd over the pixels of a map and the channels of a group;  xh = (x - mean) rstd,  z = xh gamma + beta,  y = act(z)
//   with dz = dy act'(z), g = dz gamma:  dx = rstd (g - mean(g) - xh mean(g xh)),  dgamma = sum over maps and pixels dz xh,  dbeta = sum dz
//
// What bounds them: memory, one read and one write of the map (two reads and a write for the gradients).
//
// A slice is the columns of a map that a CTA works on: some whole groups, or a piece of one that is wider than a CTA.  A thread has one column (16 bytes of
// each of its rows, or two elements or one where rows are not aligned to 16 bytes) and so one set of weights and of sums.
//
// Sums of squares: a CTA takes its values' distances from a number within 2 sigma of their mean (statistics()), so that no more than 4/5 of the squares are taken off again as the mean's own,
// and threads' sums just add up; CTAs' means and squares are then joined by M2 = sum M2_i + sum n_i (mean_i - mean)^2, in a fixed order: equal calls give equal bits.
#include <atomic>

#include "dc_quantise.cuh"

namespace {

// Two elements of a row, where it does not lie on 16 bytes.
template <> struct Vec<float, 2> {
    typedef float2 Raw; typedef float2 F;
    static constexpr int P = 1;
    static __device__ __forceinline__ void open(Raw t, float2* v) { v[0] = t; }
    static __device__ __forceinline__ Raw close(const float2* v) { return v[0]; }
};
template <> struct Vec<__nv_bfloat16, 2> {
    typedef uint32_t Raw; typedef float2 F;
    static constexpr int P = 1;
    static __device__ __forceinline__ void open(Raw t, float2* v) { v[0] = make_float2(__uint_as_float(t << 16), __uint_as_float(t & 0xffff0000u)); }
    static __device__ __forceinline__ Raw close(const float2* v) { const __nv_bfloat162 t = __floats2bfloat162_rn(v[0].x, v[0].y); return *(const uint32_t*)&t; }
};

constexpr int kThreads = 256;
constexpr int kMostChunks = 128;

struct GroupArgs {
    const void *x, *dy; void* y;                    // y: the output, or dx
    size_t x_pitch, dy_pitch, y_pitch;
    const float *gamma, *beta;                      // or NULL: ones, zeros
    float *mean, *rstd;                             // [maps][groups]: out (or NULL) of the forward pass, in of the backward pass
    float eps;
    int maps, pixels, channels, groups, per;        // per: channels of a group
    int width, slices, gs, pieces, piece_items;     // columns of a slice; slices of a map; groups of a slice; slices of a group; columns of a group (with pieces)
    int by_width, by_per;                           // slices of at most 64 columns: 65536 / width and (groups of at most 128 channels) / per, rounded up; else 0
    int chunks, rows_per;                           // CTAs to the rows of a slice, and the rows of each
    float2* part;                                   // [maps][chunks * pieces][groups]: minus the mean, and squares, or the two sums of a group's gradients
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

// 1 + e^-z, and 1 / that
__device__ __forceinline__ float exp2_of(float v)
{
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(v));
    return e;
}
__device__ __forceinline__ float one_and_exp(float z) { return 1.f + exp2_of(z * -1.4426950408889634f); }
__device__ __forceinline__ float2 one_and_exp(float2 z)
{
    z = mul2(z, both<float2>(-1.4426950408889634f));
    return add2(make_float2(exp2_of(z.x), exp2_of(z.y)), both<float2>(1.f));
}
__device__ __forceinline__ float reciprocal(float v)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
// Of four values (or two): an exponential each and, JOINT, one reciprocal for all, 1 / a = bcd / abcd (the unit for both gives 16 results a cycle); where abcd is beyond a number's
// range, or none, each has its own.  Not JOINT: a value's result depends on no other.
// The exponential's argument is rounded to float32, which takes |z| 2^-24 of e^-z; exponential and reciprocal are off by a few steps.  Chosen: of z sigmoid(z) that is 6 x 2^-24 of itself at most for z > -5
// (measured; 3 as a quotient of functions without approximations), 17 down to -20, 32 down to -40, where it is 10^-16, and below -87 all of it.  Making the argument's rounding good (4, 5 and 4)
// took 4 to 11 % longer on float32 maps: 32 x 3136 x 128 24.4 us and 25.8, gradients 40.7 and 44.1.
template <bool JOINT, int STEP>
__device__ __forceinline__ void sigmoids(const float2* z, float2* p)
{
    float2 a[STEP];
#pragma unroll
    for (int h = 0; h < STEP; ++h) a[h] = one_and_exp(z[h]);
    if (JOINT) {
        const float ab = a[0].x * a[0].y, cd = STEP > 1 ? a[STEP - 1].x * a[STEP - 1].y : 1.f, t = ab * cd;
        if (t < 1e37f) {
            const float r = reciprocal(t);
            p[0] = mul2(both<float2>(STEP > 1 ? r * cd : r), make_float2(a[0].y, a[0].x));
            if (STEP > 1) p[STEP - 1] = mul2(both<float2>(r * ab), make_float2(a[STEP - 1].y, a[STEP - 1].x));
            return;
        }
    }
#pragma unroll
    for (int h = 0; h < STEP; ++h) p[h] = make_float2(reciprocal(a[h].x), reciprocal(a[h].y));
}
template <bool JOINT, int STEP> __device__ __forceinline__ void sigmoids(const float* z, float* p) { p[0] = reciprocal(one_and_exp(z[0])); }

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
            sigmoids<JOINT, STEP>(z + k, p);
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
            sigmoids<JOINT, STEP>(z + k, p);
#pragma unroll
            for (int h = 0; h < STEP; ++h) {
                // p (1 + z (1 - p))
                const F zp = mul2(z[k + h], p[h]), rest = fma2(p[h], both<F>(-1.f), both<F>(1.f));
                dy[k + h] = mul2(dy[k + h], fma2(zp, rest, p[h]));
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

// Nothing is sent to another CTA of a cluster before every one of them runs.
__device__ __forceinline__ void cluster_started(bool cluster) { if (cluster) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait(bool cluster) { if (cluster) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// A thread's place: `turns` rows of columns at once.
struct Seat { int col, turn, turns; };
__device__ __forceinline__ Seat seat_of(const GroupArgs& a, const Place& p)
{
    Seat s;
    if (a.by_width) { s.turns = (int)blockDim.x * a.by_width >> 16; s.turn = (int)threadIdx.x * a.by_width >> 16; }
    else { s.turns = (int)blockDim.x / p.cols; s.turn = (int)threadIdx.x / p.cols; }
    s.col = (int)threadIdx.x - s.turn * p.cols;
    return s;
}

// What a thread keeps of its column: the weights, and its groups' numbers.
template <typename T, int VE, bool ONE> struct Column {
    typedef typename Vec<T, VE>::F F;
    static constexpr int P = Vec<T, VE>::P, N = ONE ? 1 : P;
    F g[P], b[P];
    __device__ __forceinline__ void weights(const GroupArgs& a, const Place& p, int col)
    {
        const int c = (p.col0 + col) * VE;
        if constexpr (VE > 2)
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
    // Two numbers of each of its groups; read(group of the slice).
    template <typename R>
    static __device__ __forceinline__ void groups(const GroupArgs& a, int col, F* first, F* second, R read)
    {
#pragma unroll
        for (int k = 0; k < N; ++k) {
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

// What threads of one column have to add up: within a warp first, where its lanes hold whole rows of columns.  Returns the rows of partial sums that are left.
__device__ __forceinline__ bool folds(int cols) { return cols <= 32 && !(cols & (cols - 1)); }
template <int N, typename F>
__device__ __forceinline__ int fold(F (&v)[N], int cols, int turns)
{
    if (!folds(cols)) return turns;
    for (int o = cols; o < 32; o <<= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = add_shuffled(v[k], o);
    return (int)blockDim.x >> 5;
}
// ... and which of them this thread leaves, or none.
__device__ __forceinline__ int fold_row(const Seat& s, int cols)
{
    if (!folds(cols)) return s.turn < s.turns ? s.turn : -1;
    return (threadIdx.x & 31) < cols ? (int)(threadIdx.x >> 5) : -1;
}
// Rows of partial sums added up: a thread to each of `wide` places.
__device__ __forceinline__ float rows_of_sums(const float* part, int left, int wide, int i)
{
    float t = 0.f;
#pragma unroll 8
    for (int k = 0; k < left; ++k) t += part[k * wide + i];
    return t;
}
// Lanes to a group of so many items: a power of two.
__device__ __forceinline__ int lanes_to(int items) { return items >= 32 ? 32 : 1 << (31 - __clz(items)); }

// Means (minus them) and squares of a group's parts, joined in their order: n(i) values in part i.  {-mean, rstd}
template <typename N, typename V>
__device__ __forceinline__ float2 join_parts(int parts, float total, float eps, int sub, int lanes, N n, V value)
{
    float s = 0.f, q = 0.f;
#pragma unroll 4
    for (int i = sub; i < parts; i += lanes) s = fmaf(n(i), value(i).x, s);
    const float minus_mean = reduce_lanes<Sum>(s, lanes) / total;
#pragma unroll 4
    for (int i = sub; i < parts; i += lanes) {
        const float w = n(i);
        const float2 v = value(i);
        const float d = v.x - minus_mean;
        q += w > 0.f ? fmaf(w * d, d, v.y) : 0.f;
    }
    return make_float2(minus_mean, inverse_root(reduce_lanes<Sum>(q, lanes) / total + eps));
}

// Gradients, first half: s holds each thread's sums of dz and of dz xh.  total(place, sum) of each channel; out(group, the two sums with gamma, lane, lanes).
template <int VE, int P2, typename F, typename Total, typename Out>
__device__ __forceinline__ void finish_sums(const GroupArgs& a, const Place& p, const Seat& seat, F (&s)[P2], float* part, bool cluster, Total total, Out out)
{
    constexpr int P = P2 / 2;
    const int wide = p.cols * VE, left = fold(s, p.cols, seat.turns), to = fold_row(seat, p.cols);
    if (to >= 0)
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            part[to * 2 * wide + seat.col * VE + i] = lane_of(s[i / 2 % P], i & 1);
            part[(to * 2 + 1) * wide + seat.col * VE + i] = lane_of(s[P + i / 2 % P], i & 1);
        }
    __syncthreads();
    cluster_wait(cluster);
    for (int i = threadIdx.x; i < 2 * wide; i += blockDim.x) {
        const float t = rows_of_sums(part, left, 2 * wide, i);
        part[i] = t;                                          // (its own column alone)
        total(i, t);
    }
    __syncthreads();
    const int of = wide / p.ngroups, lanes = lanes_to(of), sub = threadIdx.x & (lanes - 1);
    for (int base = 0; base < p.ngroups; base += blockDim.x / lanes) {
        const int g = base + threadIdx.x / lanes;
        float t1 = 0.f, t2 = 0.f;
        if (g < p.ngroups)
            for (int i = g * of + sub; i < (g + 1) * of; i += lanes) {
                const float w = a.gamma ? dc_ld(a.gamma + p.col0 * VE + i) : 1.f;
                t1 = fmaf(w, part[i], t1); t2 = fmaf(w, part[wide + i], t2);
            }
        t1 = reduce_lanes<Sum>(t1, lanes); t2 = reduce_lanes<Sum>(t2, lanes);
        if (g < p.ngroups) out(g, make_float2(t1, t2), sub, lanes);
    }
}

// A row's share of a thread, and what is done to it.
template <typename T, int VE, bool ONE> struct Work {
    typedef Vec<T, VE> V;
    typedef typename V::F F;
    typedef typename V::Raw Raw;
    static constexpr int P = V::P, N = ONE ? 1 : P;
    static __device__ __forceinline__ void stats(Raw raw, const F* first, F* s)
    {
        F d[P];
        V::open(raw, d);
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const int i = ONE ? 0 : k;
            const F t = add2(d[k], first[i]);
            s[i] = add2(s[i], t);
            s[N + i] = fma2(t, t, s[N + i]);
        }
    }
    template <int ACT>
    static __device__ __forceinline__ Raw apply(Raw raw, const Column<T, VE, ONE>& c, const F* mean, const F* rstd)
    {
        F d[P];
        V::open(raw, d);
#pragma unroll
        for (int k = 0; k < P; ++k) d[k] = affine(hat(d[k], mean[ONE ? 0 : k], rstd[ONE ? 0 : k]), c.g[k], c.b[k]);
        activate<ACT, ONE>(d);
        return V::close(d);
    }
    template <int ACT>
    static __device__ __forceinline__ void back(Raw x, Raw dy, const Column<T, VE, ONE>& c, const F* mean, const F* rstd, F (&xh)[P], F (&dz)[P])
    {
        F z[P];
        V::open(x, xh);
        V::open(dy, dz);
#pragma unroll
        for (int k = 0; k < P; ++k) { xh[k] = hat(xh[k], mean[ONE ? 0 : k], rstd[ONE ? 0 : k]); z[k] = affine(xh[k], c.g[k], c.b[k]); }
        activate_back<ACT, ONE>(dz, z);
    }
    template <int ACT>
    static __device__ __forceinline__ void sums(Raw x, Raw dy, const Column<T, VE, ONE>& c, const F* mean, const F* rstd, F* s, Raw* masked)
    {
        F xh[P], dz[P];
        back<ACT>(x, dy, c, mean, rstd, xh, dz);
#pragma unroll
        for (int k = 0; k < P; ++k) { s[k] = add2(s[k], dz[k]); s[P + k] = fma2(dz[k], xh[k], s[P + k]); }
        if (ACT == DC_ACT_RELU && masked) *masked = V::close(dz);      // dy or zero: as exact as it came
    }
    // ACT: DC_ACT_NONE where dy is dz already
    template <int ACT>
    static __device__ __forceinline__ Raw gradient(Raw x, Raw dy, const Column<T, VE, ONE>& c, const F* mean, const F* rstd, const F* m1, const F* m2)
    {
        F xh[P], dz[P];
        back<ACT>(x, dy, c, mean, rstd, xh, dz);
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const int i = ONE ? 0 : k;
            xh[k] = mul2(fma2(xh[k], m2[i], add2(mul2(dz[k], c.g[k]), m1[i])), rstd[i]);
        }
        return V::close(xh);
    }
};

// What a group's distances are taken from at first: the mean of eight of its values (of equal ones: that value), in as many of the CTA's first rows as it takes.
template <typename T>
__device__ __forceinline__ float first_of(const GroupArgs& a, const Place& p, int64_t row0, int g)
{
    const char* const x = row_at(a.x, a.x_pitch, row0) + (size_t)(p.group0 + g) * a.per * sizeof(T);
    float v[8];
    int row = 0, channel = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        Vec<T, 1>::open(((const T*)(x + (size_t)min(row, p.rows - 1) * a.x_pitch))[channel], v + k);
        if (++channel == a.per) { channel = 0; ++row; }
    }
#pragma unroll
    for (int n = 4; n > 0; n /= 2)
#pragma unroll
        for (int k = 0; k < n; ++k) v[k] += v[k + n];
    return v[0] * 0.125f;
}

// Statistics of a CTA's rows: found[group] = {-mean, squares around it}.  rows(first, s) adds the distances of a thread's values from `first` and their squares to s.
// The squares around the mean are what is left of those around `first`, and next to nothing is where that lies far from the rest: a single value 1000 sigma away as `first` of 25000 took
// 5 digits from them.  So where it turns out to lie more than 2 sigma from the mean, the rows are gone through once more with the mean in its place.  (The mean of eight normal values lies within
// 2 sigma but for one group of 10^8; with one or two values in its place 4 x 50176 x 64 in 32 groups took 27.3 us, 24.1 so.)
template <typename T, int VE, bool ONE, typename Rows>
__device__ __forceinline__ void statistics(const GroupArgs& a, const Place& p, const Seat& seat, int64_t row0, float* part, float2* found, Rows rows)
{
    typedef Work<T, VE, ONE> W;
    typedef typename W::F F;
    constexpr int IT = ONE ? 1 : VE, N = W::N;
    const int items = p.cols * IT, of = items / p.ngroups, lanes = lanes_to(of), sub = threadIdx.x & (lanes - 1);
    const float n = (float)p.rows * (float)(of * (ONE ? VE : 1));
    for (int g = threadIdx.x; g < p.ngroups; g += blockDim.x) found[g].x = p.rows > 0 ? -first_of<T>(a, p, row0, g) : 0.f;
    __syncthreads();
#pragma unroll 1
    for (bool again = false;; again = true) {
        F s[2 * N], first[N], unused[N];                      // (minus what distances are taken from)
        Column<T, VE, ONE>::groups(a, seat.col, first, unused, [&](int g) { return make_float2(found[g].x, 0.f); });
#pragma unroll
        for (int k = 0; k < 2 * N; ++k) s[k] = both<F>(0.f);
        rows(first, s);
        const int left = fold(s, p.cols, seat.turns), to = fold_row(seat, p.cols);
        if (to >= 0)
#pragma unroll
            for (int i = 0; i < IT; ++i) {
                part[to * 2 * items + seat.col * IT + i] = ONE ? sum_of(s[0]) : lane_of(s[ONE ? 0 : i / 2], i & 1);
                part[(to * 2 + 1) * items + seat.col * IT + i] = ONE ? sum_of(s[N]) : lane_of(s[N + (ONE ? 0 : i / 2)], i & 1);
            }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * items; i += blockDim.x) part[i] = rows_of_sums(part, left, 2 * items, i);       // (its own column alone)
        __syncthreads();
        bool far = false;
        for (int base = 0; base < p.ngroups; base += blockDim.x / lanes) {
            const int g = base + threadIdx.x / lanes;
            float sum = 0.f, squares = 0.f;
            if (g < p.ngroups)
                for (int i = g * of + sub; i < (g + 1) * of; i += lanes) { sum += part[i]; squares += part[items + i]; }
            sum = reduce_lanes<Sum>(sum, lanes); squares = reduce_lanes<Sum>(squares, lanes);
            if (g >= p.ngroups || sub) continue;
            if (p.rows > 0) {
                const float m = sum / n, around = fmaf(-m, sum, squares);
                found[g] = make_float2(found[g].x - m, fmaxf(around, 0.f) + (sum - sum));       // (a NaN or an infinity stays one)
                far |= m * sum > 4.f * around;
            } else found[g].y = 0.f;
        }
        if (!__syncthreads_or(far) || again) return;          // found is there for all
    }
}

// ---------------------------------------------------------------------------
// Two launches: a map's rows in up to 128 chunks, sums first, the map after
// ---------------------------------------------------------------------------
// f(row, raw) of a thread's rows, four loads in flight.
template <int U, typename Raw, typename F>
__device__ __forceinline__ void each_row(const Place& p, const Seat& s, const char* x, size_t x_pitch, F f)
{
    for (int r = s.turn; r < p.rows; r += U * s.turns) {
        Raw raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = r + u * s.turns < p.rows ? *(const Raw*)(x + (size_t)(r + u * s.turns) * x_pitch) : raw_zero<Raw>();
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (r + u * s.turns < p.rows) f(r + u * s.turns, raw[u]);
    }
}
template <int U, typename Raw, typename F>
__device__ __forceinline__ void each_two(const Place& p, const Seat& s, const char* x, size_t x_pitch, const char* dy, size_t dy_pitch, F f)
{
    for (int r = s.turn; r < p.rows; r += U * s.turns) {
        Raw rx[U], rd[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool there = r + u * s.turns < p.rows;
            rx[u] = there ? *(const Raw*)(x + (size_t)(r + u * s.turns) * x_pitch) : raw_zero<Raw>();
            rd[u] = there ? *(const Raw*)(dy + (size_t)(r + u * s.turns) * dy_pitch) : raw_zero<Raw>();
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (r + u * s.turns < p.rows) f(r + u * s.turns, rx[u], rd[u]);
    }
}

// (CTAs to an SM: as many as the grid is made for, but where a thread has sums of eight groups.)
template <typename T, int VE, bool ONE>
__global__ void __launch_bounds__(kThreads, ONE && VE <= 4 ? 6 : ONE || VE <= 4 ? 5 : 4) k_group_stats(const GroupArgs a)
{
    typedef Work<T, VE, ONE> W;
    typedef typename W::F F;
    __shared__ float part[2 * kThreads * (ONE ? 1 : VE)];
    __shared__ float2 found[kThreads * (ONE ? 1 : VE)];
    dc_pdl_wait();
    dc_pdl_release();
    const Place p = place_of(a);
    const Seat seat = seat_of(a, p);
    const int64_t row0 = (int64_t)p.map * a.pixels + p.row0;
    const char* const x = row_at(a.x, a.x_pitch, row0) + (size_t)(p.col0 + seat.col) * VE * sizeof(T);
    statistics<T, VE, ONE>(a, p, seat, row0, part, found, [&](const F* first, F* s) {
        if (seat.turn < seat.turns) each_row<4, typename W::Raw>(p, seat, x, a.x_pitch, [&](int, typename W::Raw raw) { W::stats(raw, first, s); });
    });
    for (int g = threadIdx.x; g < p.ngroups; g += kThreads) a.part[((size_t)p.map * a.chunks * a.pieces + p.chunk * a.pieces + p.piece) * a.groups + p.group0 + g] = found[g];
}

// join(group of the slice, whether there is one, lane, lanes): a slice's groups, as many lanes to each as there are parts to join, but so few that all groups go at once.
template <typename J>
__device__ __forceinline__ void each_group(const GroupArgs& a, const Place& p, J join)
{
    int lanes = lanes_to(a.chunks * a.pieces);
    while (lanes > 1 && lanes * p.ngroups > (int)blockDim.x) lanes >>= 1;
    const int sub = threadIdx.x & (lanes - 1);
    for (int base = 0; base < p.ngroups; base += blockDim.x / lanes) {
        const int g = base + threadIdx.x / lanes;
        join(min(g, p.ngroups - 1), g < p.ngroups, sub, lanes);
    }
    __syncthreads();
}
// The values of part i of a group.
template <int VE>
__device__ __forceinline__ float part_size(const GroupArgs& a, int i)
{
    if (a.pieces == 1) return (float)rows_of(a, i) * (float)a.per;
    const int chunk = i / a.pieces;
    return (float)rows_of(a, chunk) * (float)(cols_of(a, i - chunk * a.pieces) * VE);
}

template <typename T, int VE, bool ONE, int ACT>
__global__ void __launch_bounds__(kThreads) k_group_apply(const GroupArgs a)
{
    typedef Work<T, VE, ONE> W;
    typedef typename W::F F;
    __shared__ float2 fin[kThreads * (ONE ? 1 : VE)];
    dc_pdl_wait();
    dc_pdl_release();
    const Place p = place_of(a);
    const Seat seat = seat_of(a, p);
    Column<T, VE, ONE> c;
    c.weights(a, p, seat.col);
    each_group(a, p, [&](int g, bool on, int sub, int lanes) {
        const float2* const part = a.part + (size_t)p.map * a.chunks * a.pieces * a.groups + p.group0 + g;
        const float2 r = join_parts(a.chunks * a.pieces, (float)a.pixels * (float)a.per, a.eps, sub, lanes, [&](int i) { return part_size<VE>(a, i); },
                                    [&](int i) { return dc_ld(part + (size_t)i * a.groups); });
        if (!on || sub) return;
        fin[g] = r;
        if (p.chunk == 0 && p.piece == 0) {
            if (a.mean) a.mean[(size_t)p.map * a.groups + p.group0 + g] = -r.x;
            if (a.rstd) a.rstd[(size_t)p.map * a.groups + p.group0 + g] = r.y;
        }
    });
    if (seat.turn >= seat.turns) return;
    F mean[W::N], rstd[W::N];
    c.groups(a, seat.col, mean, rstd, [&](int g) { return fin[g]; });
    const int64_t row0 = (int64_t)p.map * a.pixels + p.row0;
    const size_t at = (size_t)(p.col0 + seat.col) * VE * sizeof(T);
    char* const y = row_at(a.y, a.y_pitch, row0) + at;
    each_row<4, typename W::Raw>(p, seat, row_at(a.x, a.x_pitch, row0) + at, a.x_pitch,
                                 [&](int r, typename W::Raw raw) { *(typename W::Raw*)(y + (size_t)r * a.y_pitch) = W::template apply<ACT>(raw, c, mean, rstd); });
}

template <typename T, int VE, bool ONE, int ACT>
__global__ void __launch_bounds__(kThreads) k_group_back_sums(const GroupArgs a)
{
    typedef Work<T, VE, ONE> W;
    typedef typename W::F F;
    __shared__ float part[2 * kThreads * VE];
    dc_pdl_wait();
    dc_pdl_release();
    const Place p = place_of(a);
    const Seat seat = seat_of(a, p);
    Column<T, VE, ONE> c;
    F mean[W::N], rstd[W::N], s[2 * W::P];
    c.weights(a, p, seat.col);
    const size_t of = (size_t)p.map * a.groups + p.group0;
    c.groups(a, seat.col, mean, rstd, [&](int g) { return make_float2(-dc_ld(a.mean + of + g), dc_ld(a.rstd + of + g)); });
#pragma unroll
    for (int k = 0; k < 2 * W::P; ++k) s[k] = both<F>(0.f);
    const int64_t row0 = (int64_t)p.map * a.pixels + p.row0;
    const size_t at = (size_t)(p.col0 + seat.col) * VE * sizeof(T);
    if (seat.turn < seat.turns)
        each_two<2, typename W::Raw>(p, seat, row_at(a.x, a.x_pitch, row0) + at, a.x_pitch, row_at(a.dy, a.dy_pitch, row0) + at, a.dy_pitch,
                                     [&](int, typename W::Raw x, typename W::Raw dy) { W::template sums<ACT>(x, dy, c, mean, rstd, s, nullptr); });
    const int wide = p.cols * VE;
    finish_sums<VE>(a, p, seat, s, part, false,
        [&](int i, float t) { if (a.sums) a.sums[((size_t)p.map * a.chunks + p.chunk) * 2 * a.channels + (i < wide ? p.col0 * VE + i : a.channels + p.col0 * VE + i - wide)] = t; },
        [&](int g, float2 r, int sub, int) {
            if (sub == 0) a.part[((size_t)p.map * a.chunks * a.pieces + p.chunk * a.pieces + p.piece) * a.groups + p.group0 + g] = r;
        });
}

template <typename T, int VE, bool ONE, int ACT>
__global__ void __launch_bounds__(kThreads) k_group_back_apply(const GroupArgs a)
{
    typedef Work<T, VE, ONE> W;
    typedef typename W::F F;
    __shared__ float2 fin[kThreads * (ONE ? 1 : VE)];
    dc_pdl_wait();
    dc_pdl_release();
    const Place p = place_of(a);
    const Seat seat = seat_of(a, p);
    Column<T, VE, ONE> c;
    c.weights(a, p, seat.col);
    each_group(a, p, [&](int g, bool on, int sub, int lanes) {
        const float2* const part = a.part + (size_t)p.map * a.chunks * a.pieces * a.groups + p.group0 + g;
        float t1 = 0.f, t2 = 0.f;
        for (int i = sub; i < a.chunks * a.pieces; i += lanes) { const float2 v = dc_ld(part + (size_t)i * a.groups); t1 += v.x; t2 += v.y; }
        t1 = reduce_lanes<Sum>(t1, lanes); t2 = reduce_lanes<Sum>(t2, lanes);
        const float total = (float)a.pixels * (float)a.per;
        if (on && sub == 0) fin[g] = make_float2(-t1 / total, -t2 / total);
    });
    if (seat.turn >= seat.turns) return;
    F mean[W::N], rstd[W::N], m1[W::N], m2[W::N];
    const size_t of = (size_t)p.map * a.groups + p.group0;
    c.groups(a, seat.col, mean, rstd, [&](int g) { return make_float2(-dc_ld(a.mean + of + g), dc_ld(a.rstd + of + g)); });
    c.groups(a, seat.col, m1, m2, [&](int g) { return fin[g]; });
    const int64_t row0 = (int64_t)p.map * a.pixels + p.row0;
    const size_t at = (size_t)(p.col0 + seat.col) * VE * sizeof(T);
    char* const dx = row_at(a.y, a.y_pitch, row0) + at;
    each_two<2, typename W::Raw>(p, seat, row_at(a.x, a.x_pitch, row0) + at, a.x_pitch, row_at(a.dy, a.dy_pitch, row0) + at, a.dy_pitch,
                                 [&](int r, typename W::Raw x, typename W::Raw dy) { *(typename W::Raw*)(dx + (size_t)r * a.y_pitch) = W::template gradient<ACT>(x, dy, c, mean, rstd, m1, m2); });
}

// ---------------------------------------------------------------------------
// One launch: a slice of a map in the shared memory of a cluster, read once
// ---------------------------------------------------------------------------
constexpr int kMostResident = 512;                            // threads
constexpr int kMostCluster = 8, kMostGroups = 64, kMostColumns = 64;       // CTAs to a slice; groups, columns of one

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// To the same place in CTA `rank` of the cluster.
__device__ __forceinline__ uint32_t place_in(const void* at, int rank)
{
    uint32_t to;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"((uint32_t)__cvta_generic_to_shared(at)), "r"(rank));
    return to;
}
__device__ __forceinline__ void send(const float2* at, int rank, float2 v)
{
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(place_in(at, rank)), "f"(v.x), "f"(v.y) : "memory");
}
__device__ __forceinline__ void send(const float* at, int rank, float v)
{
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(place_in(at, rank)), "f"(v) : "memory");
}
__device__ __forceinline__ Place resident_place(const GroupArgs& a)
{
    Place p;
    p.chunk = blockIdx.x; p.map = blockIdx.z; p.piece = 0; p.ngroups = a.gs; p.cols = a.width;
    p.group0 = blockIdx.y * a.gs; p.col0 = blockIdx.y * a.width; p.row0 = p.chunk * a.rows_per; p.rows = rows_of(a, p.chunk);
    return p;
}
// A thread's own values of a map into shared memory, one behind another for the threads; they are there once copies_done() has passed.
template <typename Raw>
__device__ __forceinline__ void keep_rows(const Place& p, const Seat& s, const char* x, size_t pitch, Raw* kept)
{
    if (s.turn >= s.turns) return;
    Raw* to = kept + threadIdx.x;
    const int line = s.turns * p.cols;
    x += (size_t)s.turn * pitch;
    const size_t step = (size_t)s.turns * pitch;
    if constexpr (sizeof(Raw) >= 4) {
        uint32_t at = (uint32_t)__cvta_generic_to_shared(to);
        for (int r = s.turn; r < p.rows; r += s.turns, at += (uint32_t)sizeof(Raw) * line, x += step)
            if constexpr (sizeof(Raw) == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(x) : "memory");
            else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(x), "n"((int)sizeof(Raw)) : "memory");
    } else {
#pragma unroll 8
        for (int r = s.turn; r < p.rows; r += s.turns, to += line, x += step) *to = *(const Raw*)x;
    }
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__host__ __device__ constexpr size_t up16(size_t n) { return (n + 15) / 16 * 16; }

// A CTA has rows_per rows of a slice; its cluster has the slice.  Each thread copies its own values into shared memory and reads them twice from there (three times at most: statistics()).
// Registers: 64 at most, so that four CTAs of 256 threads fit an SM; 80, and three, where a thread has sums of eight groups.
template <typename T, int VE, bool ONE, int ACT>
__global__ void __launch_bounds__(ONE || VE <= 4 ? kMostResident : 768, ONE || VE <= 4 ? 2 : 1) k_group_resident(const GroupArgs a)
{
    typedef Work<T, VE, ONE> W;
    typedef typename W::F F;
    typedef typename W::Raw Raw;
    extern __shared__ uint4 shared4[];                        // [rows_per][columns], then the partial sums
    __shared__ float2 exchange[kMostCluster][kMostGroups], fin[kMostGroups];
    const bool cluster = a.chunks > 1;
    cluster_started(cluster);
    dc_pdl_wait();
    dc_pdl_release();
    const Place p = resident_place(a);
    const Seat seat = seat_of(a, p);
    const int64_t row0 = (int64_t)p.map * a.pixels + p.row0;
    const size_t at = (size_t)(p.col0 + seat.col) * VE * sizeof(T);
    Raw* const kept = (Raw*)shared4;
    keep_rows(p, seat, row_at(a.x, a.x_pitch, row0) + at, a.x_pitch, kept);
    float* const part = (float*)((char*)shared4 + up16((size_t)a.rows_per * p.cols * sizeof(Raw)));      // [rows of partial sums][sums, squares][items]
    Column<T, VE, ONE> c;
    c.weights(a, p, seat.col);
    const int line = seat.turns * p.cols;
    statistics<T, VE, ONE>(a, p, seat, row0, part, fin, [&](const F* first, F* s) {
        copies_done();
        if (seat.turn >= seat.turns) return;
        const Raw* k4 = kept + threadIdx.x;
#pragma unroll 4
        for (int r = seat.turn; r < p.rows; r += seat.turns, k4 += line) W::stats(*k4, first, s);
    });
    cluster_wait(cluster);
    for (int rank = threadIdx.x / kMostGroups, g = threadIdx.x % kMostGroups; rank < a.chunks && g < p.ngroups; rank += blockDim.x / kMostGroups) send(&exchange[p.chunk][g], rank, fin[g]);
    if (cluster) cluster_sync(); else __syncthreads();
    if (threadIdx.x < p.ngroups) {
        const int g = threadIdx.x;
        const float2 r = join_parts(a.chunks, (float)a.pixels * (float)a.per, a.eps, 0, 1, [&](int i) { return (float)rows_of(a, i) * (float)a.per; }, [&](int i) { return exchange[i][g]; });
        fin[g] = r;
        if (p.chunk == 0) {
            if (a.mean) a.mean[(size_t)p.map * a.groups + p.group0 + g] = -r.x;
            if (a.rstd) a.rstd[(size_t)p.map * a.groups + p.group0 + g] = r.y;
        }
    }
    __syncthreads();
    if (seat.turn >= seat.turns) return;
    F mean[W::N], rstd[W::N];
    c.groups(a, seat.col, mean, rstd, [&](int g) { return fin[g]; });
    char* y = row_at(a.y, a.y_pitch, row0 + seat.turn) + at;
    const Raw* k4 = kept + threadIdx.x;
#pragma unroll 4
    for (int r = seat.turn; r < p.rows; r += seat.turns, k4 += line, y += seat.turns * a.y_pitch) *(Raw*)y = W::template apply<ACT>(*k4, c, mean, rstd);
}

// The gradients likewise: x and dy are kept (behind a ReLU dy or zero, which is as exact).  SiLU's derivative is worked out twice: 32 maps of 56 x 56 x 256 bf16 55 us; with dz
// kept as floats, which leaves an SM two CTAs in the place of four, 61.
template <typename T, int VE, bool ONE, int ACT>
__global__ void __launch_bounds__(kMostResident, ONE ? 2 : 1) k_group_back_resident(const GroupArgs a)
{
    typedef Work<T, VE, ONE> W;
    typedef typename W::F F;
    typedef typename W::Raw Raw;
    extern __shared__ uint4 shared4[];                        // [2][rows_per][columns], then the partial sums
    __shared__ float2 exchange[kMostCluster][kMostGroups], fin[kMostGroups];
    const bool cluster = a.chunks > 1;
    cluster_started(cluster);
    dc_pdl_wait();
    dc_pdl_release();
    const Place p = resident_place(a);
    const Seat seat = seat_of(a, p);
    const int wide = p.cols * VE, line = seat.turns * p.cols;
    const int64_t row0 = (int64_t)p.map * a.pixels + p.row0;
    const size_t at = (size_t)(p.col0 + seat.col) * VE * sizeof(T), half = up16((size_t)a.rows_per * p.cols * sizeof(Raw));
    Raw *const kept = (Raw*)shared4, *const kept_dy = (Raw*)((char*)shared4 + half);
    keep_rows(p, seat, row_at(a.x, a.x_pitch, row0) + at, a.x_pitch, kept);
    keep_rows(p, seat, row_at(a.dy, a.dy_pitch, row0) + at, a.dy_pitch, kept_dy);
    float* const part = (float*)((char*)shared4 + 2 * half);             // [rows of partial sums][2][channels]
    Column<T, VE, ONE> c;
    c.weights(a, p, seat.col);
    F mean[W::N], rstd[W::N], s[2 * W::P];
    const size_t of_map = (size_t)p.map * a.groups + p.group0;
    c.groups(a, seat.col, mean, rstd, [&](int g) { return make_float2(-dc_ld(a.mean + of_map + g), dc_ld(a.rstd + of_map + g)); });
#pragma unroll
    for (int k = 0; k < 2 * W::P; ++k) s[k] = both<F>(0.f);
    copies_done();
    if (seat.turn < seat.turns) {
        const Raw* x = kept + threadIdx.x;
        Raw* dy = kept_dy + threadIdx.x;
#pragma unroll 2
        for (int r = seat.turn; r < p.rows; r += seat.turns, x += line, dy += line) W::template sums<ACT>(*x, *dy, c, mean, rstd, s, dy);
    }
    const int left = folds(p.cols) ? (int)blockDim.x >> 5 : seat.turns;
    float* const sums_of_all = part + (size_t)left * 2 * wide;           // [chunks][2][channels]: of a single map, in the first CTA
    finish_sums<VE>(a, p, seat, s, part, cluster,
        [&](int i, float t) {
            if (a.dgamma || a.dbeta) send(sums_of_all + p.chunk * 2 * wide + i, 0, t);
            else if (a.sums) a.sums[((size_t)p.map * a.chunks + p.chunk) * 2 * a.channels + (i < wide ? p.col0 * VE + i : a.channels + p.col0 * VE + i - wide)] = t;
        },
        [&](int g, float2 r, int sub, int lanes) {
            for (int rank = sub; rank < a.chunks; rank += lanes) send(&exchange[p.chunk][g], rank, r);
        });
    if (cluster) cluster_sync(); else __syncthreads();
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
    if (seat.turn >= seat.turns) return;
    F m1[W::N], m2[W::N];
    c.groups(a, seat.col, m1, m2, [&](int g) { return fin[g]; });
    char* dx = row_at(a.y, a.y_pitch, row0 + seat.turn) + at;
    const Raw *x = kept + threadIdx.x, *dy = kept_dy + threadIdx.x;
    constexpr int LEFT = ACT == DC_ACT_RELU ? DC_ACT_NONE : ACT;         // of the activation, behind the first half
#pragma unroll 2
    for (int r = seat.turn; r < p.rows; r += seat.turns, x += line, dy += line, dx += seat.turns * a.y_pitch) *(Raw*)dx = W::template gradient<LEFT>(*x, *dy, c, mean, rstd, m1, m2);
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
bool plan_columns(GroupArgs& a, int ve, int elt)
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
        if (units % j == 0 && j * least <= kThreads && best * least * ve * elt < 64) best = j;             // 64 bytes of a row or more
    a.gs = best * unit; a.width = best * least; a.slices = units / best;
    if (a.width <= kMostColumns) {
        a.by_width = dc_div_up(65536, a.width);
        a.by_per = a.per <= 128 ? dc_div_up(65536, a.per) : 0;
    }
    return true;
}

// A slice in the shared memory of a cluster, if it fits: columns of 64 bytes a row, CTAs of up to 56 KB, four to an SM, so that some load while others compute
// and store, or as many as a cluster has, or larger ones; 256 threads, 128 where those would have fewer than four vectors each, 512 in CTAs of more than 110 KB (8 x 12544 x 250 in 5 groups 57 us and 72).  32 maps of 56 x 56 x 256 bf16, SiLU, us: forward 28.9
// (columns of 32 bytes 34.2, of 128 34.6; 25 KB 30.5, 100 KB 40), gradients 55.1 (60.5, 61; 100 KB and more 80).  What does not fit, and large CTAs that do not even fill the SMs, are left to two launches
// with more of them: 4 x 50176 x 64, gradients, 45 us, with columns of 32 bytes 73; 16629 x 32, one map, 12.6 us and 9.1; 9273 x 32 8.6 and 8.0, 8 x 12544 x 64 16.7 and 21.4, 7241 x 320 10.7 and 16.8.
constexpr int kWantKept = 56 * 1024, kMostKept = 200 * 1024, kFewKept = 120 * 1024, kLargeKept = 110 * 1024;
bool plan_resident(GroupArgs& a, int ve, int elt, int planes, int num_sms, int* block, size_t* smem)
{
    const int least = a.per / gcd(a.per, ve), unit = least * ve / a.per, column = ve * elt, bytes = column * planes;
    if (a.channels % ve || a.groups % unit || least > kMostColumns || a.maps > 65535) return false;
    const int units = a.groups / unit;
    int best = 0;
    for (int j = 1; j <= units && j * least <= kMostColumns; ++j) {
        if (units % j || j * unit > kMostGroups) continue;
        if ((int64_t)a.pixels * j * least * bytes > (int64_t)kMostCluster * kMostKept) return false;
        best = j;
        if (j * least * column >= 64) break;
    }
    if (!best || (int64_t)units / best > 65535) return false;
    a.pieces = 1; a.gs = best * unit; a.width = best * least; a.slices = units / best;
    const int64_t slice = (int64_t)a.pixels * a.width * bytes;
    int turns = 256 / a.width;
    a.by_width = dc_div_up(65536, a.width); a.by_per = a.per <= 128 ? dc_div_up(65536, a.per) : 0;
    int cs = 1;
    while (cs < kMostCluster && (slice > (int64_t)cs * kWantKept || ((int64_t)a.maps * a.slices * cs < num_sms && a.pixels >= 4 * cs * turns))) cs *= 2;
    if (cs > most_chunks(a.maps, a.pixels) || (slice > (int64_t)cs * kFewKept * planes && (int64_t)a.maps * a.slices * cs < num_sms)) return false;
    a.rows_per = dc_div_up(a.pixels, cs);
    a.chunks = cs;
    const int64_t columns = (int64_t)a.rows_per * a.width;
    const int threads = columns * bytes > kLargeKept ? 512 : columns >= 4 * 256 ? 256 : 128;
    turns = threads / a.width;
    const int left = a.width > 32 || a.width & (a.width - 1) ? turns : threads / 32;
    *block = threads;
    *smem = planes * up16((size_t)a.rows_per * a.width * column) + (size_t)(left + (a.dgamma || a.dbeta ? cs : 0)) * 2 * a.width * ve * sizeof(float);
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
    GroupArgs r = a;
    size_t smem = 0;
    int block = 0;
    if (a.maps > 1) r.dgamma = r.dbeta = nullptr;
    if (plan_resident(r, VE, (int)sizeof(T), back ? 2 : 1, num_sms, &block, &smem)) {      // kept: x, and dy
        a.joined = r.dgamma || r.dbeta;
        a.chunks = r.chunks;                                  // (for the join of the sums)
        return launch_resident<T, VE, ONE, ACT>(r, back, block, smem, device, stream);
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
    if constexpr (VE > 2)
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
    const bool rows = (int64_t)a.maps * a.pixels > 1;
    auto aligned = [&](size_t by) {
        auto one = [&](const void* p, size_t pitch) { return (uintptr_t)p % by == 0 && (!rows || pitch % by == 0); };
        return one(a.x, a.x_pitch) && (!a.y || one(a.y, a.y_pitch)) && (!back || one(a.dy, a.dy_pitch));
    };
    // 16 bytes of a row to a thread, or two elements of one group, or one
    const int at_once = aligned(16) && plan_columns(a, ve, elt) ? ve : aligned(2 * elt) && a.per % 2 == 0 && plan_columns(a, 2, elt) ? 2 : 1;
    if (at_once == 1) plan_columns(a, 1, elt);
    const int most = most_chunks(a.maps, a.pixels), turns = kThreads / a.width;
    // Eight CTAs to an SM with 16 rows to a thread or more (what a CTA does but once would outweigh the work of more), or two with four or more; at most 64.
    const int64_t units = (int64_t)a.maps * a.slices;
    auto of = [&](int rows, int per_sm) { const int64_t c = dc_div_up(a.pixels, rows * turns), w = (per_sm * (int64_t)sms + units - 1) / units; return (int)(c < w ? c : w); };
    a.chunks = of(4, 2) > of(16, 8) ? of(4, 2) : of(16, 8);
    if (a.chunks < dc_div_up(a.pixels, 64 * turns)) a.chunks = dc_div_up(a.pixels, 64 * turns);
    if (a.chunks > most) a.chunks = most;
    a.rows_per = dc_div_up(a.pixels, a.chunks);
    a.chunks = dc_div_up(a.pixels, a.rows_per);
    if ((int64_t)a.maps * a.slices * a.chunks > 0x7fffffff) return DC_ERR_LIMIT;
#define DC_GROUP(T, VE) DC_CUDA((launch_group_as<T, VE>(a, back, activation, device, sms, stream)))
    if (dtype == DC_BF16) { if (at_once == 8) DC_GROUP(__nv_bfloat16, 8); else if (at_once == 2) DC_GROUP(__nv_bfloat16, 2); else DC_GROUP(__nv_bfloat16, 1); }
    else if (at_once == 4) DC_GROUP(float, 4);
    else if (at_once == 2) DC_GROUP(float, 2);
    else DC_GROUP(float, 1);
#undef DC_GROUP
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
