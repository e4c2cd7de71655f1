// Layer normalisation over the channels of a pixel, its gradients, and rows in 8 bits with a scale of their own.
//
//   mean = sum x / C,  rstd = 1 / sqrt(sum (x - mean)^2 / C + eps),  y = (x - mean) rstd gamma + beta
//   with xh = (x - mean) rstd, g = dy gamma:  dx = rstd (g - mean(g) - xh mean(g xh)),  dgamma = sum over rows dy xh,  dbeta = sum over rows dy
//   a = max |x|,  scale = a / 127,  q = the integer next to 127 x / a (halves to even)
//
// What bounds them: memory, one read and one write of the map (two reads and a write for the gradients).  So a row is read once, into
// registers, by a group of 1 to 32 lanes or by a CTA, and everything that it needs (the mean, the squares around it, the largest value) is
// reduced among those.  Sums are float32 whatever the map's type; the squares are taken around the mean, not from a sum of squares,
// which loses what a row with a large mean has left.
#include <string.h>

#include "dc_rows.cuh"

namespace {

constexpr int kBackwardCtas = 296;      // partial sums of a gradient's columns: two CTAs for each SM of a B200

// Two floats at once: what bounds these kernels next to memory is the instructions per element.
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\tfma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
// The same of a single element, for rows that are read one by one.
__device__ __forceinline__ float add2(float a, float b) { return a + b; }
__device__ __forceinline__ float mul2(float a, float b) { return a * b; }
__device__ __forceinline__ float fma2(float a, float b, float c) { return fmaf(a, b, c); }
template <typename F> __device__ __forceinline__ F both(float a);
template <> __device__ __forceinline__ float both<float>(float a) { return a; }
template <> __device__ __forceinline__ float2 both<float2>(float a) { return make_float2(a, a); }
__device__ __forceinline__ float sum_of(float a) { return a; }
__device__ __forceinline__ float sum_of(float2 a) { return a.x + a.y; }
__device__ __forceinline__ uint32_t size_bits(float a) { return __float_as_uint(a) & 0x7fffffffu; }
__device__ __forceinline__ float largest(float2 a) { return fmaxf(fabsf(a.x), fabsf(a.y)); }
__device__ __forceinline__ float add_shuffled(float a, int o) { return a + __shfl_xor_sync(0xffffffffu, a, o); }
__device__ __forceinline__ float2 add_shuffled(float2 a, int o) { return make_float2(add_shuffled(a.x, o), add_shuffled(a.y, o)); }

// VE elements of a row: 16 bytes at once, or one element where alignment or the row's length do not allow that.  A lane's elements are
// kept as pairs of floats (F), P per vector, or as single ones.
template <typename T, int VE> struct Vec;
template <> struct Vec<float, 4> {
    typedef float4 Raw; typedef float2 F;
    static constexpr int P = 2;
    static __device__ __forceinline__ void open(Raw t, float2* v) { v[0] = make_float2(t.x, t.y); v[1] = make_float2(t.z, t.w); }
    static __device__ __forceinline__ Raw close(const float2* v) { return make_float4(v[0].x, v[0].y, v[1].x, v[1].y); }
};
template <> struct Vec<__nv_bfloat16, 8> {
    typedef uint4 Raw; typedef float2 F;
    static constexpr int P = 4;
    static __device__ __forceinline__ void open(Raw t, float2* v)
    {
        const uint32_t w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = make_float2(__uint_as_float(w[k] << 16), __uint_as_float(w[k] & 0xffff0000u));
    }
    static __device__ __forceinline__ Raw close(const float2* v)
    {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) { const __nv_bfloat162 t = __floats2bfloat162_rn(v[k].x, v[k].y); w[k] = *(const uint32_t*)&t; }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <> struct Vec<float, 1> {
    typedef float Raw; typedef float F;
    static constexpr int P = 1;
    static __device__ __forceinline__ void open(Raw t, float* v) { v[0] = t; }
    static __device__ __forceinline__ Raw close(const float* v) { return v[0]; }
};
template <> struct Vec<__nv_bfloat16, 1> {
    typedef __nv_bfloat16 Raw; typedef float F;
    static constexpr int P = 1;
    static __device__ __forceinline__ void open(Raw t, float* v) { v[0] = __bfloat162float(t); }
    static __device__ __forceinline__ Raw close(const float* v) { return __float2bfloat16_rn(v[0]); }
};
// The larger of m and the bits of a vector's sizes: two bfloat16 side by side, which most_of() joins.
__device__ __forceinline__ uint32_t raw_most(uint32_t m, uint4 t)
{
    m = __vmaxu2(m, t.x & 0x7fff7fffu); m = __vmaxu2(m, t.y & 0x7fff7fffu);
    m = __vmaxu2(m, t.z & 0x7fff7fffu); return __vmaxu2(m, t.w & 0x7fff7fffu);
}
__device__ __forceinline__ uint32_t raw_most(uint32_t m, float4 t)
{
    m = max(max(m, size_bits(t.x)), size_bits(t.y));
    return max(max(m, size_bits(t.z)), size_bits(t.w));
}
__device__ __forceinline__ uint32_t raw_most(uint32_t m, float t) { return max(m, size_bits(t)); }
__device__ __forceinline__ uint32_t raw_most(uint32_t m, __nv_bfloat16 t) { return max(m, (uint32_t)__bfloat16_as_ushort(t) & 0x7fffu); }
template <typename T> __device__ __forceinline__ uint32_t most_of(uint32_t m) { return sizeof(T) == 2 ? max(m >> 16, m & 0xffffu) << 16 : m; }
template <typename R> __device__ __forceinline__ R raw_zero() { R r; memset(&r, 0, sizeof(r)); return r; }

// The weights of VE channels; p NULL: `fill`.  Read after the wait for the kernel before, which may have written them.
__device__ __forceinline__ void load_weights(const float* p, int at, float fill, float (&v)[1]) { v[0] = p ? dc_ld(p + at) : fill; }
template <int P>
__device__ __forceinline__ void load_weights(const float* p, int at, float fill, float2 (&v)[P])
{
#pragma unroll
    for (int k = 0; k < P; k += 2) {
        const float4 t = p ? dc_ld((const float4*)(p + at + 2 * k)) : make_float4(fill, fill, fill, fill);
        v[k] = make_float2(t.x, t.y); v[k + 1] = make_float2(t.z, t.w);
    }
}

struct Sum { static __device__ __forceinline__ float of(float a, float b) { return a + b; } };
struct Most { static __device__ __forceinline__ uint32_t of(uint32_t a, uint32_t b) { return a > b ? a : b; } };

// Over the lanes of a group (a power of two), or over the CTA: each reduction of a row has a slot of its own, and rows alternate between two
// sets of them, so one barrier per reduction is enough.
template <typename Op, typename V>
__device__ __forceinline__ V reduce_lanes(V v, int group)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)                             // steps beyond the group are passed over: no loop to count
        if (o < group) v = Op::of(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
// The largest of a whole warp is one instruction.
template <> __device__ __forceinline__ uint32_t reduce_lanes<Most, uint32_t>(uint32_t v, int group)
{
    if (group == 32) return __reduce_max_sync(0xffffffffu, v);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1)
        if (o < group) v = Most::of(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
template <typename Op, bool BLOCK, typename V>
__device__ __forceinline__ V reduce(V v, int group, V* slot)
{
    if (!BLOCK) return reduce_lanes<Op>(v, group);
    v = reduce_lanes<Op>(v, 32);
    if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = v;
    __syncthreads();
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    V t = lane < warps ? slot[lane] : V(0);
    return reduce_lanes<Op>(t, 32);
}

// s / c by the reciprocal of c and a correction of the remainder: half a step, as the division, at a third of its instructions.  (An
// infinite s gives NaN.)
__device__ __forceinline__ float over(float s, float c, float inv_c)
{
    const float q = s * inv_c;
    return fmaf(fmaf(-q, c, s), inv_c, q);
}
// 1 / sqrt(v): the fast root (error below 2^-22) and one step of Newton's, but for zero and infinity, where that step is NaN.
__device__ __forceinline__ float inverse_root(float v)
{
    const float r = rsqrtf(v), e = fmaf(-0.5f * v * r, r, 0.5f);
    return e == e ? fmaf(r, e, r) : r;
}

// The values of a row in 127 steps of its largest, `most` > 0, either way; exact: the real quotient 127 x / most, halves to even.  inv: 1 / most, off by less
// than 2^-22 of itself.
// bfloat16: 127 x is exact, one step of Newton's makes the quotient the float next to the real one, and a real one that is not a half
// is off it by a 2^-17th of itself at least: with x = i 2^a and most = j 2^b, i and j from 128 to 255, 254 x and an odd multiple of most
// differ by 2^min(a, b) or not at all.  Halves are common there (0.1 % of a map), so nothing may branch on them.
// float32: 127 x / most is off by less than 2^-15, so only next to a half it is looked at again, in products that 64 bits hold exactly.
__device__ __noinline__ int quantise_next_to_half(float x, float r, float most)
{
    const float f = floorf(fabsf(r));
    const double d = 127.0 * fabs((double)x) - ((double)f + 0.5) * (double)most;
    int n = (int)f;
    if (d > 0.0 || (d == 0.0 && (n & 1))) ++n;
    return x < 0.f ? -n : n;
}
constexpr float kRound = 12582912.f;    // 1.5 * 2^23: adding it leaves the nearest integer, of two the even one, in the low bits
constexpr float kHalf = 0.5f - 0x1p-14f;
template <typename F>
__device__ __forceinline__ F quotient(F x, F inv, F minus_most)        // 127 x / most for bfloat16 x
{
    const F n = mul2(x, both<F>(127.f)), q = mul2(n, inv);
    return fma2(fma2(q, minus_most, n), inv, q);
}
template <typename T, int VE>
__device__ __forceinline__ void quantise(const float* x, float inv, float most, uint32_t* q)
{
    const float r = sizeof(T) == 2 ? quotient(x[0], inv, -most) : x[0] * (127.f * inv), t = r + kRound;
    q[0] = __float_as_uint(t);
    if (sizeof(T) == 4 && fabsf(r - (t - kRound)) > kHalf) q[0] = (uint32_t)quantise_next_to_half(x[0], r, most);
}
template <typename T, int VE>
__device__ __forceinline__ void quantise(const float2* x, float inv, float most, uint32_t* q)
{
    uint32_t b[VE];
    float far = 0.f;
    const float2 inv2 = both<float2>(sizeof(T) == 2 ? inv : 127.f * inv), round = both<float2>(kRound), minus = both<float2>(-1.f);
#pragma unroll
    for (int k = 0; k < VE / 2; ++k) {
        const float2 r = sizeof(T) == 2 ? quotient(x[k], inv2, both<float2>(-most)) : mul2(x[k], inv2), t = add2(r, round);
        if (sizeof(T) == 4) far = fmaxf(far, largest(add2(r, fma2(t, minus, round))));
        b[2 * k] = __float_as_uint(t.x); b[2 * k + 1] = __float_as_uint(t.y);
    }
    if (sizeof(T) == 4 && far > kHalf) {
#pragma unroll
        for (int k = 0; k < VE; ++k) quantise<T, 1>(k & 1 ? &x[k / 2].y : &x[k / 2].x, inv, most, b + k);
    }
#pragma unroll
    for (int k = 0; k < VE; k += 4) q[k / 4] = __byte_perm(__byte_perm(b[k], b[k + 1], 0x0040), __byte_perm(b[k + 2], b[k + 3], 0x0040), 0x5410);
}
template <int VE>
__device__ __forceinline__ void store_q(int8_t* p, const uint32_t* q)
{
    if constexpr (VE == 8) *(uint2*)p = make_uint2(q[0], q[1]);
    else if constexpr (VE == 4) *(uint32_t*)p = q[0];
    else *p = (int8_t)q[0];
}
// What a row's largest bits say of it: its scale, the inverse of `most`, and a power of two that first moves rows of very small or very large
// numbers to where that inverse is a normal number.  A row with an infinity or a NaN gets the scale NaN and zeros.
struct RowScale { float scale, inv, most, lift; };
__device__ __forceinline__ RowScale row_scale(uint32_t bits)
{
    RowScale s;
    s.most = __uint_as_float(bits);
    s.lift = 1.f;
    s.scale = over(s.most, 127.f, 1.f / 127.f);
    if (bits < 0x21800000u || bits >= 0x71800000u) {             // below 2^-60 (a row of zeros too), from 2^100 on
        s.scale = bits >= 0x7f800000u ? __uint_as_float(0x7fffffffu) : s.most / 127.f;
        s.lift = bits >= 0x7f800000u ? 0.f : bits < 0x21800000u ? 0x1p64f : 0x1p-64f;
        s.most = bits >= 0x7f800000u || bits == 0 ? 1.f : s.most * s.lift;
    }
    asm("rcp.approx.f32 %0, %1;" : "=f"(s.inv) : "f"(s.most));
    return s;
}

// A row's place in q and scale: see dc_rows_args.
__device__ __forceinline__ int q_row(const dc_rows_args& a, int row)
{
    if (a.padded == 0) return row;
    const int line = row / a.width;
    return line * a.padded + (row - line * a.width);
}
// Row `row` of a map: rows and pitches are below 2^32, so the place is one multiplication of 32 bits by 32.
__device__ __forceinline__ char* row_at(const void* p, size_t pitch, int row) { return (char*)p + (uint64_t)(uint32_t)row * (uint32_t)pitch; }

// Is the row wanted?  (Reused pixels' are not.)
__device__ __forceinline__ bool wanted(const dc_rows_args& a, int row)
{
    if (row >= (int)a.rows) return false;
    if (!a.masks) return true;
    const int q = q_row(a, row);
    return !((a.masks[q >> 5] >> (q & 31)) & 1u);
}

// Rows in registers: NV vectors of VE elements per lane.  A row belongs to `group` lanes of a warp, which takes 32 / group rows at once, or
// (BLOCK, its most threads) to the CTA.  Lanes beyond the row's end hold zeros (FULL: there are none).  The next rows' loads are in flight while
// a row is worked on, but for CTAs of 1024 threads, whose registers have no room for them.
template <typename T, int VE, int NV, int BLOCK, bool NORM, bool QUANT, bool FULL>
__global__ void __launch_bounds__(BLOCK ? BLOCK : 256, BLOCK ? 1 : VE == 1 ? (NV <= 8 ? 3 : 2) : NORM && VE == 8 && NV <= 2 ? 3 : 2) k_rows(const dc_rows_args a, int group)
{
    typedef Vec<T, VE> V;
    typedef typename V::F F;
    constexpr int P = V::P;
    constexpr bool AHEAD = BLOCK < 1024;
    __shared__ float red[BLOCK ? 6 * 32 : 1];
    const int lane = threadIdx.x & 31, sub = BLOCK ? threadIdx.x : lane & (group - 1), lanes = BLOCK ? blockDim.x : group;
    const int per_warp = BLOCK ? 1 : 32 / group, rows = (int)a.rows;
    const int first = BLOCK ? blockIdx.x : (blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5)) * per_warp;
    const int step = BLOCK ? gridDim.x : gridDim.x * (blockDim.x >> 5) * per_warp;
    const int nvec = a.channels / VE;
    const float c = (float)a.channels, inv_c = 1.f / c;
    // weights of few channels per lane stay in registers; others come from L1 for every row
    constexpr bool KEEP = NORM && NV * VE <= 16;
    F gk[KEEP ? NV : 1][P], bk[KEEP ? NV : 1][P];
    dc_pdl_wait();
    dc_pdl_release();
    if (KEEP)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int i = v * lanes + sub;
            if (FULL || i < nvec) { load_weights(a.gamma, i * VE, 1.f, gk[v]); load_weights(a.beta, i * VE, 0.f, bk[v]); }
        }
    typename V::Raw next[NV];
    bool next_live;
    constexpr int VB = VE * (int)sizeof(T);
    const int line = lanes * VB;
    // lanes beyond the row's end never load and keep their zeros; a row that is not there leaves the last one's values, and nothing of it is stored
#pragma unroll
    for (int v = 0; v < NV; ++v) next[v] = raw_zero<typename V::Raw>();
    auto fetch = [&](int r) {
        next_live = NORM ? r < rows : wanted(a, r);
        const char* const x = row_at(a.x, a.x_pitch, r) + sub * VB;
#pragma unroll
        for (int v = 0; v < NV; ++v)
            if (next_live && (FULL || v * lanes + sub < nvec)) next[v] = *(const typename V::Raw*)(x + v * line);
    };
    int row = BLOCK ? first : first + lane / group;
    if (AHEAD) fetch(row);
    int parity = 0;
    for (int base = first; base < rows; base += step, row += step, parity ^= 1) {
        float* const slot = red + (BLOCK ? parity * 96 : 0);
        F d[NV * P];
        uint32_t m = 0;
        if (!AHEAD) fetch(row);
        const bool on = next_live;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            V::open(next[v], d + v * P);
            if (QUANT && !NORM) m = raw_most(m, next[v]);
        }
        if (AHEAD) fetch(row + step);
        if (NORM) {
            F s = d[0];
#pragma unroll
            for (int k = 1; k < NV * P; ++k) s = add2(s, d[k]);
            const float mean = over(reduce<Sum, (BLOCK > 0)>(sum_of(s), group, slot), c, inv_c);
            const F minus = both<F>(-mean);
            s = both<F>(0.f);
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if (FULL || v * lanes + sub < nvec)
#pragma unroll
                    for (int k = v * P; k < v * P + P; ++k) { d[k] = add2(d[k], minus); s = fma2(d[k], d[k], s); }
            const float rstd = inverse_root(over(reduce<Sum, (BLOCK > 0)>(sum_of(s), group, slot + 32), c, inv_c) + a.eps);
            if (on && sub == 0) {
                if (a.mean) a.mean[(uint32_t)row] = mean;
                if (a.rstd) a.rstd[(uint32_t)row] = rstd;
            }
            char* const y = NORM ? row_at(a.y, a.y_pitch, row) + sub * VB : nullptr;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int i = v * lanes + sub;
                if (FULL || i < nvec) {
                    F g[P], b[P];
                    if (!KEEP) { load_weights(a.gamma, i * VE, 1.f, g); load_weights(a.beta, i * VE, 0.f, b); }
#pragma unroll
                    for (int k = 0; k < P; ++k) d[v * P + k] = fma2(mul2(d[v * P + k], both<F>(rstd)), KEEP ? gk[KEEP ? v : 0][k] : g[k], KEEP ? bk[KEEP ? v : 0][k] : b[k]);
                }
                const typename V::Raw r = V::close(d + v * P);
                if (on && a.y && (FULL || i < nvec)) *(typename V::Raw*)(y + v * line) = r;
                if (QUANT && sizeof(T) == 2) V::open(r, d + v * P);             // as the map holds it
                if (QUANT) m = raw_most(m, r);
            }
        }
        if (QUANT) {
            m = reduce<Most, (BLOCK > 0)>(most_of<T>(m), group, (uint32_t*)slot + 64);
            const RowScale s = row_scale(m);
            const int qr = q_row(a, row);
            if (on && sub == 0) a.scale[(uint32_t)qr] = s.scale;
            if (s.lift != 1.f)
#pragma unroll
                for (int k = 0; k < NV * P; ++k) d[k] = s.lift != 0.f ? mul2(d[k], both<F>(s.lift)) : both<F>(0.f);
            int8_t* const q = (int8_t*)row_at(a.q, a.q_pitch, qr) + sub * VE;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                uint32_t w[VE == 8 ? 2 : 1];
                quantise<T, VE>(d + v * P, s.inv, s.most, w);
                if (on && (FULL || v * lanes + sub < nvec)) store_q<VE>(q + v * lanes * VE, w);
            }
        }
    }
}

// Rows that do not fit the registers: a CTA per row, which it reads once for each thing that it has to know of it (from L2 then).
template <typename T, bool NORM, bool QUANT>
__global__ void __launch_bounds__(1024) k_rows_long(const dc_rows_args a)
{
    typedef Vec<T, 1> V;
    __shared__ float red[6 * 32];
    dc_pdl_wait();
    dc_pdl_release();
    int parity = 0;
    const float c = (float)a.channels, inv_c = 1.f / c;
    for (int row = blockIdx.x; row < (int)a.rows; row += gridDim.x, parity ^= 1) {
        if (QUANT && !NORM && !wanted(a, row)) continue;
        float* const slot = red + parity * 96;
        const T* const x = (const T*)row_at(a.x, a.x_pitch, row);
        T* const y = (T*)row_at(a.y, a.y_pitch, row);
        float mean = 0.f, rstd = 1.f;
        auto at = [&](int i) { float v; V::open(x[i], &v); return v; };
        auto value = [&](int i) -> T {                            // as the map holds it
            float v = at(i);
            if (NORM) v = fmaf((v - mean) * rstd, a.gamma ? dc_ld(a.gamma + i) : 1.f, a.beta ? dc_ld(a.beta + i) : 0.f);
            return V::close(&v);
        };
        if (NORM) {
            float s = 0.f;
            for (int i = threadIdx.x; i < a.channels; i += blockDim.x) s += at(i);
            mean = over(reduce<Sum, true>(s, 32, slot), c, inv_c);
            s = 0.f;
            for (int i = threadIdx.x; i < a.channels; i += blockDim.x) { const float d = at(i) - mean; s = fmaf(d, d, s); }
            rstd = inverse_root(over(reduce<Sum, true>(s, 32, slot + 32), c, inv_c) + a.eps);
            if (threadIdx.x == 0) {
                if (a.mean) a.mean[row] = mean;
                if (a.rstd) a.rstd[row] = rstd;
            }
        }
        RowScale s = {};
        const int qr = q_row(a, row);
        if (QUANT) {
            uint32_t m = 0;
            for (int i = threadIdx.x; i < a.channels; i += blockDim.x) { float v; V::open(value(i), &v); m = Most::of(m, size_bits(v)); }
            m = reduce<Most, true>(m, 32, (uint32_t*)slot + 64);
            s = row_scale(m);
            if (threadIdx.x == 0) a.scale[qr] = s.scale;
        }
#pragma unroll 1
        for (int i = threadIdx.x; i < a.channels; i += blockDim.x) {
            const T v = value(i);
            if (NORM && a.y) y[i] = v;
            if (QUANT) {
                float t;
                V::open(v, &t);
                t = s.lift != 0.f ? t * s.lift : 0.f;
                uint32_t w;
                quantise<T, 1>(&t, s.inv, s.most, &w);
                a.q[(size_t)qr * a.q_pitch + i] = (int8_t)w;
            }
        }
    }
}

struct dc_backward_args {
    const void* dy; size_t dy_pitch; const void* x; size_t x_pitch;
    const float *gamma, *mean, *rstd;
    int64_t rows; int channels;
    void* dx; size_t dx_pitch;          // or NULL
    float* partial;                     // [CTAs][2][channels], or NULL: no gradients of the weights
};

// Gradients.  A row belongs to `group` lanes of a warp, or (BLOCK) to `group` threads of whole warps, several such groups to a CTA.  They keep the same
// channels through all their rows and add up those channels' sums in registers; at the end a CTA joins its warps' or groups' sums in a fixed
// order and leaves them for k_join.
template <typename T, int VE, int NV, bool BLOCK, int THREADS, int CTAS, bool FULL>
__global__ void __launch_bounds__(THREADS, CTAS) k_norm_backward(const dc_backward_args a, int group)
{
    typedef Vec<T, VE> V;
    typedef typename V::F F;
    constexpr int P = V::P;
    extern __shared__ float join[];     // [warps or groups][2][channels]
    __shared__ float red[BLOCK ? 4 * 32 : 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, lanes = group;
    const int team = BLOCK ? threadIdx.x / group : warp, sub = BLOCK ? threadIdx.x - team * group : lane & (group - 1);
    const int per_team = BLOCK ? 1 : 32 / group, teams = BLOCK ? blockDim.x / group : blockDim.x >> 5;
    const int first = (blockIdx.x * teams + team) * per_team, step = gridDim.x * teams * per_team, rows = (int)a.rows;
    const int nvec = a.channels / VE;
    const float c = (float)a.channels, inv_c = 1.f / c;
    F g[NV][P], dg[NV * P], db[NV * P];
    dc_pdl_wait();
    dc_pdl_release();
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int i = v * lanes + sub;
#pragma unroll
        for (int k = 0; k < P; ++k) g[v][k] = dg[v * P + k] = db[v * P + k] = both<F>(0.f);
        if (i < nvec) load_weights(a.gamma, i * VE, 1.f, g[v]);
    }
    typename V::Raw next_x[NV], next_dy[NV];
    float next_mean, next_rstd;
    constexpr int VB = VE * (int)sizeof(T);
    const int line = lanes * VB;
    // as in k_rows: lanes beyond the row's end keep zeros, a row that is not there the last one's values
#pragma unroll
    for (int v = 0; v < NV; ++v) next_x[v] = next_dy[v] = raw_zero<typename V::Raw>();
    next_mean = next_rstd = 0.f;
    auto fetch = [&](int r) {
        const bool live = r < rows;
        const char *const x = row_at(a.x, a.x_pitch, r) + sub * VB, *const dy = row_at(a.dy, a.dy_pitch, r) + sub * VB;
        if (live) { next_mean = a.mean[(uint32_t)r]; next_rstd = a.rstd[(uint32_t)r]; }
#pragma unroll
        for (int v = 0; v < NV; ++v)
            if (live && (FULL || v * lanes + sub < nvec)) { next_x[v] = *(const typename V::Raw*)(x + v * line); next_dy[v] = *(const typename V::Raw*)(dy + v * line); }
    };
    int row = BLOCK ? first : first + lane / group;
    fetch(row);
    int parity = 0;
    for (int base = first; base < rows; base += step, row += step, parity ^= 1) {
        const bool on = row < rows;
        F xh[NV * P], d[NV * P];
        const float mean = next_mean, rstd = next_rstd;
#pragma unroll
        for (int v = 0; v < NV; ++v) { V::open(next_x[v], xh + v * P); V::open(next_dy[v], d + v * P); }
        fetch(row + step);
        F p1 = both<F>(0.f), p2 = p1;
#pragma unroll
        for (int v = 0; v < NV; ++v)
            if (FULL || v * lanes + sub < nvec)                    // lanes beyond the row's end: zeros, whatever the mean and the scale are
#pragma unroll
                for (int k = v * P; k < v * P + P; ++k) {
                    xh[k] = mul2(add2(xh[k], both<F>(-mean)), both<F>(rstd));
                    if (on) { dg[k] = fma2(d[k], xh[k], dg[k]); db[k] = add2(db[k], d[k]); }
                    d[k] = mul2(d[k], g[v][k - v * P]);
                    p1 = add2(p1, d[k]);
                    p2 = fma2(d[k], xh[k], p2);
                }
        if (!a.dx) continue;
        float s1 = sum_of(p1), s2 = sum_of(p2);
        if (BLOCK) {                    // both sums behind one barrier
            float* const slot = red + parity * 64;
            s1 = reduce_lanes<Sum>(s1, 32); s2 = reduce_lanes<Sum>(s2, 32);
            if (lane == 0) { slot[warp] = s1; slot[32 + warp] = s2; }
            asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(group) : "memory");
            const int warps = group >> 5, at = team * warps + lane;
            s1 = lane < warps ? slot[at] : 0.f; s2 = lane < warps ? slot[32 + at] : 0.f;
        }
        const int over_lanes = BLOCK ? 32 : group;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            if (o < over_lanes) { s1 += __shfl_xor_sync(0xffffffffu, s1, o); s2 += __shfl_xor_sync(0xffffffffu, s2, o); }
        s1 *= -inv_c; s2 *= -inv_c;
        char* const dx = row_at(a.dx, a.dx_pitch, row) + sub * VB;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
#pragma unroll
            for (int k = v * P; k < v * P + P; ++k) d[k] = mul2(fma2(xh[k], both<F>(s2), add2(d[k], both<F>(s1))), both<F>(rstd));
            if (on && (FULL || v * lanes + sub < nvec)) *(typename V::Raw*)(dx + v * line) = V::close(d + v * P);
        }
    }
    if (!a.partial) return;
    float* const out = a.partial + (size_t)blockIdx.x * 2 * a.channels;
    float* const mine = BLOCK && teams == 1 ? out : join + team * 2 * a.channels;
    if (!BLOCK)
        for (int o = group; o < 32; o <<= 1)                         // rows of one warp
#pragma unroll
            for (int k = 0; k < NV * P; ++k) { dg[k] = add_shuffled(dg[k], o); db[k] = add_shuffled(db[k], o); }
    if (BLOCK || lane < group)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int i = v * lanes + sub;
            if (i < nvec) {
                if constexpr (VE == 1) { mine[i] = dg[v]; mine[a.channels + i] = db[v]; }
                else
#pragma unroll
                    for (int k = 0; k < VE; k += 4) {
                        const int j = v * P + k / 2;
                        *(float4*)(mine + i * VE + k) = make_float4(dg[j].x, dg[j].y, dg[j + 1].x, dg[j + 1].y);
                        *(float4*)(mine + a.channels + i * VE + k) = make_float4(db[j].x, db[j].y, db[j + 1].x, db[j + 1].y);
                    }
            }
        }
    if (BLOCK && teams == 1) return;
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.channels; i += blockDim.x) {
        float s = 0.f;
        for (int t = 0; t < teams; ++t) s += join[t * 2 * a.channels + i];
        out[i] = s;
    }
}

// The CTAs' sums of 32 columns: 32 threads per column, each every 32nd CTA's, joined in a fixed order.
__global__ void __launch_bounds__(1024) k_join(const float* partial, int ctas, int channels, float* dgamma, float* dbeta)
{
    __shared__ float part[32][33];
    dc_pdl_wait();
    dc_pdl_release();
    const int lane = threadIdx.x & 31, turn = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (col < 2 * channels)
#pragma unroll 4
        for (int c = turn; c < ctas; c += 32) s += partial[(size_t)c * 2 * channels + col];
    part[turn][lane] = s;
    __syncthreads();
    s = reduce_lanes<Sum>(part[lane][turn], 32);
    const int mine = blockIdx.x * 32 + turn;
    if (lane == 0 && mine < 2 * channels) {
        if (mine < channels) { if (dgamma) dgamma[mine] = s; }
        else if (dbeta) dbeta[mine - channels] = s;
    }
}

bool aligned16(const void* p, size_t pitch) { return (uintptr_t)p % 16 == 0 && pitch % 16 == 0; }

// Lanes per row and vectors per lane for rows of nvec vectors: at most `most` per lane, as few idle places as possible, then as
// few lanes per row as possible (more rows of a warp in flight).  group 0: more than a warp holds.
struct Split { int group, nv; };
Split split_row(int nvec, int most)
{
    Split best = {0, 0};
    for (int g = 1; g <= 32; g <<= 1) {
        const int nv = dc_div_up(nvec, g);
        if (nv <= most && (best.group == 0 || g * nv < best.group * best.nv)) best = {g, nv};
    }
    return best;
}

template <typename T, int VE, int NV, int BLOCK, bool NORM, bool QUANT, bool FULL>
cudaError_t launch_rows_as(const dc_rows_args& a, int group, int threads, int64_t ctas, int num_sms, cudaStream_t stream)
{
    static int resident[33];            // CTAs of so many warps that an SM holds
    int& fit = resident[threads / 32];
    if (!fit) {
        int n = 0;
        const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, k_rows<T, VE, NV, BLOCK, NORM, QUANT, FULL>, threads, 0);
        if (e != cudaSuccess) return e;
        fit = n > 0 ? n : 1;
    }
    const int64_t cap = (int64_t)num_sms * fit;
    return dc_launch_pdl(k_rows<T, VE, NV, BLOCK, NORM, QUANT, FULL>, dim3((unsigned)(ctas < cap ? ctas : cap)), threads, 0, stream, a, group);
}

template <typename T, int VE, bool NORM, bool QUANT>
cudaError_t launch_rows(const dc_rows_args& a, int num_sms, cudaStream_t stream)
{
    const int nvec = a.channels / VE;
#define DC_ROWS(NV, BLOCK, G, THREADS, CTAS)                                                                                                       return nvec == (NV) * ((BLOCK) ? (THREADS) : (G)) ? launch_rows_as<T, VE, NV, BLOCK, NORM, QUANT, true>(a, G, THREADS, CTAS, num_sms, stream)                                                            : launch_rows_as<T, VE, NV, BLOCK, NORM, QUANT, false>(a, G, THREADS, CTAS, num_sms, stream)
    // few rows: a CTA for each, a vector per thread
    if (nvec > 32 && nvec <= 1024 && a.rows <= 2 * num_sms) DC_ROWS(1, 1024, 32, dc_div_up(nvec, 32) * 32, a.rows);
    // Normalised: 16 channels per lane, whose weights stay in its registers (56 x 56 x 256, 32 streams, bf16: 19.3 us, 22.3 with 32).
    Split s = split_row(nvec, VE == 1 ? 8 : NORM ? 16 / VE : 4);
    // Longer ones likewise, with a CTA to a row: 12000 x 2048 bf16 20.7 us, 26.5 with a warp; into 8 bits, with its third reduction, 12000 x 768 13.1 and
    // 11.0, 6000 x 1536 11.3 and 15.0.
    if constexpr (NORM && VE == 8)
        if (s.group == 0 && nvec > (QUANT ? 96 : 64) && nvec <= 1024) DC_ROWS(2, 512, 32, dc_div_up(dc_div_up(nvec, 2), 32) * 32, a.rows);
    if (s.group == 0) s = split_row(nvec, VE == 1 ? 16 : 4);
    if (s.group == 0 && nvec <= 32 * 8) s = {32, 8};
    if (s.group != 0) {
        const int64_t warps = (a.rows + 32 / s.group - 1) / (32 / s.group);
        const int per_cta = warps >= 8 * (int64_t)num_sms ? 8 : warps >= 4 * (int64_t)num_sms ? 4 : warps >= 2 * (int64_t)num_sms ? 2 : 1;
        const int64_t ctas = (warps + per_cta - 1) / per_cta;
        switch (s.nv) {
        case 1: DC_ROWS(1, 0, s.group, per_cta * 32, ctas);
        case 2: DC_ROWS(2, 0, s.group, per_cta * 32, ctas);
        case 3: DC_ROWS(3, 0, s.group, per_cta * 32, ctas);
        case 4: DC_ROWS(4, 0, s.group, per_cta * 32, ctas);
        case 5: case 6: case 7: case 8: DC_ROWS(8, 0, s.group, per_cta * 32, ctas);
        default:
            if constexpr (VE == 1) {
                if (s.nv <= 12) DC_ROWS(12, 0, s.group, per_cta * 32, ctas);
                DC_ROWS(16, 0, s.group, per_cta * 32, ctas);
            }
        }
    }
    if constexpr (VE == 1) if (nvec <= 512 * 12) DC_ROWS(12, 512, 32, dc_div_up(dc_div_up(nvec, 12), 32) * 32, a.rows);
    // a CTA per row: as many threads as leave each four vectors, up to 1024
    const int want = dc_div_up(dc_div_up(nvec, 4), 32) * 32, threads = want < 128 ? 128 : want > 1024 ? 1024 : want;
    if (threads <= 512) DC_ROWS(4, 512, 32, threads, a.rows);
    if (nvec <= 4096) DC_ROWS(4, 1024, 32, threads, a.rows);
    if constexpr (VE < 8) if (nvec <= 8192) DC_ROWS(8, 1024, 32, threads, a.rows);
#undef DC_ROWS
    return dc_launch_pdl(k_rows_long<T, NORM, QUANT>, dim3((unsigned)(a.rows < 2 * num_sms ? a.rows : 2 * num_sms)), 1024, 0, stream, a);
}

template <typename T, int VE>
cudaError_t launch_rows_kind(const dc_rows_args& a, bool norm, int num_sms, cudaStream_t stream)
{
    if (!norm) return launch_rows<T, VE, false, true>(a, num_sms, stream);
    return a.q ? launch_rows<T, VE, true, true>(a, num_sms, stream) : launch_rows<T, VE, true, false>(a, num_sms, stream);
}

template <typename T, int VE, int NV, bool BLOCK, int THREADS, int CTAS, bool FULL>
cudaError_t launch_backward_as(const dc_backward_args& a, int group, int num_sms, cudaStream_t stream, int* ctas)
{
    const int teams = BLOCK ? (THREADS / group > 1 ? THREADS / group : 1) : THREADS / 32, threads = BLOCK ? teams * group : THREADS;
    const size_t smem = BLOCK && teams == 1 ? 0 : (size_t)teams * 2 * a.channels * sizeof(float);
    const int64_t per_cta = (int64_t)teams * (BLOCK ? 1 : 32 / group), want = (a.rows + per_cta - 1) / per_cta;
    const int most = CTAS * num_sms < kBackwardCtas ? CTAS * num_sms : kBackwardCtas;          // as many as are resident
    *ctas = (int)(want < 1 ? 1 : want < most ? want : most);
    return dc_launch_pdl(k_norm_backward<T, VE, NV, BLOCK, THREADS, CTAS, FULL>, dim3((unsigned)*ctas), threads, smem, stream, a, group);
}

// Rows of up to 512 channels belong to a warp's lanes, with 8 or 16 channels each: 16 of bfloat16, whose raw values ahead take half the registers
// (56 x 56 x 256, 32 streams: 32.6 us, 37.0 with 8), 8 of float32 (50000 x 128: 17.4 us, 19.8 with 16).  Longer rows belong to teams of warps.
template <typename T, int VE>
cudaError_t launch_backward(const dc_backward_args& a, int num_sms, cudaStream_t stream, int* ctas)
{
    const int nvec = a.channels / VE;
    constexpr int N8 = 8 / VE, N16 = 16 / VE, T16 = VE == 8 ? 256 : 384, C16 = VE == 8 ? 2 : 1;
    Split s = split_row(nvec, VE == 8 ? N16 : N8);
    if (s.group == 0) s = split_row(nvec, N16);
    if (s.group != 0) {
        const bool full = nvec == s.group * s.nv;
        if (s.nv <= N8) {
            if (full && s.nv == N8) return launch_backward_as<T, VE, N8, false, 320, 2, true>(a, s.group, num_sms, stream, ctas);
            return launch_backward_as<T, VE, N8, false, 320, 2, false>(a, s.group, num_sms, stream, ctas);
        }
        if constexpr (VE == 1) if (s.nv <= 12) return launch_backward_as<T, VE, 12, false, 256, 2, false>(a, s.group, num_sms, stream, ctas);
        if (full && s.nv == N16) return launch_backward_as<T, VE, N16, false, T16, C16, true>(a, s.group, num_sms, stream, ctas);
        return launch_backward_as<T, VE, N16, false, T16, C16, false>(a, s.group, num_sms, stream, ctas);
    }
    const int want = dc_div_up(dc_div_up(nvec, N8), 32) * 32;
    if (want <= 512) {
        if (want * N8 == nvec) return launch_backward_as<T, VE, N8, true, 512, 1, true>(a, want, num_sms, stream, ctas);
        return launch_backward_as<T, VE, N8, true, 512, 1, false>(a, want, num_sms, stream, ctas);
    }
    if (want <= 1024) return launch_backward_as<T, VE, N8, true, 1024, 1, false>(a, want, num_sms, stream, ctas);
    return launch_backward_as<T, VE, N16, true, 1024, 1, false>(a, dc_div_up(dc_div_up(nvec, N16), 32) * 32, num_sms, stream, ctas);
}

constexpr int kMostNormChannels = 16384;
constexpr int64_t kMostRows = DC_MOST_ROWS;

}  // namespace

int dc_current_device(int* device, int* num_sms)
{
    static int sms[64];
    DC_CUDA(cudaGetDevice(device));
    if (*device < 0 || *device >= 64) { DC_CUDA(cudaDeviceGetAttribute(num_sms, cudaDevAttrMultiProcessorCount, *device)); return DC_OK; }
    if (!sms[*device]) DC_CUDA(cudaDeviceGetAttribute(&sms[*device], cudaDevAttrMultiProcessorCount, *device));
    *num_sms = sms[*device];
    return DC_OK;
}

int dc_launch_rows(const dc_rows_args& a, bool norm, int dtype, int num_sms, cudaStream_t stream)
{
    if (a.rows <= 0) return DC_OK;
    const int elt = dtype == DC_BF16 ? 2 : 4;
    const bool vec = aligned16(a.x, a.x_pitch) && (!a.y || aligned16(a.y, a.y_pitch)) && (a.channels * (size_t)elt) % 16 == 0 &&
                     (uintptr_t)a.gamma % 16 == 0 && (uintptr_t)a.beta % 16 == 0;
    if (dtype == DC_BF16) DC_CUDA(vec ? (launch_rows_kind<__nv_bfloat16, 8>(a, norm, num_sms, stream)) : (launch_rows_kind<__nv_bfloat16, 1>(a, norm, num_sms, stream)));
    else DC_CUDA(vec ? (launch_rows_kind<float, 4>(a, norm, num_sms, stream)) : (launch_rows_kind<float, 1>(a, norm, num_sms, stream)));
    return DC_OK;
}

// What every entry point asks of rows of a map.
static bool rows_within(size_t a, size_t b, size_t c, int64_t rows) { return rows <= kMostRows && (rows < 2 || (a | b | c) <= 0xffffffffu); }
static bool rows_ok(const void* p, size_t pitch, int64_t rows, int64_t columns, int elt)
{
    return p && (uintptr_t)p % elt == 0 && pitch % elt == 0 && (rows < 2 || pitch >= (size_t)columns * elt);
}
static bool floats_ok(const float* p) { return (uintptr_t)p % sizeof(float) == 0; }
static bool quant_ok(const int8_t* q, size_t pitch, const float* scale, int64_t rows, int64_t columns)
{
    return q && scale && floats_ok(scale) && (uintptr_t)q % 16 == 0 && pitch % 16 == 0 && (rows < 2 || pitch >= (size_t)columns);
}

static int norm_call(const void* x, size_t x_pitch, const float* gamma, const float* beta, int64_t rows, int32_t channels, double eps, int32_t dtype, void* y, size_t y_pitch,
                     float* mean, float* rstd, int8_t* q, size_t q_pitch, float* scale, bool want_y, bool want_q, void* stream)
{
    if (dtype != DC_FP32 && dtype != DC_BF16) return DC_ERR_CONFIG;
    const int elt = dtype == DC_BF16 ? 2 : 4;
    if (rows < 0 || channels < 1 || !(eps >= 0.0) || !(eps < 1e30)) return DC_ERR_ARG;
    if (channels > kMostNormChannels || !rows_within(x_pitch, y ? y_pitch : 0, want_q ? q_pitch : 0, rows)) return DC_ERR_LIMIT;
    if (!floats_ok(gamma) || !floats_ok(beta) || !floats_ok(mean) || !floats_ok(rstd)) return DC_ERR_ARG;
    if (rows == 0) return DC_OK;
    if (!rows_ok(x, x_pitch, rows, channels, elt) || ((want_y || y) && !rows_ok(y, y_pitch, rows, channels, elt))) return DC_ERR_ARG;
    if (want_q && !quant_ok(q, q_pitch, scale, rows, channels)) return DC_ERR_ARG;
    dc_rows_args a = {};
    a.x = x; a.x_pitch = x_pitch; a.gamma = gamma; a.beta = beta; a.rows = rows; a.channels = channels; a.eps = (float)eps;
    a.y = y; a.y_pitch = y_pitch; a.mean = mean; a.rstd = rstd; a.q = q; a.q_pitch = q_pitch; a.scale = scale;
    int device = 0, sms = 0;
    const int rc = dc_current_device(&device, &sms);
    return rc != DC_OK ? rc : dc_launch_rows(a, true, dtype, sms, (cudaStream_t)stream);
}

extern "C" {

int dc_layer_norm(const void* x_dev, size_t x_pitch, const float* gamma_dev, const float* beta_dev, int64_t rows, int32_t channels, double eps, int32_t dtype,
                  void* y_dev, size_t y_pitch, float* mean_dev, float* rstd_dev, void* cuda_stream)
{
    return norm_call(x_dev, x_pitch, gamma_dev, beta_dev, rows, channels, eps, dtype, y_dev, y_pitch, mean_dev, rstd_dev, nullptr, 0, nullptr, true, false, cuda_stream);
}

int dc_layer_norm_quantize(const void* x_dev, size_t x_pitch, const float* gamma_dev, const float* beta_dev, int64_t rows, int32_t channels, double eps, int32_t dtype,
                           void* y_dev, size_t y_pitch, int8_t* q_dev, size_t q_pitch, float* scale_dev, void* cuda_stream)
{
    return norm_call(x_dev, x_pitch, gamma_dev, beta_dev, rows, channels, eps, dtype, y_dev, y_pitch, nullptr, nullptr, q_dev, q_pitch, scale_dev, false, true, cuda_stream);
}

int dc_quantize_rows(const void* x_dev, size_t x_pitch, int64_t rows, int32_t channels, int32_t dtype, int8_t* q_dev, size_t q_pitch, float* scale_dev, void* cuda_stream)
{
    if (dtype != DC_FP32 && dtype != DC_BF16) return DC_ERR_CONFIG;
    if (rows < 0 || channels < 1) return DC_ERR_ARG;
    if (!rows_within(x_pitch, q_pitch, 0, rows)) return DC_ERR_LIMIT;
    if (rows == 0) return DC_OK;
    if (!rows_ok(x_dev, x_pitch, rows, channels, dtype == DC_BF16 ? 2 : 4) || !quant_ok(q_dev, q_pitch, scale_dev, rows, channels)) return DC_ERR_ARG;
    dc_rows_args a = {};
    a.x = x_dev; a.x_pitch = x_pitch; a.rows = rows; a.channels = channels; a.q = q_dev; a.q_pitch = q_pitch; a.scale = scale_dev;
    int device = 0, sms = 0;
    const int rc = dc_current_device(&device, &sms);
    return rc != DC_OK ? rc : dc_launch_rows(a, false, dtype, sms, (cudaStream_t)cuda_stream);
}

int dc_layer_norm_workspace(int32_t channels, size_t* bytes)
{
    if (channels < 1 || !bytes) return DC_ERR_ARG;
    *bytes = (size_t)kBackwardCtas * 2 * sizeof(float) * (size_t)channels;
    return DC_OK;
}

int dc_layer_norm_backward(const void* dy_dev, size_t dy_pitch, const void* x_dev, size_t x_pitch, const float* gamma_dev, const float* mean_dev, const float* rstd_dev,
                           int64_t rows, int32_t channels, int32_t dtype, void* dx_dev, size_t dx_pitch, float* dgamma_dev, float* dbeta_dev,
                           void* workspace_dev, size_t workspace_bytes, void* cuda_stream)
{
    if (dtype != DC_FP32 && dtype != DC_BF16) return DC_ERR_CONFIG;
    const int elt = dtype == DC_BF16 ? 2 : 4;
    if (rows < 0 || channels < 1) return DC_ERR_ARG;
    if (channels > kMostNormChannels || !rows_within(dy_pitch, x_pitch, dx_dev ? dx_pitch : 0, rows)) return DC_ERR_LIMIT;
    if (!floats_ok(gamma_dev) || !floats_ok(mean_dev) || !floats_ok(rstd_dev) || !floats_ok(dgamma_dev) || !floats_ok(dbeta_dev)) return DC_ERR_ARG;
    const bool weights = dgamma_dev || dbeta_dev;
    size_t need = 0;
    dc_layer_norm_workspace(channels, &need);
    if (weights && (!workspace_dev || (uintptr_t)workspace_dev % 16 || workspace_bytes < need)) return DC_ERR_ARG;
    if (rows == 0) {                    // sums of nothing
        if (dgamma_dev) DC_CUDA(cudaMemsetAsync(dgamma_dev, 0, sizeof(float) * channels, (cudaStream_t)cuda_stream));
        if (dbeta_dev) DC_CUDA(cudaMemsetAsync(dbeta_dev, 0, sizeof(float) * channels, (cudaStream_t)cuda_stream));
        return DC_OK;
    }
    if (!mean_dev || !rstd_dev || !rows_ok(dy_dev, dy_pitch, rows, channels, elt) || !rows_ok(x_dev, x_pitch, rows, channels, elt)) return DC_ERR_ARG;
    if (dx_dev && !rows_ok(dx_dev, dx_pitch, rows, channels, elt)) return DC_ERR_ARG;
    if (!dx_dev && !weights) return DC_OK;
    dc_backward_args a = {dy_dev, dy_pitch, x_dev, x_pitch, gamma_dev, mean_dev, rstd_dev, rows, channels, dx_dev, dx_pitch, weights ? (float*)workspace_dev : nullptr};
    int device = 0, sms = 0, ctas = 0;
    const int rc = dc_current_device(&device, &sms);
    if (rc != DC_OK) return rc;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    const bool vec = aligned16(x_dev, x_pitch) && aligned16(dy_dev, dy_pitch) && (!dx_dev || aligned16(dx_dev, dx_pitch)) && ((size_t)channels * elt) % 16 == 0 &&
                     (uintptr_t)gamma_dev % 16 == 0;
    if (dtype == DC_BF16) DC_CUDA(vec ? (launch_backward<__nv_bfloat16, 8>(a, sms, stream, &ctas)) : (launch_backward<__nv_bfloat16, 1>(a, sms, stream, &ctas)));
    else DC_CUDA(vec ? (launch_backward<float, 4>(a, sms, stream, &ctas)) : (launch_backward<float, 1>(a, sms, stream, &ctas)));
    if (weights)
        DC_CUDA(dc_launch_pdl(k_join, dim3((unsigned)dc_div_up(2 * channels, 32)), 1024, 0, stream, (const float*)workspace_dev, ctas, (int)channels, dgamma_dev, dbeta_dev));
    return DC_OK;
}

}  // extern "C"
