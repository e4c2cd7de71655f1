// Device-side building blocks of the kernels on rows of channels (dc_norm.cu, dc_few.cu): vectors of a row as floats, reductions among the threads
// that share a row, and a row's values in 8 bits.
#pragma once
#include <string.h>

#include "dc_rows.cuh"

namespace {

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
// A product that is rounded whatever follows it.  The compiler may join a * b with an addition, and where gamma is absent, and so 1, fmaf(a * b, 1, beta) is one: a
// row's values would have other bits in one kernel than in another.
__device__ __forceinline__ float rounded(float a, float b) { return __fmul_rn(a, b); }
__device__ __forceinline__ float2 rounded(float2 a, float2 b) { return mul2(a, b); }
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
// The larger of m and the bits of a vector's sizes: two bfloat16 side by side, which most_of() joins.  One instruction for two elements; the
// sign that it leaves is cut off at the end, and a NaN stays one.  (With a mask and an integer maximum: 13.4 us, not 13.1, for 25088 rows of 512.)
__device__ __forceinline__ uint32_t larger2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t raw_most(uint32_t m, uint4 t) { return larger2(larger2(larger2(larger2(m, t.x), t.y), t.z), t.w) & 0x7fff7fffu; }
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

// s / c by the reciprocal of c and one correction by the remainder, which a fused multiply-add has exactly (Markstein 1990): half a step, as the division, at a
// third of its instructions.  (An infinite s gives NaN.)
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

}  // namespace
