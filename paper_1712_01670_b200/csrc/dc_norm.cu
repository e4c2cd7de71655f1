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
#include "dc_rows.cuh"

namespace {

constexpr int kBackwardCtas = 296;      // partial sums of a gradient's columns: two CTAs for each SM of a B200

// VE elements of a row as floats: 16 bytes at once, or one element where alignment or the row's length do not allow that.
template <typename T, int VE> struct Vec;
template <> struct Vec<float, 4> {
    static __device__ __forceinline__ void load(const float* p, float* v) { const float4 t = *(const float4*)p; v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w; }
    static __device__ __forceinline__ void store(float* p, const float* v) { *(float4*)p = make_float4(v[0], v[1], v[2], v[3]); }
};
template <> struct Vec<__nv_bfloat16, 8> {
    static __device__ __forceinline__ void load(const __nv_bfloat16* p, float* v)
    {
        const uint4 t = *(const uint4*)p;
        const uint32_t w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) { v[2 * k] = __uint_as_float(w[k] << 16); v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u); }
    }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float* v)
    {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) { const __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]); w[k] = *(const uint32_t*)&t; }
        *(uint4*)p = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <> struct Vec<float, 1> {
    static __device__ __forceinline__ void load(const float* p, float* v) { v[0] = *p; }
    static __device__ __forceinline__ void store(float* p, const float* v) { *p = v[0]; }
};
template <> struct Vec<__nv_bfloat16, 1> {
    static __device__ __forceinline__ void load(const __nv_bfloat16* p, float* v) { v[0] = __bfloat162float(*p); }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float* v) { *p = __float2bfloat16_rn(v[0]); }
};
template <typename T> __device__ __forceinline__ float as_stored(float v);
template <> __device__ __forceinline__ float as_stored<float>(float v) { return v; }
template <> __device__ __forceinline__ float as_stored<__nv_bfloat16>(float v) { return __bfloat162float(__float2bfloat16_rn(v)); }

// VE channel weights; p NULL: `fill`.
template <int VE>
__device__ __forceinline__ void load_weights(const float* p, int at, float fill, float* v)
{
    if (p) {
        if constexpr (VE == 1) v[0] = __ldg(p + at);
        else
#pragma unroll
            for (int k = 0; k < VE; k += 4) {
                const float4 t = __ldg((const float4*)(p + at + k));
                v[k] = t.x; v[k + 1] = t.y; v[k + 2] = t.z; v[k + 3] = t.w;
            }
    } else {
#pragma unroll
        for (int k = 0; k < VE; ++k) v[k] = fill;
    }
}

struct Sum { static __device__ __forceinline__ float of(float a, float b) { return a + b; } };
struct Most { static __device__ __forceinline__ uint32_t of(uint32_t a, uint32_t b) { return a > b ? a : b; } };

// Over the lanes of a group (a power of two), or over the CTA: each reduction of a row has a slot of its own, and rows alternate between two
// sets of them, so one barrier per reduction is enough.
template <typename Op, typename V>
__device__ __forceinline__ V reduce_lanes(V v, int group)
{
    for (int o = group >> 1; o > 0; o >>= 1) v = Op::of(v, __shfl_xor_sync(0xffffffffu, v, o));
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

// One value of a row in 127 steps of the row's largest, `most` > 0, either way; exact: the real quotient 127 x / most, halves to even.
// x * inv is off by less than 3 * 2^-24 of itself, so below 2^-15 absolutely: only next to a half is the quotient looked at again,
// in products that 64 bits hold exactly.
__device__ __noinline__ int quantise_next_to_half(float x, float r, float most)
{
    const float f = floorf(fabsf(r));
    const double d = 127.0 * fabs((double)x) - ((double)f + 0.5) * (double)most;
    int n = (int)f;
    if (d > 0.0 || (d == 0.0 && (n & 1))) ++n;
    return x < 0.f ? -n : n;
}
constexpr float kRound = 12582912.f;    // 1.5 * 2^23: adding it leaves the nearest integer in the low bits
template <int VE>
__device__ __forceinline__ void quantise(const float* x, float inv, float most, uint32_t* q)
{
    uint32_t b[VE];
    float far = 0.f;
#pragma unroll
    for (int k = 0; k < VE; ++k) {
        const float r = x[k] * inv, t = r + kRound;
        far = fmaxf(far, fabsf(r - (t - kRound)));
        b[k] = __float_as_uint(t);
    }
    if (far > 0.5f - 0x1p-14f) {
#pragma unroll
        for (int k = 0; k < VE; ++k) {
            const float r = x[k] * inv, t = r + kRound;
            if (fabsf(r - (t - kRound)) > 0.5f - 0x1p-14f) b[k] = (uint32_t)quantise_next_to_half(x[k], r, most);
        }
    }
    if constexpr (VE == 1) q[0] = b[0];
    else
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
// What a row's largest bits say of it: its scale, its steps' inverse, and a power of two that lifts rows of the smallest numbers first (their
// inverse would be infinite).  A row with an infinity or a NaN gets the scale NaN and zeros.
struct RowScale { float scale, inv, most, lift; };
__device__ __forceinline__ RowScale row_scale(uint32_t bits)
{
    RowScale s;
    s.most = __uint_as_float(bits);
    s.lift = 1.f;
    s.scale = s.most / 127.f;
    if (bits < 0x21800000u) { s.lift = 0x1p64f; s.most *= s.lift; }              // below 2^-60
    s.inv = s.most > 0.f ? 127.f / s.most : 0.f;
    if (bits >= 0x7f800000u) { s.scale = __uint_as_float(0x7fffffffu); s.inv = 0.f; s.lift = 0.f; s.most = 1.f; }
    return s;
}

// A row's place in q and scale: see dc_rows_args.
__device__ __forceinline__ int64_t q_row(const dc_rows_args& a, int64_t row)
{
    if (a.padded == 0) return row;
    const int64_t line = row / a.width;
    return line * a.padded + (row - line * a.width);
}

// Rows in registers: NV vectors of VE elements per lane.  A row belongs to `group` lanes of a warp, which takes 32 / group rows at once, or
// (BLOCK) to the CTA.  Lanes beyond the row's end hold zeros.
template <typename T, int VE, int NV, bool BLOCK, bool NORM, bool QUANT>
__global__ void __launch_bounds__(BLOCK ? 1024 : 256) k_rows(const dc_rows_args a, int group)
{
    __shared__ float red[BLOCK ? 6 * 32 : 1];
    const int lane = threadIdx.x & 31, sub = BLOCK ? threadIdx.x : lane & (group - 1), lanes = BLOCK ? blockDim.x : group;
    const int per_warp = BLOCK ? 1 : 32 / group;
    const int64_t first = BLOCK ? blockIdx.x : ((int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5)) * per_warp;
    const int64_t step = BLOCK ? gridDim.x : (int64_t)gridDim.x * (blockDim.x >> 5) * per_warp;
    const int nvec = a.channels / VE;
    const float c = (float)a.channels;
    // weights of few channels per lane stay in registers; others come from L1 for every row
    constexpr bool KEEP = NORM && NV * VE <= 16;
    float gk[KEEP ? NV * VE : 1], bk[KEEP ? NV * VE : 1];
    if (KEEP)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int i = v * lanes + sub;
            if (i < nvec) { load_weights<VE>(a.gamma, i * VE, 1.f, gk + v * VE); load_weights<VE>(a.beta, i * VE, 0.f, bk + v * VE); }
        }
    dc_pdl_wait();
    dc_pdl_release();
    int parity = 0;
    for (int64_t base = first; base < a.rows; base += step, parity ^= 1) {
        const int64_t row = BLOCK ? base : base + lane / group;
        const bool on = row < a.rows;
        float* const slot = red + (BLOCK ? parity * 96 : 0);
        const T* const x = (const T*)((const char*)a.x + (size_t)row * a.x_pitch);
        float d[NV * VE];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int i = v * lanes + sub;
            if (on && i < nvec) Vec<T, VE>::load(x + i * VE, d + v * VE);
            else
#pragma unroll
                for (int k = 0; k < VE; ++k) d[v * VE + k] = 0.f;
        }
        if (NORM) {
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < NV * VE; ++k) s += d[k];
            const float mean = reduce<Sum, BLOCK>(s, group, slot) / c;
            s = 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if (v * lanes + sub < nvec)
#pragma unroll
                    for (int k = 0; k < VE; ++k) { d[v * VE + k] -= mean; s += d[v * VE + k] * d[v * VE + k]; }
            const float rstd = 1.f / sqrtf(reduce<Sum, BLOCK>(s, group, slot + 32) / c + a.eps);
            if (on && sub == 0) {
                if (a.mean) a.mean[row] = mean;
                if (a.rstd) a.rstd[row] = rstd;
            }
            T* const y = (T*)((char*)a.y + (size_t)row * a.y_pitch);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int i = v * lanes + sub;
                if (i >= nvec) continue;
                float g[VE], b[VE];
                if (!KEEP) { load_weights<VE>(a.gamma, i * VE, 1.f, g); load_weights<VE>(a.beta, i * VE, 0.f, b); }
#pragma unroll
                for (int k = 0; k < VE; ++k) d[v * VE + k] = fmaf(d[v * VE + k] * rstd, KEEP ? gk[(v * VE + k) % (NV * VE)] : g[k], KEEP ? bk[v * VE + k] : b[k]);
                if (on && a.y) Vec<T, VE>::store(y + i * VE, d + v * VE);
                if (QUANT)
#pragma unroll
                    for (int k = 0; k < VE; ++k) d[v * VE + k] = as_stored<T>(d[v * VE + k]);
            }
        }
        if (QUANT) {
            uint32_t m = 0;
#pragma unroll
            for (int k = 0; k < NV * VE; ++k) m = Most::of(m, __float_as_uint(d[k]) & 0x7fffffffu);
            m = reduce<Most, BLOCK>(m, group, (uint32_t*)slot + 64);
            const RowScale s = row_scale(m);
            const int64_t qr = q_row(a, row);
            if (on && sub == 0) a.scale[qr] = s.scale;
            if (s.lift != 1.f)
#pragma unroll
                for (int k = 0; k < NV * VE; ++k) d[k] = s.lift != 0.f ? d[k] * s.lift : 0.f;
            int8_t* const q = a.q + (size_t)qr * a.q_pitch;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int i = v * lanes + sub;
                uint32_t w[VE == 8 ? 2 : 1];
                quantise<VE>(d + v * VE, s.inv, s.most, w);
                if (on && i < nvec) store_q<VE>(q + i * VE, w);
            }
        }
    }
}

// Rows that do not fit the registers: a CTA per row, which it reads once for each thing that it has to know of it (from L2 then).
template <typename T, bool NORM, bool QUANT>
__global__ void __launch_bounds__(1024) k_rows_long(const dc_rows_args a)
{
    __shared__ float red[6 * 32];
    dc_pdl_wait();
    dc_pdl_release();
    int parity = 0;
    const float c = (float)a.channels;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, parity ^= 1) {
        float* const slot = red + parity * 96;
        const T* const x = (const T*)((const char*)a.x + (size_t)row * a.x_pitch);
        T* const y = (T*)((char*)a.y + (size_t)row * a.y_pitch);
        float mean = 0.f, rstd = 1.f;
        auto value = [&](int i) {
            float v;
            Vec<T, 1>::load(x + i, &v);
            if (!NORM) return v;
            return fmaf((v - mean) * rstd, a.gamma ? __ldg(a.gamma + i) : 1.f, a.beta ? __ldg(a.beta + i) : 0.f);
        };
        if (NORM) {
            float s = 0.f, v;
            for (int i = threadIdx.x; i < a.channels; i += blockDim.x) { Vec<T, 1>::load(x + i, &v); s += v; }
            mean = reduce<Sum, true>(s, 32, slot) / c;
            s = 0.f;
            for (int i = threadIdx.x; i < a.channels; i += blockDim.x) { Vec<T, 1>::load(x + i, &v); s += (v - mean) * (v - mean); }
            rstd = 1.f / sqrtf(reduce<Sum, true>(s, 32, slot + 32) / c + a.eps);
            if (threadIdx.x == 0) {
                if (a.mean) a.mean[row] = mean;
                if (a.rstd) a.rstd[row] = rstd;
            }
        }
        RowScale s = {};
        const int64_t qr = q_row(a, row);
        if (QUANT) {
            uint32_t m = 0;
            for (int i = threadIdx.x; i < a.channels; i += blockDim.x) m = Most::of(m, __float_as_uint(as_stored<T>(value(i))) & 0x7fffffffu);
            m = reduce<Most, true>(m, 32, (uint32_t*)slot + 64);
            s = row_scale(m);
            if (threadIdx.x == 0) a.scale[qr] = s.scale;
        }
        for (int i = threadIdx.x; i < a.channels; i += blockDim.x) {
            const float v = value(i);
            if (NORM && a.y) Vec<T, 1>::store(y + i, &v);
            if (QUANT) {
                const float t = s.lift != 0.f ? as_stored<T>(v) * s.lift : 0.f;
                uint32_t w;
                quantise<1>(&t, s.inv, s.most, &w);
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

// Gradients.  The lanes of a group (or the CTA) keep the same channels through all their rows and add up those channels' sums in registers; at the
// end a CTA joins its groups' sums in a fixed order and leaves them for k_join.
template <typename T, int VE, int NV, bool BLOCK, int THREADS>
__global__ void __launch_bounds__(THREADS) k_norm_backward(const dc_backward_args a, int group)
{
    extern __shared__ float join[];     // [2][channels] (not BLOCK)
    __shared__ float red[BLOCK ? 4 * 32 : 1];
    const int lane = threadIdx.x & 31, sub = BLOCK ? threadIdx.x : lane & (group - 1), lanes = BLOCK ? blockDim.x : group;
    const int per_warp = BLOCK ? 1 : 32 / group;
    const int64_t first = BLOCK ? blockIdx.x : ((int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5)) * per_warp;
    const int64_t step = BLOCK ? gridDim.x : (int64_t)gridDim.x * (blockDim.x >> 5) * per_warp;
    const int nvec = a.channels / VE;
    const float c = (float)a.channels;
    float g[NV * VE], dg[NV * VE], db[NV * VE];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int i = v * lanes + sub;
#pragma unroll
        for (int k = 0; k < VE; ++k) { g[v * VE + k] = 0.f; dg[v * VE + k] = 0.f; db[v * VE + k] = 0.f; }
        if (i < nvec) load_weights<VE>(a.gamma, i * VE, 1.f, g + v * VE);
    }
    dc_pdl_wait();
    dc_pdl_release();
    int parity = 0;
    for (int64_t base = first; base < a.rows; base += step, parity ^= 1) {
        const int64_t row = BLOCK ? base : base + lane / group;
        const bool on = row < a.rows;
        const T* const x = (const T*)((const char*)a.x + (size_t)row * a.x_pitch);
        const T* const dy = (const T*)((const char*)a.dy + (size_t)row * a.dy_pitch);
        float xh[NV * VE], d[NV * VE];
        const float mean = on ? a.mean[row] : 0.f, rstd = on ? a.rstd[row] : 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int i = v * lanes + sub;
            if (on && i < nvec) { Vec<T, VE>::load(x + i * VE, xh + v * VE); Vec<T, VE>::load(dy + i * VE, d + v * VE); }
            else
#pragma unroll
                for (int k = 0; k < VE; ++k) { xh[v * VE + k] = mean; d[v * VE + k] = 0.f; }
        }
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < NV * VE; ++k) {
            xh[k] = (xh[k] - mean) * rstd;
            dg[k] = fmaf(d[k], xh[k], dg[k]);
            db[k] += d[k];
            d[k] *= g[k];
            s1 += d[k];
            s2 = fmaf(d[k], xh[k], s2);
        }
        if (!a.dx) continue;
        float* const slot = red + (BLOCK ? parity * 64 : 0);
        if (BLOCK) {                    // both sums behind one barrier
            s1 = reduce_lanes<Sum>(s1, 32); s2 = reduce_lanes<Sum>(s2, 32);
            if (lane == 0) { slot[threadIdx.x >> 5] = s1; slot[32 + (threadIdx.x >> 5)] = s2; }
            __syncthreads();
            const int warps = blockDim.x >> 5;
            s1 = lane < warps ? slot[lane] : 0.f; s2 = lane < warps ? slot[32 + lane] : 0.f;
        }
        s1 = reduce_lanes<Sum>(s1, BLOCK ? 32 : group) / c;
        s2 = reduce_lanes<Sum>(s2, BLOCK ? 32 : group) / c;
        T* const dx = (T*)((char*)a.dx + (size_t)row * a.dx_pitch);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int i = v * lanes + sub;
#pragma unroll
            for (int k = 0; k < VE; ++k) d[v * VE + k] = (d[v * VE + k] - s1 - xh[v * VE + k] * s2) * rstd;
            if (on && i < nvec) Vec<T, VE>::store(dx + i * VE, d + v * VE);
        }
    }
    if (!a.partial) return;
    float* const out = a.partial + (size_t)blockIdx.x * 2 * a.channels;
    if constexpr (BLOCK) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int i = v * lanes + sub;
            if (i < nvec)
#pragma unroll
                for (int k = 0; k < VE; ++k) { out[i * VE + k] = dg[v * VE + k]; out[a.channels + i * VE + k] = db[v * VE + k]; }
        }
    } else {
    for (int o = group; o < 32; o <<= 1)                         // rows of one warp
#pragma unroll
        for (int k = 0; k < NV * VE; ++k) {
            dg[k] += __shfl_xor_sync(0xffffffffu, dg[k], o);
            db[k] += __shfl_xor_sync(0xffffffffu, db[k], o);
        }
    for (int w = 0; w < (int)(blockDim.x >> 5); ++w) {           // warp after warp
        if ((int)(threadIdx.x >> 5) == w && lane < group) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int i = v * lanes + sub;
                if (i < nvec)
#pragma unroll
                    for (int k = 0; k < VE; ++k) {
                        float* const p = join + i * VE + k;
                        p[0] = w ? p[0] + dg[v * VE + k] : dg[v * VE + k];
                        p[a.channels] = w ? p[a.channels] + db[v * VE + k] : db[v * VE + k];
                    }
            }
        }
        __syncthreads();
    }
    for (int i = threadIdx.x; i < 2 * a.channels; i += blockDim.x) out[i] = join[i];
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

template <typename T, int VE, bool NORM, bool QUANT>
cudaError_t launch_rows(const dc_rows_args& a, int num_sms, cudaStream_t stream)
{
    const int nvec = a.channels / VE;
    Split s = split_row(nvec, 4);
    if (s.group == 0 && nvec <= 32 * 8) s = {32, 8};
    if (s.group != 0) {
        const int64_t per_cta = (int64_t)8 * (32 / s.group), want = (a.rows + per_cta - 1) / per_cta, cap = (int64_t)num_sms * 8;
        const dim3 grid((unsigned)(want < cap ? want : cap));
        switch (s.nv) {
        case 1: return dc_launch_pdl(k_rows<T, VE, 1, false, NORM, QUANT>, grid, 256, 0, stream, a, s.group);
        case 2: return dc_launch_pdl(k_rows<T, VE, 2, false, NORM, QUANT>, grid, 256, 0, stream, a, s.group);
        case 3: return dc_launch_pdl(k_rows<T, VE, 3, false, NORM, QUANT>, grid, 256, 0, stream, a, s.group);
        case 4: return dc_launch_pdl(k_rows<T, VE, 4, false, NORM, QUANT>, grid, 256, 0, stream, a, s.group);
        default: return dc_launch_pdl(k_rows<T, VE, 8, false, NORM, QUANT>, grid, 256, 0, stream, a, s.group);
        }
    }
    // a CTA per row: as many threads as leave each four vectors, up to 1024
    const int want = dc_div_up(dc_div_up(nvec, 4), 32) * 32, threads = want < 128 ? 128 : want > 1024 ? 1024 : want;
    const int64_t cap = (int64_t)num_sms * (2048 / threads);
    const dim3 grid((unsigned)(a.rows < cap ? a.rows : cap));
    if (nvec <= threads * 4) return dc_launch_pdl(k_rows<T, VE, 4, true, NORM, QUANT>, grid, threads, 0, stream, a, 32);
    if (VE < 8 && nvec <= threads * 8) return dc_launch_pdl(k_rows<T, VE, 8, true, NORM, QUANT>, grid, threads, 0, stream, a, 32);
    return dc_launch_pdl(k_rows_long<T, NORM, QUANT>, grid, 1024, 0, stream, a);
}

template <typename T, int VE>
cudaError_t launch_rows_kind(const dc_rows_args& a, bool norm, int num_sms, cudaStream_t stream)
{
    if (!norm) return launch_rows<T, VE, false, true>(a, num_sms, stream);
    return a.q ? launch_rows<T, VE, true, true>(a, num_sms, stream) : launch_rows<T, VE, true, false>(a, num_sms, stream);
}

template <typename T, int VE>
cudaError_t launch_backward(const dc_backward_args& a, int num_sms, cudaStream_t stream, int* ctas)
{
    const int nvec = a.channels / VE;
    constexpr int MOST = 16 / VE;                                    // 16 channels per lane: their sums, values and weights stay in registers
    const Split s = split_row(nvec, MOST);
    const int most_ctas = 2 * num_sms < kBackwardCtas ? 2 * num_sms : kBackwardCtas;
    if (s.group != 0) {
        constexpr int THREADS = 384;
        const int64_t per_cta = (int64_t)(THREADS / 32) * (32 / s.group), want = (a.rows + per_cta - 1) / per_cta;
        *ctas = (int)(want < 1 ? 1 : want < most_ctas ? want : most_ctas);
        const size_t smem = (size_t)2 * a.channels * sizeof(float);
#define DC_BWD(N) return dc_launch_pdl(k_norm_backward<T, VE, N, false, THREADS>, dim3((unsigned)*ctas), THREADS, smem, stream, a, s.group)
        if (s.nv <= 1) DC_BWD(1);
        if (s.nv <= 2) DC_BWD(MOST < 2 ? MOST : 2);
        if (s.nv <= 4) DC_BWD(MOST < 4 ? MOST : 4);
        if (s.nv <= 8) DC_BWD(MOST < 8 ? MOST : 8);
        DC_BWD(MOST);
#undef DC_BWD
    }
    *ctas = (int)(a.rows < 1 ? 1 : a.rows < most_ctas ? a.rows : most_ctas);
    const int want = dc_div_up(dc_div_up(nvec, MOST), 32) * 32;
    if (want <= 512) return dc_launch_pdl(k_norm_backward<T, VE, MOST, true, 512>, dim3((unsigned)*ctas), want, 0, stream, a, 32);
    return dc_launch_pdl(k_norm_backward<T, VE, MOST, true, 1024>, dim3((unsigned)*ctas), want, 0, stream, a, 32);
}

constexpr int kMostNormChannels = 16384;

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
    if (channels > kMostNormChannels) return DC_ERR_LIMIT;
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
    if (channels > kMostNormChannels) return DC_ERR_LIMIT;
    if (!floats_ok(gamma_dev) || !floats_ok(mean_dev) || !floats_ok(rstd_dev) || !floats_ok(dgamma_dev) || !floats_ok(dbeta_dev)) return DC_ERR_ARG;
    const bool weights = dgamma_dev || dbeta_dev;
    size_t need = 0;
    dc_layer_norm_workspace(channels, &need);
    if (weights && (!workspace_dev || (uintptr_t)workspace_dev % sizeof(float) || workspace_bytes < need)) return DC_ERR_ARG;
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
