// A layer of 8-bit integers on one row, or a few short ones, in one launch.
//
// What bounds such a layer is its weights, each read once, and the launch; it needs no tensor core.  Every CTA puts the rows into 8 bits itself, into
// shared memory (about a microsecond, beside a launch and a wait of its own), while its first weights are on their way to L2.  A channel's
// weights belong to `group` lanes of a warp, 16 values to a lane and step, four or eight steps in flight; a step is one 16-byte load and four dp4a per
// row of x.  The sums are exact, so they are the same as the other kernels'.
// us in a graph (us a pass from the host), so and with dc_norm.cu's and dc_quant.cu's kernels: 1 x 1024 x 256 3.2 (3.3) and 3.9 (5.7), 1 x 4096 x 1000
// 4.2 (4.2) and 5.0 (5.7), 1 x 4096 x 4096 5.3 and 6.6, 1 x 9216 x 4096 11.5 and 11.7, 1 x 16384 x 4096 16.2 and 15.8; 2 x 2048 x 4096 5.2 (5.0) and 5.2 (6.1), 2 x 4096 x 4096
// 6.7 and 6.7; 4 x 1024 x 256 4.1 (4.2) and 4.0 (5.7), 4 x 4096 x 1000 6.2 and 5.3, 8 x 1024 x 256 4.9 (5.0) and 4.3 (5.8).
#include "dc_quantise.cuh"

namespace {

struct FewArgs {
    dc_product_args p;
    const void* x; size_t x_pitch;      // rows of the map's type
    int group, units;                   // lanes per channel; units of 16 values in a row, the last one perhaps cut
};

constexpr int kFewThreads = 512;

// Sixteen weights; the last unit of a row may be cut: nothing behind the row's values is read.
__device__ __forceinline__ int4 unit_of(const int8_t* row, int u, int k)
{
    if (16 * u + 16 <= k) return *(const int4*)(row + 16 * u);
    int4 v = make_int4(0, 0, 0, 0);
    int8_t* const b = (int8_t*)&v;
#pragma unroll
    for (int e = 0; e < 16; ++e)
        if (16 * u + e < k) b[e] = row[16 * u + e];
    return v;
}

template <typename T, int VE, int M>
__global__ void __launch_bounds__(kFewThreads) k_product_few(const FewArgs a)
{
    typedef Vec<T, VE> V;
    extern __shared__ int4 xs[];                                  // [M][units]
    __shared__ uint32_t most[M];
    __shared__ float scale[M];
    const dc_product_args& p = a.p;
    const int lane = threadIdx.x & 31, m = (int)p.m, k = p.k;
    const int group = a.group, sub = lane & (group - 1), per_warp = 32 / group, warps = blockDim.x >> 5;
    const int first = (blockIdx.x * warps + (threadIdx.x >> 5)) * per_warp + lane / group, step = gridDim.x * warps * per_warp;
    dc_pdl_wait();
    dc_pdl_release();

    // the first channel's weights on their way to L2 meanwhile: a warp has one channel or few
    if (first < p.n)
        for (int at = sub * 128; at < k; at += group * 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(p.b + (size_t)first * p.b_pitch + at));

    // ---------------- the rows into shared memory ----------------
    {
        // some warps to a row; what four vectors per lane do not hold is read twice, the second time from L1
        typename V::Raw raw[4];
        const int nvec = k / VE, team = warps > M ? warps / M : 1, turn = warps / team, warp = threadIdx.x >> 5, at = (warp % team) * 32 + lane, r0 = warp / team;
        auto vec_at = [&](int r, int i) { return *(const typename V::Raw*)((const char*)a.x + (size_t)r * a.x_pitch + (size_t)i * sizeof(typename V::Raw)); };
        if (threadIdx.x < M) most[threadIdx.x] = 0;
        for (int r = threadIdx.x; r < M; r += blockDim.x) xs[r * a.units + a.units - 1] = make_int4(0, 0, 0, 0);   // behind the values of the last unit
        for (int i = m * a.units + threadIdx.x; i < M * a.units; i += blockDim.x) xs[i] = make_int4(0, 0, 0, 0);
        __syncthreads();
        const int wide = team * 32;
        auto fetch = [&](int r, int i0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) raw[e] = i0 + e * wide < nvec ? vec_at(r, i0 + e * wide) : raw_zero<typename V::Raw>();
        };
        const bool held = nvec <= 4 * wide && m <= turn;
        for (int r = r0; r < m; r += turn) {
            uint32_t t = 0;
            for (int i0 = at; i0 < nvec; i0 += 4 * wide) {
                fetch(r, i0);
#pragma unroll
                for (int e = 0; e < 4; ++e) t = raw_most(t, raw[e]);
            }
            t = __reduce_max_sync(0xffffffffu, most_of<T>(t));
            if (lane == 0) atomicMax(&most[r], t);                // the same whatever the order
        }
        __syncthreads();
        for (int r = r0; r < m; r += turn) {
            const RowScale s = row_scale(most[r]);
            int8_t* const to = (int8_t*)(xs + r * a.units);
            for (int i0 = at; i0 < nvec; i0 += 4 * wide) {
                if (!held) fetch(r, i0);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = i0 + e * wide;
                    if (i >= nvec) break;
                    typename V::F f[V::P];
                    V::open(raw[e], f);
                    if (s.lift != 1.f)
#pragma unroll
                        for (int h = 0; h < V::P; ++h) f[h] = s.lift != 0.f ? mul2(f[h], both<typename V::F>(s.lift)) : both<typename V::F>(0.f);
                    uint32_t w[VE == 8 ? 2 : 1];
                    quantise<T, VE>(f, s.inv, s.most, w);
                    store_q<VE>(to + i * VE, w);
                }
            }
        }
        if (threadIdx.x < M) scale[threadIdx.x] = row_scale(most[threadIdx.x]).scale;
        __syncthreads();
    }

    // ---------------- channels ----------------
    for (int base = first - lane / group; base < p.n; base += step) {        // the same in all lanes of a warp
        const int j = base + lane / group;
        const bool there = j < p.n;
        const int8_t* const row = p.b + (size_t)(there ? j : 0) * p.b_pitch;
        int sum[M];
#pragma unroll
        for (int r = 0; r < M; ++r) sum[r] = 0;
        constexpr int U = M == 1 ? 8 : 4;                         // steps in flight
        for (int u0 = sub; u0 < a.units; u0 += U * group) {
            int4 w[U];
#pragma unroll
            for (int e = 0; e < U; ++e) w[e] = u0 + e * group < a.units ? unit_of(row, u0 + e * group, k) : make_int4(0, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < U; ++e) {
                if (u0 + e * group >= a.units) break;
#pragma unroll
                for (int r = 0; r < M; ++r) {
                    const int4 x = xs[r * a.units + u0 + e * group];
                    sum[r] = __dp4a(w[e].x, x.x, __dp4a(w[e].y, x.y, __dp4a(w[e].z, x.z, __dp4a(w[e].w, x.w, sum[r]))));
                }
            }
        }
#pragma unroll
        for (int r = 0; r < M; ++r)
#pragma unroll
            for (int o = 16; o > 0; o >>= 1)
                if (o < group) sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], o);
        if (!there) continue;
        const float sb = dc_ld(p.b_scale + j), bias = p.bias ? dc_ld(p.bias + j) : 0.f;
#pragma unroll
        for (int r = 0; r < M; ++r)
            if (r < m && sub == (r & (group - 1))) {
                float f = fmaf((float)sum[r] * scale[r], sb, bias);
                if (p.relu) asm("max.NaN.f32 %0, %0, 0f00000000;" : "+f"(f));
                T* const out = (T*)((char*)p.out + (size_t)r * p.out_pitch) + j;
                if constexpr (sizeof(T) == 4) *out = f;
                else *out = __float2bfloat16_rn(f);
            }
    }
}

template <typename T, int VE, int M>
int launch(const FewArgs& a, int threads, size_t smem, int device, int num_sms, cudaStream_t stream)
{
    static dc_once_per_device attr_set;
    DC_CUDA(attr_set.ensure(device, [] { return cudaFuncSetAttribute(k_product_few<T, VE, M>, cudaFuncAttributeMaxDynamicSharedMemorySize, DC_FEW_BYTES); }));
    const int per_cta = threads / 32 * (32 / a.group), want = dc_div_up(a.p.n, per_cta), fit = (int)(DC_FEW_BYTES / (smem + 1024)), cap = num_sms * (fit < 2 ? 1 : 2 * (kFewThreads / threads));
    DC_CUDA(dc_launch_pdl(k_product_few<T, VE, M>, dim3((unsigned)(want < cap ? want : cap)), threads, smem, stream, a));
    return DC_OK;
}

template <typename T, int VE>
int launch_rows(const FewArgs& a, int threads, size_t per_row, int device, int num_sms, cudaStream_t stream)
{
    if (a.p.m <= 1) return launch<T, VE, 1>(a, threads, per_row, device, num_sms, stream);
    if (a.p.m <= 2) return launch<T, VE, 2>(a, threads, 2 * per_row, device, num_sms, stream);
    if (a.p.m <= 4) return launch<T, VE, 4>(a, threads, 4 * per_row, device, num_sms, stream);
    return launch<T, VE, 8>(a, threads, 8 * per_row, device, num_sms, stream);
}

}  // namespace

// Up to 52 MB of weights for one row, 12 for two, 1 for more, whose values are at most 4096 in all.  bf16, us in a graph, so and with the two launches: one row of
// 4096 channels out 9.3 and 11.1 at 34 MB, 11.3 and 12.3 at 42, 12.0 and 12.4 at 46, 13.0 and 13.2 at 50, 13.9 and 13.6 at 55, 14.4 and 14.3 at 59, 16.3 and 15.6 at 67, 23.8 and 21.0 at 103;
// longer rows meet there too (16384 x 3584, 59 MB, 14.9 and 14.6), shorter ones later (4096 x 16384, 67 MB, 13.9 and 21.7); two rows 6.2 and 7.2 at 10 MB, 8.4 and 8.0 at 14.
bool dc_few_pays(int64_t m, int n, int k)
{
    const double weights = (double)n * (double)dc_quant_pitch(k);
    if (dc_quant_pitch(k) * (size_t)(m < 2 ? 1 : 2) > DC_FEW_BYTES) return false;
    return m == 1 ? weights <= 52e6 : m == 2 ? weights <= 12e6 : m <= 8 && m * k <= 4096 && weights <= 1e6;
}

int dc_launch_few(const dc_product_args& p, const void* x, size_t x_pitch, int dtype, int device, int num_sms, cudaStream_t stream)
{
    FewArgs a = {};
    a.p = p; a.x = x; a.x_pitch = x_pitch;
    a.units = (int)(dc_quant_pitch(p.k) / 16);
    a.group = 32;                                                 // four units to a lane at most, where that leaves a channel fewer lanes
    while (a.group > 8 && a.group * 2 >= a.units) a.group >>= 1;
    // large products: whole SMs; small ones: more CTAs
    const long long lanes = (long long)p.n * a.group;
    const long long values = p.m * p.k / 32;                      // four vectors of x to a thread
    const int threads = lanes >= (long long)num_sms * 512 || values > 256 ? 512 : lanes >= (long long)num_sms * 256 || values > 128 ? 256 : 128;
    const size_t per_row = (size_t)a.units * 16;
    const int elt = dtype == DC_BF16 ? 2 : 4;
    const bool vec = (uintptr_t)x % 16 == 0 && (p.m < 2 || x_pitch % 16 == 0) && ((size_t)p.k * elt) % 16 == 0;
    if (dtype == DC_BF16) return vec ? launch_rows<__nv_bfloat16, 8>(a, threads, per_row, device, num_sms, stream) : launch_rows<__nv_bfloat16, 1>(a, threads, per_row, device, num_sms, stream);
    return vec ? launch_rows<float, 4>(a, threads, per_row, device, num_sms, stream) : launch_rows<float, 1>(a, threads, per_row, device, num_sms, stream);
}
