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
#include <atomic>

#include "dc_quantise.cuh"

namespace {

constexpr int kBackwardCtas = 296;      // partial sums of a gradient's columns: two CTAs for each SM of a B200

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
    constexpr bool KEEP = NORM && NV * VE <= (VE == 8 && BLOCK == 0 ? 32 : 16);
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
                    for (int k = 0; k < P; ++k) d[v * P + k] = fma2(rounded(d[v * P + k], both<F>(rstd)), KEEP ? gk[KEEP ? v : 0][k] : g[k], KEEP ? bk[KEEP ? v : 0][k] : b[k]);
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
    for (int row = blockIdx.x; row < (int)a.rows; row += gridDim.x) {
        if (QUANT && !NORM && !wanted(a, row)) continue;
        float* const slot = red + parity * 96;
        const T* const x = (const T*)row_at(a.x, a.x_pitch, row);
        T* const y = (T*)row_at(a.y, a.y_pitch, row);
        float mean = 0.f, rstd = 1.f;
        auto at = [&](int i) { float v; V::open(x[i], &v); return v; };
        auto value = [&](int i) -> T {                            // as the map holds it
            float v = at(i);
            if (NORM) v = fmaf(rounded(v - mean, rstd), a.gamma ? dc_ld(a.gamma + i) : 1.f, a.beta ? dc_ld(a.beta + i) : 0.f);
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
        parity ^= 1;                    // rows that are passed over reduce nothing and take no turn: two neighbouring reductions would meet in one slot
    }
}

struct dc_backward_args {
    const void* dy; size_t dy_pitch; const void* x; size_t x_pitch;
    const float *gamma, *mean, *rstd;
    int64_t rows; int channels;
    void* dx; size_t dx_pitch;          // or NULL
    float* partial;                     // [CTAs][2][channels], or NULL: no gradients of the weights
    float *dgamma, *dbeta;              // a single CTA's sums go straight there (either may be NULL)
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
        if (gridDim.x > 1) out[i] = s;
        else if (i < a.channels) { if (a.dgamma) a.dgamma[i] = s; }
        else if (a.dbeta) a.dbeta[i - a.channels] = s;
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
    static std::atomic<int> resident[33];            // CTAs of so many warps that an SM holds
    int fit = resident[threads / 32].load(std::memory_order_relaxed);
    if (!fit) {
        int n = 0;
        const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, k_rows<T, VE, NV, BLOCK, NORM, QUANT, FULL>, threads, 0);
        if (e != cudaSuccess) return e;
        resident[threads / 32].store(fit = n > 0 ? n : 1, std::memory_order_relaxed);
    }
    const int64_t cap = (int64_t)num_sms * fit;
    return dc_launch_pdl(k_rows<T, VE, NV, BLOCK, NORM, QUANT, FULL>, dim3((unsigned)(ctas < cap ? ctas : cap)), threads, 0, stream, a, group);
}

// PART: rows that leave places idle come here too.
template <typename T, int VE, int NV, int BLOCK, bool NORM, bool QUANT, bool PART>
cudaError_t launch_rows_of(const dc_rows_args& a, int group, int threads, int64_t ctas, int num_sms, cudaStream_t stream)
{
    if constexpr (PART)
        if (a.channels / VE != NV * (BLOCK ? threads : group)) return launch_rows_as<T, VE, NV, BLOCK, NORM, QUANT, false>(a, group, threads, ctas, num_sms, stream);
    return launch_rows_as<T, VE, NV, BLOCK, NORM, QUANT, true>(a, group, threads, ctas, num_sms, stream);
}

template <typename T, int VE, bool NORM, bool QUANT>
cudaError_t launch_rows(const dc_rows_args& a, int num_sms, cudaStream_t stream)
{
    const int nvec = a.channels / VE;
    constexpr bool NORM8 = NORM && VE == 8;
#define DC_ROWS(NV, BLOCK, PART, G, THREADS, CTAS) return launch_rows_of<T, VE, NV, BLOCK, NORM, QUANT, (PART)>(a, G, THREADS, CTAS, num_sms, stream)
    // few rows: a CTA for each, a vector per thread
    if (nvec > 32 && nvec <= 1024 && a.rows <= 2 * num_sms) DC_ROWS(1, 1024, true, 32, dc_div_up(nvec, 32) * 32, a.rows);
    // Normalised: 16 channels per lane, whose weights stay in its registers (56 x 56 x 256, 32 streams, bf16: 19.3 us, 22.3 with 32), or 24 of bfloat16
    // where that leaves fewer places idle: 25088 x 384 into 8 bits 10.8 us and 13.8, x 768 17.6 and 21.0 (its weights from L1 before).
    constexpr int MOST = VE == 1 ? 8 : NORM8 ? 3 : 4;
    Split s = split_row(nvec, MOST);
    // Longer ones likewise, with a CTA to a row: 12000 x 2048 bf16 20.7 us, 26.5 with a warp; into 8 bits 6000 x 1536 11.3 and 15.0.  Four vectors for
    // every lane of a warp need no barriers and just fit: 25088 x 1024 into 8 bits 21.7 us and 24.7, 25000 x 1024 19.2 and 20.4; with places idle
    // (25088 x 1000 26.6 and 25.5) or fewer than four rows to a resident warp (5000 x 1024 5.4 and 5.2) the CTA is better.
    if constexpr (NORM8)
        if (s.group == 0 && nvec <= 1024 && !(nvec == 4 * 32 && a.rows >= 64 * num_sms)) DC_ROWS(2, 512, true, 32, dc_div_up(dc_div_up(nvec, 2), 32) * 32, a.rows);
    if (s.group == 0) s = split_row(nvec, VE == 1 ? 16 : 4);
    if constexpr (VE > 1 && !NORM8) if (s.group == 0 && nvec <= 32 * 8) s = {32, 8};
    if (s.group != 0) {
        const int64_t warps = (a.rows + 32 / s.group - 1) / (32 / s.group);
        const int per_cta = warps >= 8 * (int64_t)num_sms ? 8 : warps >= 4 * (int64_t)num_sms ? 4 : warps >= 2 * (int64_t)num_sms ? 2 : 1;
        const int64_t ctas = (warps + per_cta - 1) / per_cta;
        // With places idle no count is split_row's choice whose double is within its limit: half the lanes then have as few places in all.
        switch (s.nv) {
        case 1: DC_ROWS(1, 0, false, s.group, per_cta * 32, ctas);
        case 2: DC_ROWS(2, 0, 2 * 2 > MOST, s.group, per_cta * 32, ctas);
        case 3: DC_ROWS(3, 0, 2 * 3 > MOST, s.group, per_cta * 32, ctas);
        case 4: DC_ROWS(4, 0, 2 * 4 > MOST && !NORM8, s.group, per_cta * 32, ctas);        // (NORM8: see above)
        }
        if constexpr (VE == 1) {
            if (s.nv > 12) DC_ROWS(16, 0, true, s.group, per_cta * 32, ctas);
            if (s.nv > 8) DC_ROWS(12, 0, true, s.group, per_cta * 32, ctas);
        }
        if constexpr (!NORM8) DC_ROWS(8, 0, true, s.group, per_cta * 32, ctas);
    }
    // a CTA per row: as many threads as leave each four vectors (single elements: 12), up to 1024; normalised rows end at kMostNormChannels
    if constexpr (VE == 1) {
        if (nvec <= 512 * 12) DC_ROWS(12, 512, true, 32, dc_div_up(dc_div_up(nvec, 12), 32) * 32, a.rows);
        if (nvec <= 8192) DC_ROWS(8, 1024, true, 32, 1024, a.rows);
    } else {
        const int want = dc_div_up(dc_div_up(nvec, 4), 32) * 32, threads = want < 128 ? 128 : want > 1024 ? 1024 : want;
        if (threads <= 512) DC_ROWS(4, 512, true, 32, threads, a.rows);
        if constexpr (!NORM8) if (nvec <= 4096) DC_ROWS(4, 1024, true, 32, threads, a.rows);
        if constexpr (VE == 4 && !NORM) if (nvec <= 8192) DC_ROWS(8, 1024, true, 32, threads, a.rows);
    }
#undef DC_ROWS
    if constexpr (NORM && VE > 1) return cudaErrorInvalidValue;       // (no row is that long)
    else return dc_launch_pdl(k_rows_long<T, NORM, QUANT>, dim3((unsigned)(a.rows < 2 * num_sms ? a.rows : 2 * num_sms)), 1024, 0, stream, a);
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
    // Up to three rows to a team: one CTA, which needs no second launch to join others' sums (20 x 100 bf16 3.3 us in a graph and 7.4 a pass, 4.3 and 9.7
    // with one; from the fourth row on a turn's half microsecond adds up to more than the join).
    const bool alone = want <= 3 && !(BLOCK && teams == 1);
    *ctas = alone ? 1 : (int)(want < 2 ? 2 : want < most ? want : most);
    if (smem > 48 * 1024 - 1024) {
        static dc_once_per_device attr_set;
        int device;
        cudaError_t e = cudaGetDevice(&device);
        if (e == cudaSuccess)
            e = attr_set.ensure(device, [] { return cudaFuncSetAttribute(k_norm_backward<T, VE, NV, BLOCK, THREADS, CTAS, FULL>, cudaFuncAttributeMaxDynamicSharedMemorySize, 128 * 1024); });
        if (e != cudaSuccess) return e;
    }
    return dc_launch_pdl(k_norm_backward<T, VE, NV, BLOCK, THREADS, CTAS, FULL>, dim3((unsigned)*ctas), threads, smem, stream, a, group);
}

// Rows of up to 512 channels belong to a warp's lanes, with 8 or 16 channels each: 16 of bfloat16, whose raw values ahead take half the registers
// (56 x 56 x 256, 32 streams: 32.6 us, 37.0 with 8), 8 of float32 (50000 x 128: 17.4 us, 19.8 with 16).  Longer rows belong to teams of warps.
template <typename T, int VE>
cudaError_t launch_backward(const dc_backward_args& a, int num_sms, cudaStream_t stream, int* ctas)
{
    const int nvec = a.channels / VE;
    constexpr int N8 = 8 / VE, N16 = 16 / VE, T16 = VE == 8 ? 256 : 384, C16 = VE == 8 ? 2 : 1, T24 = VE == 8 ? 384 : 512;
    if constexpr (VE > 1) {
        // Three vectors where two leave more places idle: bf16 50000 x 384 24.9 us and 28.4, 25000 x 768 25.2 and 32.9 (as teams of 96 threads), f32
        // 50000 x 192 22.8 and 26.1, 25000 x 384 23.0 and 25.1.  Their one large CTA starts later: bf16 100 x 384 5.1 us and 4.6, 1000 x 768 6.2 either way.
        const Split t = split_row(nvec, 3);
        if (t.nv == 3 && a.rows > 1000) {
            if (nvec == t.group * 3) return launch_backward_as<T, VE, 3, false, T24, 1, true>(a, t.group, num_sms, stream, ctas);
            return launch_backward_as<T, VE, 3, false, T24, 1, false>(a, t.group, num_sms, stream, ctas);
        }
    }
    Split s = split_row(nvec, VE == 8 ? N16 : N8);
    if (s.group == 0) s = split_row(nvec, N16);
    if (s.group != 0) {
        const bool full = nvec == s.group * s.nv;
        if (s.nv <= N8) {
            if constexpr (N8 > 1)                                 // (a single vector per lane leaves no place idle)
                if (!full || s.nv != N8) return launch_backward_as<T, VE, N8, false, 320, 2, false>(a, s.group, num_sms, stream, ctas);
            return launch_backward_as<T, VE, N8, false, 320, 2, true>(a, s.group, num_sms, stream, ctas);
        }
        if constexpr (VE == 1) if (s.nv <= 12) return launch_backward_as<T, VE, 12, false, 256, 2, false>(a, s.group, num_sms, stream, ctas);
        if (full && s.nv == N16) return launch_backward_as<T, VE, N16, false, T16, C16, true>(a, s.group, num_sms, stream, ctas);
        return launch_backward_as<T, VE, N16, false, T16, C16, false>(a, s.group, num_sms, stream, ctas);
    }
    // Of large maps, longer rows too have two vectors per thread, or three where that takes no more places: bf16 20000 x 1024 26.9 us and 33.5 with one,
    // 5000 x 4096 29.7 and 34.6, 14000 x 1536 28.7 and 29.8 with two, f32 12000 x 768 22.7 and 25.5 with two; of small ones more threads: bf16
    // 2000 x 1024 7.5 and 7.4, f32 1500 x 1024 8.4 and 7.2.
    if constexpr (VE > 1)
        if (a.rows * a.channels > 1 << 21) {
            const int two = dc_div_up(dc_div_up(nvec, 2), 32) * 32, three = dc_div_up(dc_div_up(nvec, 3), 32) * 32;
            if (three <= T24 && 3 * three <= 2 * two) {
                if (nvec == three * 3) return launch_backward_as<T, VE, 3, true, T24, 1, true>(a, three, num_sms, stream, ctas);
                return launch_backward_as<T, VE, 3, true, T24, 1, false>(a, three, num_sms, stream, ctas);
            }
            if constexpr (VE == 8)
                if (two <= 512) {
                    if (nvec == two * 2) return launch_backward_as<T, VE, 2, true, 512, 1, true>(a, two, num_sms, stream, ctas);
                    return launch_backward_as<T, VE, 2, true, 512, 1, false>(a, two, num_sms, stream, ctas);
                }
        }
    // Beyond 512 threads there are 64 registers for each, too few for a row ahead and the sums: 40 to 230 bytes a thread spill up to 8192 channels, 810 to 910 beyond.
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
    static std::atomic<int> sms[64];
    DC_CUDA(cudaGetDevice(device));
    if (*device < 0 || *device >= 64) { DC_CUDA(cudaDeviceGetAttribute(num_sms, cudaDevAttrMultiProcessorCount, *device)); return DC_OK; }
    *num_sms = sms[*device].load(std::memory_order_relaxed);
    if (*num_sms) return DC_OK;
    DC_CUDA(cudaDeviceGetAttribute(num_sms, cudaDevAttrMultiProcessorCount, *device));
    sms[*device].store(*num_sms, std::memory_order_relaxed);
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
    dc_backward_args a = {dy_dev, dy_pitch, x_dev, x_pitch, gamma_dev, mean_dev, rstd_dev, rows, channels, dx_dev, dx_pitch, weights ? (float*)workspace_dev : nullptr, dgamma_dev, dbeta_dev};
    int device = 0, sms = 0, ctas = 0;
    const int rc = dc_current_device(&device, &sms);
    if (rc != DC_OK) return rc;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    const bool vec = aligned16(x_dev, x_pitch) && aligned16(dy_dev, dy_pitch) && (!dx_dev || aligned16(dx_dev, dx_pitch)) && ((size_t)channels * elt) % 16 == 0 &&
                     (uintptr_t)gamma_dev % 16 == 0;
    if (dtype == DC_BF16) DC_CUDA(vec ? (launch_backward<__nv_bfloat16, 8>(a, sms, stream, &ctas)) : (launch_backward<__nv_bfloat16, 1>(a, sms, stream, &ctas)));
    else DC_CUDA(vec ? (launch_backward<float, 4>(a, sms, stream, &ctas)) : (launch_backward<float, 1>(a, sms, stream, &ctas)));
    if (weights && ctas != 1)
        DC_CUDA(dc_launch_pdl(k_join, dim3((unsigned)dc_div_up(2 * channels, 32)), 1024, 0, stream, (const float*)workspace_dev, ctas, (int)channels, dgamma_dev, dbeta_dev));
    return DC_OK;
}

}  // extern "C"
