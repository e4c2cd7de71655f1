// Matrix products in 8-bit integers with a scale for each row of either side: fully connected layers and 1 x 1 convolutions whose
// pixels and weights are held in 8 bits.
//
//   out[r][j] = relu(a_scale[r] b_scale[j] sum_k a[r][k] b[j][k] + bias[j])
//
// The sums are int32 and exact (at most 131071 terms, so that even 128 * 128 in every term fits); they are scaled and the bias is
// added in float32 and rounded once, to the map's type.
//
// k_product: tcgen05.mma kind::i8 on tiles of 128 rows, operands by TMA in 128-byte swizzled rows of 128 values, accumulators double
// buffered in tensor memory, so that the sixteen warps that scale and store a tile work beside the MMAs of the next.  Large products run on
// CTA pairs: 256 rows x 256 columns, each CTA loading its own 128 rows of a and half of b's, which is a third less traffic from L2 per
// product than a CTA alone has.
#include <atomic>

#include "dc_product.cuh"

namespace {

constexpr int kMaxStages = 9;
constexpr int kEpiWarps = 16, kThreads = (2 + kEpiWarps) * 32;
constexpr int kStage = 32 * 64;                               // a warp's 32 rows on their way out, 64 bytes each

__device__ int32_t g_status;                                  // the status word of launches without a cache

struct ProductArgs {
    dc_product_args p;
    int bufs;                                                 // places a warp stages its boxes in, 1 or 2
    int BN, NB, stages, stage_bytes, kchunks, k_last;         // columns per tile, column blocks; k_last: MMAs (32 values) of the last chunk
    int m_tiles;
    uint32_t idesc, tmem_cols;
    int wide, boxes;                                          // out takes 16-byte stores; is written in boxes by TMA
};

struct Ctl {
    unsigned long long full[kMaxStages], empty[kMaxStages], tmem_full[2], tmem_empty[2];
    uint32_t tmem_base;
    volatile int abort_flag;
    unsigned long long wait_ns;
};
constexpr int kSmem = 227 * 1024, kRoom = kSmem - 1024 - (int)sizeof(Ctl);      // for the ring and the staging

// As DC_UMMA_CHUNK, for 8-bit integers: n (1 to 4) MMAs of K = 32.
#define DC_UMMA_I8(name, group)                                                                                                                 \
    __device__ __forceinline__ void name(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate, int n)       \
    {                                                                                                                                           \
        _Pragma("unroll") for (int k = 0; k < 4; ++k)                                                                                           \
            if (k < n)                                                                                                                          \
                asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t" \
                             "tcgen05.mma." group ".kind::i8 [%0], da, db, %4, p;\n\t}"                                                         \
                             ::"r"(d), "r"(a_lo + 2u * k), "r"(b_lo + 2u * k), "r"(hi), "r"(idesc), "r"(k == 0 ? accumulate : 1u) : "memory");   \
    }
DC_UMMA_I8(umma_i8, "cta_group::1")
DC_UMMA_I8(umma_i8_pair, "cta_group::2")
#undef DC_UMMA_I8

__device__ __forceinline__ bool wait_at(uint32_t bar, uint32_t parity, Ctl* ctl, int32_t* status)
{
    return mbar_wait_at(bar, parity, &ctl->abort_flag, &ctl->wait_ns, status);
}

// acc sa scale + bias of two columns, for one row: float32, two at once.
__device__ __forceinline__ float2 finish2(uint32_t a0, uint32_t a1, float sa, float2 s, float2 b)
{
    float2 f;
    asm("{\n\t.reg .b64 a, s, b, m;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 m, {%4, %4};\n\tmov.b64 s, {%5, %6};\n\tmov.b64 b, {%7, %8};\n\t"
        "mul.rn.f32x2 a, a, m;\n\tfma.rn.f32x2 a, a, s, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "=f"(f.x), "=f"(f.y) : "f"((float)(int)a0), "f"((float)(int)a1), "f"(sa), "f"(s.x), "f"(s.y), "f"(b.x), "f"(b.y));
    return f;
}
// Sixteen rows x 32 columns of tensor memory: column group j (8 columns) in r[4 j ...]; a lane has columns 2 (lane % 4), + 1 of rows lane / 4
// (r[4 j], r[4 j + 1]) and lane / 4 + 8.
__device__ __forceinline__ void tmem_ld_16x32(uint32_t taddr, uint32_t* r)
{
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void stmatrix4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
// The scales and biases of two neighbouring columns in each of four groups of eight, from `col` on; beyond the last column: zeros.  (dc_ld: the
// kernel before may have written them.)
__device__ __forceinline__ void column_weights(const dc_product_args& p, int col, bool whole, float2* s, float2* b)
{
    if (whole) {
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = dc_ld((const float2*)(p.b_scale + col + 8 * j));
        if (p.bias)
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = dc_ld((const float2*)(p.bias + col + 8 * j));
        else
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = make_float2(0.f, 0.f);
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int c = col + 8 * j;
        s[j] = make_float2(c < p.n ? dc_ld(p.b_scale + c) : 0.f, c + 1 < p.n ? dc_ld(p.b_scale + c + 1) : 0.f);
        b[j] = make_float2(p.bias && c < p.n ? dc_ld(p.bias + c) : 0.f, p.bias && c + 1 < p.n ? dc_ld(p.bias + c + 1) : 0.f);
    }
}

// The place of row r of a tile-ordered map in the map itself, or -1: beyond the map, in the gap behind a line of pixels, or reused.
__device__ __forceinline__ int64_t out_row(const dc_product_args& p, int tile, int r)
{
    const int row = tile * kTileM + r;
    if (row >= p.m) return -1;
    if (p.masks && ((__ldcg(p.masks + (size_t)tile * 4 + (r >> 5)) >> (r & 31)) & 1u)) return -1;
    if (p.padded == 0) return row;
    const int line = row / p.padded, x = row - line * p.padded;
    return x < p.width ? (int64_t)line * p.width + x : -1;
}

// LIST: a partial convolution's pixels (tile_list, masks, gaps behind lines).
template <bool PAIR, bool LIST, bool RELU, typename T>
__global__ void __launch_bounds__(kThreads, 1) k_product(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmC, const ProductArgs a)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* ring = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* staging = ring + a.stages * a.stage_bytes;
    Ctl* ctl = (Ctl*)(staging + kEpiWarps * kStage * a.bufs);
    const dc_product_args& p = a.p;
    int32_t* const status = p.status ? p.status : &g_status;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int rank = PAIR ? (int)cluster_rank() : 0, first = PAIR ? blockIdx.x >> 1 : blockIdx.x, step = PAIR ? gridDim.x >> 1 : gridDim.x;
    constexpr int M = PAIR ? 2 : 1;                           // tiles per item

    if (threadIdx.x == 0) {
        for (int i = 0; i < a.stages; ++i) { mbar_init(&ctl->full[i], 1); mbar_init(&ctl->empty[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&ctl->tmem_full[i], 1); mbar_init(&ctl->tmem_empty[i], kEpiWarps * M); }
        ctl->abort_flag = 0;
        ctl->wait_ns = kWaitNs;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmA) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmB) : "memory");
    }
    if (warp == 1) {
        if (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(a.tmem_cols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(a.tmem_cols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();                             // both CTAs' barriers exist before either is signalled from outside
    tc_fence_after();
    const uint32_t tmem_base = ctl->tmem_base;
    dc_pdl_wait();
    dc_pdl_release();
    const int n_tiles = LIST && p.tile_list ? __ldcg(p.tile_count) : a.m_tiles;
    const int n_items = (n_tiles + M - 1) / M * a.NB;
    // tile `rank` of an item; an absent second tile repeats the first, and nothing of it is stored
    auto tile_of = [&](int group, bool* there) -> int {
        const int idx = group * M + rank;
        *there = idx < n_tiles;
        const int at = *there ? idx : idx - rank;
        return LIST && p.tile_list ? __ldcg(p.tile_list + at) : at;
    };
    const uint32_t full0 = smem_u32(&ctl->full[0]), empty0 = smem_u32(&ctl->empty[0]), ring0 = smem_u32(ring);

    if (warp == 0) {
        // ---------------- producer ----------------
        if (elect_one()) {
            const uint32_t lead_full = PAIR ? map_to_cta(&ctl->full[0], 0) : full0;
            RingPos r;
            r.start(ring0, (uint32_t)a.stages);
            bool ok = true, there;
            for (int item = first; item < n_items && ok; item += step) {
                const int group = item / a.NB, row = tile_of(group, &there) * kTileM, col = (item - group * a.NB) * a.BN + rank * (a.BN / 2);
                for (int kc = 0; kc < a.kchunks; ++kc) {
                    ok = wait_at(empty0 + r.off, r.phase ^ 1u, ctl, status);
                    if (!ok) break;
                    if (PAIR) {
                        if (rank == 0) mbar_expect_tx(full0 + r.off, 2u * (uint32_t)a.stage_bytes);
                        load_pair(r.data, &tmA, kc * kBytesK, row, lead_full + r.off);
                        load_pair(r.data + kATile, &tmB, kc * kBytesK, col, lead_full + r.off);
                    } else {
                        mbar_expect_tx(full0 + r.off, (uint32_t)a.stage_bytes);
                        tma_load_2d(r.data, &tmA, kc * kBytesK, row, full0 + r.off);
                        tma_load_2d(r.data + kATile, &tmB, kc * kBytesK, col, full0 + r.off);
                    }
                    r.next(ring0, (uint32_t)a.stages, (uint32_t)a.stage_bytes);
                }
            }
            // on an abort: give the copies already issued a bounded chance to land before the CTA exits
            if (!ok) { const unsigned long long t0 = now_ns(); while (now_ns() - t0 < 2000000ull) { } }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---------------- MMA issuer (of a pair: the leader's, for both CTAs) ----------------
        if (rank == 0 && elect_one()) {
            const uint64_t dconst = umma_desc(0, 1024, 2);
            const uint32_t d_hi = (uint32_t)(dconst >> 32), r0 = (uint32_t)dconst + (ring0 >> 4), slot = (uint32_t)a.stage_bytes >> 4;
            RingPos r;
            r.start(r0, (uint32_t)a.stages);
            uint32_t acc = 0, acc_ph = 0;
            bool ok = true;
            for (int item = first; item < n_items && ok; item += step) {
                const uint32_t d = tmem_base + acc * (uint32_t)a.BN;
                ok = wait_at(smem_u32(&ctl->tmem_empty[acc]), acc_ph ^ 1u, ctl, status);
                tc_fence_after();
                for (int kc = 0; kc < a.kchunks && ok; ++kc) {
                    ok = wait_at(full0 + r.off, r.phase, ctl, status);
                    if (!ok) break;
                    tc_fence_after();
                    const int n = kc + 1 < a.kchunks ? 4 : a.k_last;
                    if (PAIR) { umma_i8_pair(d, r.data, r.data + (kATile >> 4), d_hi, a.idesc, kc != 0, n); commit_pair(empty0 + r.off); }
                    else { umma_i8(d, r.data, r.data + (kATile >> 4), d_hi, a.idesc, kc != 0, n); umma_commit_at(empty0 + r.off); }
                    r.next(r0, (uint32_t)a.stages, slot);
                }
                if (ok) { if (PAIR) commit_pair(smem_u32(&ctl->tmem_full[acc])); else umma_commit(&ctl->tmem_full[acc]); }
                if (++acc == 2u) { acc = 0; acc_ph ^= 1u; }
            }
        }
        __syncwarp();
    } else {
        // ---------------- scales, bias, ReLU, rounding, store ----------------
        // A warp has 32 rows (the quadrant of tensor memory that it may read) and of their columns 32 at a time: of the four warps with the same
        // rows each every fourth.  A lane holds two neighbouring columns of four rows in each group of eight columns, so that it needs the scales and
        // biases of a quarter of the columns: with a row per lane every lane needed all of them, and reading those from shared memory took
        // more of its bandwidth than the operands.  Where out takes 16-byte stores the warp turns its rows through shared memory and they leave
        // as boxes of 32 rows x 64 bytes by TMA: 25088 x 512 x 2048 to bf16 in 28.6 us, 3.6 TB/s written (to float32 41, 5.0); before the
        // instructions were cut 30.6, and then with the lanes' own stores of 64 bytes of a row 40.0, of 128 bytes 45.1.
        const int q = warp & 3, part = (warp - 2) >> 2;
        uint32_t stage = smem_u32(staging) + (uint32_t)(warp - 2) * kStage;
        const uint32_t to_stage = (lane & 7) * 64 + (((lane >> 3) ^ ((lane >> 1) & 3)) << 4);           // + 512 per eight rows
        const uint32_t both = a.bufs == 2 ? stage ^ (stage + kEpiWarps * kStage) : 0;                   // from one place to the other
        const uint32_t lead_empty = PAIR ? map_to_cta(&ctl->tmem_empty[0], 0) : 0;
        const bool pairs = (((uintptr_t)p.b_scale | (uintptr_t)p.bias) & 7) == 0;
        uint32_t acc = 0, acc_ph = 0;
        bool ok = true, there;
        auto row_scales = [&](int tile, float* s) {
            const int64_t r = (int64_t)tile * kTileM + q * 32 + (lane >> 2);
#pragma unroll
            for (int k = 0; k < 4; ++k) s[k] = r + 8 * k < p.m ? p.a_scale[r + 8 * k] : 0.f;
        };
        auto stage_bf16 = [&](const uint32_t (&v)[2][16], const float* sa, const float2* s, const float2* b) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint32_t w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = two_bf16<RELU>(finish2(v[k >> 1][4 * j + 2 * (k & 1)], v[k >> 1][4 * j + 2 * (k & 1) + 1], sa[k], s[j], b[j]));
                stmatrix4(stage + to_stage + k * 512, w[0], w[1], w[2], w[3]);
            }
        };
        auto stage_f32 = [&](const uint32_t (&v)[2][16], const float* sa, const float2* s, const float2* b, int h) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int j = 2 * h; j < 2 * h + 2; ++j) {
                    const float2 f = finish2(v[k >> 1][4 * j + 2 * (k & 1)], v[k >> 1][4 * j + 2 * (k & 1) + 1], sa[k], s[j], b[j]);
                    const int r = 8 * k + (lane >> 2), u = 2 * (j & 1) + ((lane >> 1) & 1);
                    asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(stage + r * 64 + ((u ^ ((r >> 1) & 3)) << 4) + 8 * (lane & 1)), "f"(clamped<RELU>(f.x)),
                                 "f"(clamped<RELU>(f.y)) : "memory");
                }
        };
        float next[4];
        if (first < n_items) row_scales(tile_of(first / a.NB, &there), next);
        for (int item = first; item < n_items; item += step) {
            const int group = item / a.NB, tile = tile_of(group, &there), n0 = (item - group * a.NB) * a.BN;
            const int64_t row0 = (int64_t)tile * kTileM + q * 32;                                  // of a
            const int rows = LIST ? 32 : there ? (int)max((int64_t)0, min((int64_t)32, p.m - row0)) : 0;   // that exist (LIST: where `mine` says so)
            const int64_t mine = LIST ? (there ? out_row(p, tile, q * 32 + lane) : -1) : 0;        // row `lane` in out
            float sa[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) sa[k] = next[k];
            bool later;
            if (item + step < n_items) row_scales(tile_of((item + step) / a.NB, &later), next);      // on their way meanwhile
            if (ok) ok = wait_at(smem_u32(&ctl->tmem_full[acc]), acc_ph, ctl, status);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) sa[0] = sa[1] = sa[2] = sa[3] = __uint_as_float(0x7fffffffu);                 // a wait ran out: what is stored says so
            tc_fence_after();
            const uint32_t from = tmem_base + acc * (uint32_t)a.BN + ((uint32_t)(q * 32) << 16);
            const int n_here = min(a.BN, p.n - n0);
            bool held = true;                                 // the accumulator is still to be read
            auto hand_back = [&]() {
                tc_fence_before();
                __syncwarp();
                if (lane == 0 && ok) {                        // (a warp whose wait ran out has read nothing; what others still read stays)
                    if (PAIR) asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(lead_empty + 8u * acc) : "memory");
                    else mbar_arrive_relaxed(&ctl->tmem_empty[acc]);
                }
                held = false;
            };
            for (int c0 = part * 32; c0 < n_here; c0 += 4 * 32) {
                uint32_t v[2][16];
                tmem_ld_16x32(from + c0, v[0]);
                tmem_ld_16x32(from + (16u << 16) + c0, v[1]);
                float2 s[4], b[4];
                column_weights(p, n0 + c0 + 2 * (lane & 3), pairs && c0 + 32 <= n_here, s, b);
                tmem_ld_wait();
                if (c0 + 4 * 32 >= n_here) hand_back();
                if (sizeof(T) == 4 && a.boxes) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {             // 16 columns at a time
                        if (lane == 0) store_read(a.bufs);
                        __syncwarp();
                        stage_f32(v, sa, s, b, h);
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                        if (lane == 0 && rows > 0) store_box(&tmC, stage, n0 + c0 + 16 * h, (int)row0);
                        stage ^= both;
                    }
                } else if (sizeof(T) == 2 && a.boxes) {
                    if (lane == 0) store_read(a.bufs);        // the box before has left its place
                    __syncwarp();
                    stage_bf16(v, sa, s, b);
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0 && rows > 0) store_box(&tmC, stage, n0 + c0, (int)row0);
                    stage ^= both;
                } else {
#pragma unroll
                    for (int h = 0; h < (sizeof(T) == 4 ? 2 : 1); ++h) {
                        if constexpr (sizeof(T) == 2) stage_bf16(v, sa, s, b); else stage_f32(v, sa, s, b, h);
                        __syncwarp();
                        const int c1 = n0 + c0 + 16 * h;
                        if (a.wide && c1 + 64 / (int)sizeof(T) <= p.n) {      // four lanes to 64 bytes
                            const int u = lane & 3;
#pragma unroll
                            for (int it = 0; it < 4; ++it) {
                                const int r = it * 8 + (lane >> 2);
                                const int64_t to = LIST ? __shfl_sync(0xffffffffu, mine, r) : r < rows ? row0 + r : -1;
                                if (to >= 0) *(uint4*)((char*)p.out + (size_t)to * p.out_pitch + (size_t)c1 * sizeof(T) + u * 16) = lds128(stage + r * 64 + ((u ^ ((r >> 1) & 3)) << 4));
                            }
                        } else {                              // an element per lane, side by side
                            constexpr int PER = sizeof(T) == 4 ? 2 : 1;       // rows at once
                            const int e = lane & (32 / PER - 1), u = e * (int)sizeof(T) >> 4;
#pragma unroll 4
                            for (int it = 0; it < 32 / PER; ++it) {
                                const int r = it * PER + (PER == 2 ? lane >> 4 : 0);
                                const int64_t to = LIST ? __shfl_sync(0xffffffffu, mine, r) : r < rows ? row0 + r : -1;
                                const uint32_t at = stage + r * 64 + ((u ^ ((r >> 1) & 3)) << 4) + (e * (int)sizeof(T) & 15);
                                if (to >= 0 && c1 + e < p.n) {
                                    T* const out = (T*)((char*)p.out + (size_t)to * p.out_pitch) + c1 + e;
                                    if constexpr (sizeof(T) == 4) { uint32_t w; asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(at) : "memory"); *(uint32_t*)out = w; }
                                    else { uint16_t w; asm volatile("ld.shared.b16 %0, [%1];" : "=h"(w) : "r"(at) : "memory"); *(uint16_t*)out = w; }
                                }
                            }
                        }
                        __syncwarp();
                    }
                }
            }
            if (held) hand_back();                            // a warp whose columns do not exist
            if (++acc == 2u) { acc = 0; acc_ph ^= 1u; }
        }
        if (a.boxes && lane == 0) store_done();
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();                             // neither CTA frees tensor memory or leaves while the other may still use it
    if (warp == 1) {
        tc_fence_after();
        if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(a.tmem_cols) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(a.tmem_cols) : "memory");
    }
}

// Few tiles: the reduction of 128 output channels x up to 128 rows split over a cluster of CTAs, as in dc_conv_cluster.cu.  What bounds such
// products are the weights, each read once, so the weights are the side of 128 rows (tensor memory's lanes), the rows of x (16 to 128 of them) its columns, and the split
// makes enough CTAs for the weights to stream at HBM's rate.  Each CTA takes its part of K; the int32 sums meet in distributed shared memory, where CTA r
// finishes channels r * 128 / CS and on; they are exact, so the split changes no bit.  `early`: everything older than the kernel before is
// complete (dc_linear_quantized: that kernel puts x into 8 bits), so the weights' loads start before the wait for it.
// With the rows put into 8 bits, us, in turns with k_product's 64 CTAs that walk K alone: 1 x 9216 x 4096 11.3 and 27.7, 32 x 25088 x 4096 23.1
// and 45.9, 100 x 4096 x 1000 7.6 and 11.3; 196 x 1024 x 512 7.2 and 6.1.
constexpr int kSplitThreads = 192, kSplitStages = 12;
// A CTA of it waits for its cluster, and tensor memory is given out without a limit on the wait.  So it may not share an SM with a kernel of another stream that takes all 512
// columns and waits for other CTAs too (the convolutions on CTA pairs, which leave up to 48 KB of shared memory): each could hold what the other's
// cluster is waiting for.  It takes at least this much; what fits beside it then, and it itself twice or three times, have columns for all.
constexpr size_t kSplitLeast = 64 * 1024;
struct SplitArgs {
    dc_product_args p;
    int NT, CS, stages, stage_bytes, kchunks, k_last, m_tiles, early;     // NT: rows of x in a tile
    uint32_t idesc, tmem_cols;
};
struct SplitCtl {
    unsigned long long full[kSplitStages], empty[kSplitStages], done;
    alignas(16) float scale[128];
    uint32_t tmem_base;
    volatile int abort_flag;
    unsigned long long wait_ns;
};

template <typename T>
__global__ void __launch_bounds__(kSplitThreads, 1) k_product_split(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const SplitArgs a)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* ring = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    // [CS][NT / 4][128 / CS]: this CTA's channels, four rows' sums each, from every CTA; a warp's stores lie side by side
    int4* red = (int4*)(ring + (size_t)a.stages * a.stage_bytes);
    SplitCtl* ctl = (SplitCtl*)(red + 32 * a.NT);
    const dc_product_args& p = a.p;
    int32_t* const status = p.status ? p.status : &g_status;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int rank = (int)cluster_rank(), item = blockIdx.x / a.CS, mt = item % a.m_tiles, nt = item / a.m_tiles;
    const int nk = (a.kchunks - rank + a.CS - 1) / a.CS;         // chunk it * CS + rank: a cluster reads whole stretches of a row at once

    if (threadIdx.x == 0) {
        for (int i = 0; i < a.stages; ++i) { mbar_init(&ctl->full[i], 2); mbar_init(&ctl->empty[i], 1); }   // weights and rows arrive apart
        mbar_init(&ctl->done, 1);
        ctl->abort_flag = 0;
        ctl->wait_ns = kWaitNs;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmW) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmX) : "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(a.tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");    // waited for before another CTA's shared memory is written
    tc_fence_after();
    const uint32_t tmem_base = ctl->tmem_base;
    const uint32_t full0 = smem_u32(&ctl->full[0]), empty0 = smem_u32(&ctl->empty[0]), ring0 = smem_u32(ring);
    const int ahead = nk < a.stages ? nk : a.stages;
    auto load_weights = [&](int it, uint32_t off, uint32_t slot) {
        mbar_expect_tx(full0 + off, (uint32_t)kATile);
        tma_load_2d(slot, &tmW, (it * a.CS + rank) * kBytesK, nt * kTileM, full0 + off);
    };
    if (!a.early) { dc_pdl_wait(); dc_pdl_release(); }
    if (warp == 0 && elect_one())
        for (int it = 0; it < ahead; ++it) load_weights(it, 8u * it, ring0 + it * a.stage_bytes);
    __syncwarp();
    if (a.early) { dc_pdl_wait(); dc_pdl_release(); }

    bool waited = false;                                                     // for the cluster
    // the channel that this thread finishes: the threads are a multiple of a CTA's channels
    const int rows = 128 / a.CS, ch = threadIdx.x % rows, j = nt * kTileM + rank * rows + ch;
    const float sb = j < p.n ? dc_ld(p.b_scale + j) : 0.f, bias = j < p.n && p.bias ? dc_ld(p.bias + j) : 0.f;
    if (warp == 0) {
        // ---------------- producer ----------------
        if (elect_one()) {
            RingPos r;
            r.start(ring0, (uint32_t)a.stages);
            bool ok = true;
            for (int it = 0; it < nk; ++it) {
                if (it >= a.stages) {
                    ok = mbar_wait_at(empty0 + r.off, r.phase ^ 1u, &ctl->abort_flag, &ctl->wait_ns, status);
                    if (!ok) break;
                    load_weights(it, r.off, r.data);
                }
                mbar_expect_tx(full0 + r.off, (uint32_t)(a.NT * kBytesK));
                tma_load_2d(r.data + kATile, &tmX, (it * a.CS + rank) * kBytesK, mt * a.NT, full0 + r.off);
                r.next(ring0, (uint32_t)a.stages, (uint32_t)a.stage_bytes);
            }
            if (!ok) { const unsigned long long t0 = now_ns(); while (now_ns() - t0 < 2000000ull) { } }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        if (elect_one()) {
            const uint64_t dconst = umma_desc(0, 1024, 2);
            const uint32_t d_hi = (uint32_t)(dconst >> 32), r0 = (uint32_t)dconst + (ring0 >> 4), slot = (uint32_t)a.stage_bytes >> 4;
            RingPos r;
            r.start(r0, (uint32_t)a.stages);
            for (int it = 0; it < nk; ++it) {
                if (!mbar_wait_at(full0 + r.off, r.phase, &ctl->abort_flag, &ctl->wait_ns, status)) break;
                tc_fence_after();
                umma_i8(tmem_base, r.data, r.data + (kATile >> 4), d_hi, a.idesc, it != 0, it * a.CS + rank + 1 < a.kchunks ? 4 : a.k_last);
                if (it + a.stages < nk) umma_commit_at(empty0 + r.off);
                if (it + 1 == nk) umma_commit(&ctl->done);
                r.next(r0, (uint32_t)a.stages, slot);
            }
        }
        __syncwarp();
    } else {
        // ---------------- partial sums to the CTA that finishes the channel ----------------
        const int q = warp & 3, m = q * 32 + lane, owner = m / rows;
        if (m < a.NT) ctl->scale[m] = (int64_t)mt * a.NT + m < p.m ? p.a_scale[(int64_t)mt * a.NT + m] : 0.f;
        const uint32_t dst = map_to_cta(red + rank * (a.NT / 4) * rows + m - owner * rows, (uint32_t)owner);
        bool ok = mbar_wait_at(smem_u32(&ctl->done), 0, &ctl->abort_flag, &ctl->wait_ns, status);
        ok = __all_sync(0xffffffffu, ok);
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        waited = true;
        if (ok) {
            tc_fence_after();
            const int there = (int)min((int64_t)a.NT, p.m - (int64_t)mt * a.NT);
            for (int c = 0; c < a.NT && c < there; c += 16) {
                uint32_t v[16];
                asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                             : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
                               "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                             : "r"(tmem_base + ((uint32_t)(q * 32) << 16) + c) : "memory");
                tmem_ld_wait();
#pragma unroll
                for (int k = 0; k < 16; k += 4)
                    if (c + k < there)
                        asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + (uint32_t)((c + k) / 4 * rows * 16)), "r"(v[k]), "r"(v[k + 1]), "r"(v[k + 2]), "r"(v[k + 3]) : "memory");
            }
        }
        tc_fence_before();
    }
    if (!waited) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    // a CTA that gave up has not sent its sums: every CTA of the cluster hears of it
    if (ctl->abort_flag != 0)
        for (int r = 0; r < a.CS; ++r)
            asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(map_to_cta((const void*)&ctl->abort_flag, (uint32_t)r)), "r"(1) : "memory");
    cluster_sync_all();                      // this CTA's channels have arrived from every CTA
    {
        // ---------------- this CTA's channels: sums from all ranks, scales, bias, ReLU, rounding, store ----------------
        const int there = (int)min((int64_t)a.NT, p.m - (int64_t)mt * a.NT);
        const bool dead = ctl->abort_flag != 0;                              // what is stored says so
        for (int t = threadIdx.x / rows * 4; t < there && j < p.n; t += kSplitThreads / rows * 4) {    // four rows of x
            int4 sum = make_int4(0, 0, 0, 0);
            for (int r = 0; r < a.CS; ++r) {
                const int4 v = red[(r * (a.NT / 4) + t / 4) * rows + ch];
                sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
            }
            const int32_t sums[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (t + k >= there) break;
                const int64_t row = (int64_t)mt * a.NT + t + k;
                float f = fmaf((float)sums[k] * (dead ? __uint_as_float(0x7fffffffu) : ctl->scale[t + k]), sb, bias);
                if (p.relu) f = clamped<true>(f);
                T* const out = (T*)((char*)p.out + (size_t)row * p.out_pitch) + j;
                if constexpr (sizeof(T) == 4) *out = f;
                else *out = __float2bfloat16_rn(f);
            }
        }
    }
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(a.tmem_cols) : "memory");
    }
}

template <bool PAIR, bool LIST, bool RELU, typename T>
int launch_product(const CUtensorMap& tmA, const CUtensorMap& tmB, const CUtensorMap& tmC, const ProductArgs& a, int ctas, int device, cudaStream_t stream)
{
    static dc_once_per_device attr_set;
    DC_CUDA(attr_set.ensure(device, [] { return cudaFuncSetAttribute(k_product<PAIR, LIST, RELU, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem); }));
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = PAIR ? 2 : 1; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = kSmem; cfg.stream = stream;
    // g_dc_pdl off: see dc_launch_pdl
    cfg.attrs = g_dc_pdl ? attr : attr + 1; cfg.numAttrs = g_dc_pdl ? 2 : 1;
    DC_CUDA(cudaLaunchKernelEx(&cfg, k_product<PAIR, LIST, RELU, T>, tmA, tmB, tmC, a));
    return DC_OK;
}

// Clusters of so many CTAs, each with an SM of its own, that the device holds at once.
int clusters_at_once(int cs, int device)
{
    static std::atomic<int> known[64][4];
    const int at = cs == 1 ? 0 : cs == 2 ? 1 : cs == 4 ? 2 : 3;
    if (device >= 0 && device < 64)
        if (const int n = known[device][at].load(std::memory_order_relaxed)) return n;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cs; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)cs); cfg.blockDim = dim3(kSplitThreads); cfg.dynamicSmemBytes = 200 * 1024; cfg.attrs = attr; cfg.numAttrs = 1;
    int n = 0;
    if (cudaFuncSetAttribute(k_product_split<float>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, k_product_split<float>, &cfg) != cudaSuccess) { cudaGetLastError(); n = 0; }
    if (n < 1) n = 1;
    if (device >= 0 && device < 64) known[device][at].store(n, std::memory_order_relaxed);
    return n;
}

// How a product of few tiles is split, and the cycles that it takes (as dc_launch_product counts them).
struct SplitPlan { int NT, CS; double cost; };
SplitPlan split_plan(const dc_product_args& p, int kc, int device)
{
    SplitPlan best = {};
    const int NT = p.m <= 16 ? 16 : p.m <= 32 ? 32 : p.m <= 64 ? 64 : 128;
    const long long tiles = (p.m + NT - 1) / NT * (long long)dc_div_up(p.n, kTileM);
    for (int cs = 2; cs <= 8 && cs <= kc; cs *= 2) {
        const int at_once = clusters_at_once(cs, device);
        const long long rounds = (tiles + at_once - 1) / at_once;
        // HBM's 3400 bytes a cycle shared by the CTAs; to send the sums, join and store them
        const double load = (kATile + NT * kBytesK) / 50.0, hbm = kATile * (double)(tiles * cs < at_once * cs ? tiles * cs : at_once * cs) / 3400.0;
        const double join = 2500.0 + NT * (cs == 8 ? 30.0 : cs == 4 ? 40.0 : 50.0);
        const double cost = rounds * (dc_div_up(kc, cs) * (load > hbm ? load : hbm) + join);
        if (rounds <= 2 && (best.CS == 0 || cost < best.cost)) best = {NT, cs, cost};
    }
    return best;
}

template <typename T>
int launch_split(const dc_product_args& p, const SplitPlan& s, int kc, int device, cudaStream_t stream)
{
    SplitArgs a = {};
    a.p = p; a.NT = s.NT; a.CS = s.CS; a.kchunks = kc; a.k_last = dc_div_up(p.k - (kc - 1) * kBytesK, 32); a.early = p.early;
    a.m_tiles = (int)((p.m + s.NT - 1) / s.NT);
    a.stage_bytes = kATile + s.NT * kBytesK;
    const int red = 128 * s.NT * 4, fixed = red + (int)sizeof(SplitCtl) + 1024, room = (227 * 1024 - fixed) / a.stage_bytes, most = dc_div_up(kc, s.CS);
    a.stages = room < kSplitStages ? room : kSplitStages;
    if (a.stages > most) a.stages = most;
    a.idesc = (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(s.NT >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
    a.tmem_cols = s.NT < 32 ? 32u : (uint32_t)s.NT;
    CUtensorMap tmW, tmX;
    if (!encode_rows(&tmW, p.b, p.b_pitch, p.n, p.k, kTileM) || !encode_rows(&tmX, p.a, p.a_pitch, p.m, p.k, s.NT)) return DC_ERR_CUDA;
    static dc_once_per_device attr_set;
    DC_CUDA(attr_set.ensure(device, [] { return cudaFuncSetAttribute(k_product_split<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024); }));
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)s.CS; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.m_tiles * dc_div_up(p.n, kTileM) * s.CS)); cfg.blockDim = dim3(kSplitThreads);
    const size_t smem = (size_t)a.stages * a.stage_bytes + fixed;
    cfg.dynamicSmemBytes = smem > kSplitLeast ? smem : kSplitLeast; cfg.stream = stream;
    cfg.attrs = attr; cfg.numAttrs = g_dc_pdl ? 2 : 1;
    DC_CUDA(cudaLaunchKernelEx(&cfg, k_product_split<T>, tmW, tmX, a));
    return DC_OK;
}

}  // namespace

int dc_launch_product(const dc_product_args& p, int dtype, int device, int num_sms, cudaStream_t stream)
{
    if (p.m <= 0) return DC_OK;
    ProductArgs a = {};
    a.p = p;
    a.m_tiles = (int)((p.m + kTileM - 1) / kTileM);
    const long long tiles = p.tile_list ? p.max_tiles : a.m_tiles;
    // The tile that takes the fewest cycles, as counted from measurements: operands arrive at about 50 bytes a cycle, an SM's share of out leaves
    // at about 24 where others pause, and an item costs 500 to begin and end.
    const int elt = dtype == DC_BF16 ? 2 : 4, kc = dc_div_up(p.k, kBytesK);
    bool pair = false;
    double best = 0.0;
    for (int c = 0; c < 4; ++c) {
        const bool two = c < 2;
        const int bn = c == 0 ? 256 : c == 3 ? 64 : 128;
        const long long n_items = (two ? (tiles + 1) / 2 : tiles) * dc_div_up(p.n, bn), at_once = two ? num_sms / 2 : num_sms, rounds = (n_items + at_once - 1) / at_once;
        const double load = kc * (double)(kATile + (two ? bn / 2 : bn) * kBytesK) / 50.0, mma = kc * 2.0 * bn, out = 128.0 * bn * elt / 24.0;
        const double cost = rounds * ((load > mma ? load : mma) + out + 500.0);
        if (c == 0 || cost < best) { best = cost; pair = two; a.BN = bn; }
    }
    if (!p.padded && p.n <= (1 << 20) && p.m <= (1 << 20)) {
        const SplitPlan s = split_plan(p, kc, device);
        if (s.CS > 1 && s.cost < best) return dtype == DC_BF16 ? launch_split<__nv_bfloat16>(p, s, kc, device, stream) : launch_split<float>(p, s, kc, device, stream);
    }
    a.NB = dc_div_up(p.n, a.BN);
    const int b_rows = pair ? a.BN / 2 : a.BN;
    a.stage_bytes = kATile + b_rows * kBytesK;
    a.bufs = kc <= 8 ? 2 : 1;                                 // long products take the room for operands
    a.stages = (kRoom - kEpiWarps * kStage * a.bufs) / a.stage_bytes;
    if (a.stages > kMaxStages) a.stages = kMaxStages;
    a.kchunks = kc;
    a.k_last = dc_div_up(p.k - (a.kchunks - 1) * kBytesK, 32);
    // int32 accumulators, both operands signed 8-bit integers, K-major
    a.idesc = (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(a.BN >> 3) << 17) | ((uint32_t)((pair ? 256 : 128) >> 4) << 24);
    a.tmem_cols = (uint32_t)(2 * a.BN);
    a.wide = (uintptr_t)p.out % 16 == 0 && p.out_pitch % 16 == 0;
    CUtensorMap tmA, tmB, tmC = {};
    if (!encode_rows(&tmA, p.a, p.a_pitch, p.m, p.k, kTileM) || !encode_rows(&tmB, p.b, p.b_pitch, p.n, p.k, b_rows)) return DC_ERR_CUDA;
    // (a box is cut at whole 16 bytes, not at the row's last column)
    if (a.wide && !p.padded && (size_t)p.n * elt % 16 == 0) a.boxes = encode_out(&tmC, p.out, p.out_pitch, p.m, p.n, elt);
    const long long items = (pair ? (tiles + 1) / 2 : tiles) * a.NB, cap = pair ? num_sms / 2 : num_sms;
    if (items >= 0x70000000) return DC_ERR_LIMIT;
    const int ctas = (int)(items < cap ? items : cap) * (pair ? 2 : 1);
#define DC_PRODUCT(PAIR, LIST, RELU, T) return launch_product<PAIR, LIST, RELU, T>(tmA, tmB, tmC, a, ctas, device, stream)
#define DC_PRODUCT_OF(LIST, RELU, T) do { if (pair) DC_PRODUCT(true, LIST, RELU, T); DC_PRODUCT(false, LIST, RELU, T); } while (0)
#define DC_PRODUCT_TO(T) do { if (p.padded) { if (p.relu) DC_PRODUCT_OF(true, true, T); DC_PRODUCT_OF(true, false, T); } if (p.relu) DC_PRODUCT_OF(false, true, T); DC_PRODUCT_OF(false, false, T); } while (0)
    if (dtype == DC_BF16) DC_PRODUCT_TO(__nv_bfloat16);
    DC_PRODUCT_TO(float);
#undef DC_PRODUCT_TO
#undef DC_PRODUCT_OF
#undef DC_PRODUCT
}

constexpr int kMostTerms = 131071;

// What both products ask of their operands.
static int product_check(const int8_t* b, size_t b_pitch, const float* b_scale, const float* bias, int64_t m, int32_t n, int32_t k, int32_t dtype, const void* out, size_t out_pitch)
{
    if (dtype != DC_FP32 && dtype != DC_BF16) return DC_ERR_CONFIG;
    const int elt = dtype == DC_BF16 ? 2 : 4;
    if (m < 0 || n < 1 || k < 1) return DC_ERR_ARG;
    if (k > kMostTerms || m > DC_MOST_ROWS || n > (1 << 28) || (n > 1 && b_pitch > kMostPitch)) return DC_ERR_LIMIT;
    if (m == 0) return DC_OK;
    if (!b || !b_scale || !out || (uintptr_t)b % 16 || b_pitch % 16 || (n > 1 && b_pitch < (size_t)k)) return DC_ERR_ARG;
    if ((uintptr_t)b_scale % 4 || (uintptr_t)bias % 4 || (uintptr_t)out % elt || out_pitch % elt || (m > 1 && out_pitch < (size_t)n * elt)) return DC_ERR_ARG;
    return DC_OK;
}

// Do the rows of two maps share no memory?  (false too where that is not seen at once: stretches that cross, of different pitches.)
static bool rows_apart(uintptr_t a, size_t a_pitch, size_t a_row, uintptr_t b, size_t b_pitch, size_t b_row, int64_t rows)
{
    const size_t before = (size_t)(rows - 1);
    if (b >= a + before * a_pitch + a_row || a >= b + before * b_pitch + b_row) return true;
    if (a_pitch != b_pitch || rows < 2) return false;
    const size_t d = b >= a ? (b - a) % a_pitch : (a_pitch - (a - b) % a_pitch) % a_pitch;      // columns of one buffer
    return d >= a_row && d + b_row <= a_pitch;
}

extern "C" {

int dc_matmul_quantized(const int8_t* a_dev, size_t a_pitch, const float* a_scale_dev, const int8_t* b_dev, size_t b_pitch, const float* b_scale_dev, const float* bias_dev,
                        int64_t m, int32_t n, int32_t k, int32_t relu, int32_t dtype, void* out_dev, size_t out_pitch, void* cuda_stream)
{
    int rc = product_check(b_dev, b_pitch, b_scale_dev, bias_dev, m, n, k, dtype, out_dev, out_pitch);
    if (rc != DC_OK || m == 0) return rc;
    if (m > 1 && a_pitch > kMostPitch) return DC_ERR_LIMIT;
    if (!a_dev || !a_scale_dev || (uintptr_t)a_dev % 16 || a_pitch % 16 || (m > 1 && a_pitch < (size_t)k) || (uintptr_t)a_scale_dev % 4) return DC_ERR_ARG;
    int device = 0, sms = 0;
    if ((rc = dc_current_device(&device, &sms)) != DC_OK) return rc;
    dc_product_args p = {};
    p.a = a_dev; p.a_pitch = a_pitch; p.a_scale = a_scale_dev; p.b = b_dev; p.b_pitch = b_pitch; p.b_scale = b_scale_dev; p.bias = bias_dev;
    p.m = m; p.n = n; p.k = k; p.relu = relu; p.out = out_dev; p.out_pitch = out_pitch;
    return dc_launch_product(p, dtype, device, sms, (cudaStream_t)cuda_stream);
}

int dc_linear_workspace(int64_t m, int32_t k, size_t* bytes)
{
    if (m < 0 || k < 1 || !bytes) return DC_ERR_ARG;
    *bytes = (size_t)m * (dc_quant_pitch(k) + sizeof(float)) + 256;
    return DC_OK;
}

int dc_linear_quantized(const void* x_dev, size_t x_pitch, const int8_t* w_dev, size_t w_pitch, const float* w_scale_dev, const float* bias_dev, int64_t m, int32_t n, int32_t k,
                        int32_t relu, int32_t dtype, void* out_dev, size_t out_pitch, void* workspace_dev, size_t workspace_bytes, void* cuda_stream)
{
    int rc = product_check(w_dev, w_pitch, w_scale_dev, bias_dev, m, n, k, dtype, out_dev, out_pitch);
    if (rc != DC_OK || m == 0) return rc;
    const int elt = dtype == DC_BF16 ? 2 : 4;
    size_t need = 0;
    dc_linear_workspace(m, k, &need);
    if (m > 1 && x_pitch > 0xffffffffu) return DC_ERR_LIMIT;
    if (!x_dev || (uintptr_t)x_dev % elt || x_pitch % elt || (m > 1 && x_pitch < (size_t)k * elt) || !workspace_dev || workspace_bytes < need) return DC_ERR_ARG;
    int device = 0, sms = 0;
    if ((rc = dc_current_device(&device, &sms)) != DC_OK) return rc;
    dc_product_args p = {};
    p.b = w_dev; p.b_pitch = w_pitch; p.b_scale = w_scale_dev; p.bias = bias_dev;
    p.m = m; p.n = n; p.k = k; p.relu = relu; p.out = out_dev; p.out_pitch = out_pitch;
    // one launch writes out while other CTAs still read x: where they may share memory, x is put into the workspace first
    if (dc_few_pays(m, n, k) && rows_apart((uintptr_t)x_dev, x_pitch, (size_t)k * elt, (uintptr_t)out_dev, out_pitch, (size_t)n * elt, m)) return dc_launch_few(p, x_dev, x_pitch, dtype, device, sms, (cudaStream_t)cuda_stream);
    const size_t pitch = dc_quant_pitch(k);
    int8_t* const q = (int8_t*)(((uintptr_t)workspace_dev + 255) & ~(uintptr_t)255);
    float* const scale = (float*)(q + (size_t)m * pitch);
    dc_rows_args r = {};
    r.x = x_dev; r.x_pitch = x_pitch; r.rows = m; r.channels = k; r.q = q; r.q_pitch = pitch; r.scale = scale;
    if ((rc = dc_launch_rows(r, false, dtype, sms, (cudaStream_t)cuda_stream)) != DC_OK) return rc;
    p.a = q; p.a_pitch = pitch; p.a_scale = scale; p.early = 1;
    return dc_launch_product(p, dtype, device, sms, (cudaStream_t)cuda_stream);
}

}  // extern "C"
