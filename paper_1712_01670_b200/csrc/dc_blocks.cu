// Rows in 8-bit floating point (e4m3) with a scale for each block of 128 values, and their products.
//
//   scale = the smallest power of two with max |x| <= 448 scale,  q = e4m3(x / scale)
//   out[r][j] = relu(sum_i a_scale[r][i] b_scale[j'][i] sum_{k in block i} a[r][k] b[j][k] + bias[j])
//
// Rows in 8 bits: memory bounds them: a value is read once (turned ones of small maps twice) and leaves in its row, turned, or both.  A power of two as scale costs a floating-point format no
// precision, and makes x / scale exact: one rounding, and the same bits whichever kernel, row or column works it out.
//
// Products: tcgen05.mma kind::f8f6f4 on tiles of 128 rows, operands by TMA in 128-byte swizzled rows of 128 values, which are one block.  A block's sums leave
// tensor memory as soon as they are there, are scaled and added up in the registers of sixteen warps, beside the MMAs of the next blocks (two to four accumulators in turns).  The scales
// are any floats, so they cannot be left to the MMA, which takes powers of two.  8192 x 4096 x 4096 to bf16 125 us, 2.2 PFLOP/s at 1.6 GHz: tensor pipe 58 % busy, instruction issue 63 %;
// the same product of 8-bit integers, whose sums stay in tensor memory, 86.
//   k_blocks        256 x 256 (CTA pairs) to 128 x 64 tiles
//   k_blocks_split  few tiles: the blocks of K dealt to a cluster
#include "dc_product.cuh"
#include "dc_quantise.cuh"

namespace {

// ---------------------------------------------------------------------------
// rows in 8 bits
// ---------------------------------------------------------------------------
struct BlocksArgs {
    const void* x; size_t x_pitch;
    int rows, channels, kb, rb;                               // kb, rb: blocks of 128 columns, of 128 rows
    uint8_t* q; size_t q_pitch; float* scale;                 // or NULL
    uint8_t* qt; size_t qt_pitch; float* scale_t;             // or NULL
    int block_rows;
};

// What the bits of a block's largest size say: its scale and 1 / scale, both powers of two, so x / scale is exact.  448 = 1.75 * 2^8: with most = 1.f * 2^e the scale is
// 2^(e - 8), or twice that where 1.f > 1.75.
struct BlockScale { float scale, inv; bool bad; };
__device__ __forceinline__ BlockScale block_scale(uint32_t bits)
{
    BlockScale s;
    s.bad = bits >= 0x7f800000u;
    const int e = max((int)((bits + 0x1fffffu) >> 23) - 8, 1);
    s.scale = s.bad ? __uint_as_float(0x7fffffffu) : bits == 0 ? 0.f : __uint_as_float((uint32_t)e << 23);
    s.inv = __uint_as_float((uint32_t)(254 - e) << 23);
    return s;
}
// Two floats as e4m3, the first one in the low byte.
__device__ __forceinline__ uint32_t two_e4m3(float2 v)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(r) : "f"(v.x), "f"(v.y));
    return r;
}

// Eight values of a row.
template <typename T> struct Eight;
template <> struct Eight<__nv_bfloat16> {
    uint4 raw;
    __device__ __forceinline__ void zero() { raw = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void load(const char* p) { raw = *(const uint4*)p; }
    __device__ __forceinline__ void put(int k, __nv_bfloat16 v)
    {
        uint32_t* const w = &raw.x;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i == k >> 1) w[i] |= (uint32_t)__bfloat16_as_ushort(v) << (16 * (k & 1));
    }
    __device__ __forceinline__ void open(float2* v) const { Vec<__nv_bfloat16, 8>::open(raw, v); }
    __device__ __forceinline__ uint32_t most() const { return most_of<__nv_bfloat16>(raw_most(0u, raw)); }        // the bits of the largest size; above infinity's: a NaN
    __device__ __forceinline__ void keep(uint4* p) const { p[0] = raw; }
};
template <> struct Eight<float> {
    float4 raw[2];
    __device__ __forceinline__ void zero() { raw[0] = raw[1] = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void load(const char* p) { raw[0] = *(const float4*)p; raw[1] = *(const float4*)(p + 16); }
    __device__ __forceinline__ void put(int k, float v)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i == k) (&raw[i >> 2].x)[i & 3] = v;
    }
    __device__ __forceinline__ void open(float2* v) const { Vec<float, 4>::open(raw[0], v); Vec<float, 4>::open(raw[1], v + 2); }
    __device__ __forceinline__ uint32_t most() const { return raw_most(raw_most(0u, raw[0]), raw[1]); }
    __device__ __forceinline__ void keep(uint4* p) const { ((float4*)p)[0] = raw[0]; ((float4*)p)[1] = raw[1]; }
};

__device__ __forceinline__ void store_bytes(uint8_t* p, uint2 w, int there)       // the first `there` of eight
{
    if (there >= 8) { *(uint2*)p = w; return; }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < there) p[i] = (uint8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
}
__device__ __forceinline__ void store_bytes(uint8_t* p, uint4 w, int there)       // of sixteen
{
    if (there >= 16) { *(uint4*)p = w; return; }
    if (there > 0) store_bytes(p, make_uint2(w.x, w.y), there);
    if (there > 8) store_bytes(p + 8, make_uint2(w.z, w.w), there - 8);
}
// The largest among sixteen lanes.  (A reduction of half a warp runs once for each half, behind branches.)
__device__ __forceinline__ uint32_t most_of_half(uint32_t m, int lane)
{
    const bool upper = lane & 16;
    const uint32_t a = __reduce_max_sync(0xffffffffu, upper ? 0u : m), b = __reduce_max_sync(0xffffffffu, upper ? m : 0u);
    return upper ? b : a;
}
// Eight columns of a row, `there` of which exist.  WIDE: rows are aligned to 16 bytes and of whole eights, so all of them or none.
template <bool WIDE, typename T>
__device__ __forceinline__ void load_eight(Eight<T>& v, const char* x, int there)
{
    v.zero();
    if (WIDE) { if (there > 0) v.load(x); }
    else
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < there) v.put(k, ((const T*)x)[k]);
}
template <bool WIDE>
__device__ __forceinline__ void store_eight(uint8_t* q, uint2 w, int there)
{
    if (WIDE) { if (there > 0) *(uint2*)q = w; }
    else if (there > 0) store_bytes(q, w, there);
}
template <typename T>
__device__ __forceinline__ uint2 eight_e4m3(const Eight<T>& v, const BlockScale& s)
{
    float2 f[4];
    v.open(f);
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = two_e4m3(mul2(f[k], both<float2>(s.inv)));
    const uint32_t kept = s.bad ? 0u : 0xffffffffu;
    return make_uint2(__byte_perm(w[0], w[1], 0x5410) & kept, __byte_perm(w[2], w[3], 0x5410) & kept);
}

// A tile of 128 x 128 of a map whose rows are not aligned, into shared memory: an element to a lane, side by side.  (Eight neighbours to a lane, element by element, spread each of a warp's loads over
// 512 or 1024 bytes: 25087 x 513 bf16 24.8 us, so 29.9; 4096 x 9219 with a scale for 128 rows 43.9 and 54.8.)
template <typename T>
__device__ __forceinline__ void stage_tile(const BlocksArgs& a, int row0, int col0, T* tile)
{
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (int r0 = threadIdx.x >> 5; r0 < 128; r0 += 32) {     // four rows of a warp at once
        T v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int row = row0 + r0 + i / 4 * 8, col = col0 + i % 4 * 32 + lane;
            v[i] = row < a.rows && col < a.channels ? ((const T*)((const char*)a.x + (size_t)row * a.x_pitch))[col] : T(0.f);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) tile[(r0 + i / 4 * 8) * 128 + i % 4 * 32 + lane] = v[i];
    }
}

// Rows alone: sixteen lanes to a block of each of four rows, all four in flight.  by_kb: see divided().
__device__ __forceinline__ uint32_t divided(uint32_t n, uint2 by) { return by.x ? __umulhi(n, by.x) >> by.y : n; }

template <typename T, bool WIDE>
__device__ __forceinline__ void row_blocks(const BlocksArgs& a, uint2 by_kb, uint32_t items)
{
    const int part = threadIdx.x & 15, lane = threadIdx.x & 31;
    const uint32_t item = blockIdx.x * 16u + (threadIdx.x >> 4), fours = divided(item, by_kb), block = item - fours * (uint32_t)a.kb;
    const int row0 = (int)fours * 4, rows = item < items ? min(4, a.rows - row0) : 0, col = (int)block * 128 + part * 8, there = a.channels - col;
    const char* x = (const char*)a.x + (size_t)row0 * a.x_pitch + (size_t)col * sizeof(T);
    Eight<T> v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u, x += a.x_pitch) load_eight<WIDE>(v[u], x, u < rows ? there : 0);
    BlockScale s[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) s[u] = block_scale(most_of_half(v[u].most(), lane));
    uint8_t* q = a.q + (size_t)row0 * a.q_pitch + col;
    if (there > 0)
#pragma unroll
        for (int u = 0; u < 4; ++u, q += a.q_pitch)
            if (u < rows) store_eight<WIDE>(q, eight_e4m3(v[u], s[u]), there);
    if (part < rows) {                                        // a lane to each row's scale
        const float t = part == 0 ? s[0].scale : part == 1 ? s[1].scale : part == 2 ? s[2].scale : s[3].scale;
        a.scale[(size_t)(row0 + part) * a.kb + block] = t;
    }
}

template <typename T, bool WIDE>
__global__ void __launch_bounds__(256) k_quantize_row_blocks(const BlocksArgs a, uint2 by_kb, uint32_t items)
{
    dc_pdl_wait();
    dc_pdl_release();
    row_blocks<T, WIDE>(a, by_kb, items);
}

// Turned, of few tiles: 128 rows x 32 columns to a CTA, four times as many as whole tiles; the rows, if they are wanted too, are put into 8 bits by the first row_ctas CTAs, which read x once
// more.  Both ways, us, so and as whole tiles: 196 x 1024 bf16 2.0 and 4.5, 1000 x 333 f32 3.1 and 6.6, 40000 x 96 bf16 8.3 and 9.7, 6000 x 1001 14.7 and 13.4, 12544 x 512 f32 13.3 and 13.5,
// 25088 x 512 bf16 22.0 and 16.8.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(256) k_quantize_columns(const BlocksArgs a, uint2 by_kb, uint32_t items, int row_ctas)
{
    constexpr int PER = 4 / (int)sizeof(T), TEAMS = 256 * PER / 32, ROWS = 128 / TEAMS, LINE = 32 / PER;       // columns of a thread, threads to a column, rows of each, words of a row
    __shared__ uint4 tile4[128 * 32 * sizeof(T) / 16];
    __shared__ alignas(8) uint32_t most_of[TEAMS][32];
    dc_pdl_wait();
    dc_pdl_release();
    if ((int)blockIdx.x < row_ctas) { row_blocks<T, WIDE>(a, by_kb, items); return; }
    const int quarters = (a.channels + 31) / 32, tile = (int)blockIdx.x - row_ctas, tile_r = tile / quarters, col0 = (tile - tile_r * quarters) * 32;
    {
        const int part = threadIdx.x & 3, col = col0 + part * 8, there = a.channels - col;
        Eight<T> v[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = tile_r * 128 + i * 64 + (threadIdx.x >> 2);
            load_eight<WIDE>(v[i], (const char*)a.x + (size_t)row * a.x_pitch + (size_t)col * sizeof(T), row < a.rows ? there : 0);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) v[i].keep(tile4 + ((i * 64 + (threadIdx.x >> 2)) * 4 + part) * (sizeof(T) / 2));
    }
    __syncthreads();
    const int c = threadIdx.x % LINE * PER, turn = threadIdx.x / LINE, row0 = tile_r * 128 + turn * ROWS;
    const uint32_t* const word = (const uint32_t*)tile4 + turn * ROWS * LINE + threadIdx.x % LINE;
    uint32_t w[ROWS], m = 0;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) w[r] = word[r * LINE];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) m = PER == 2 ? larger2(m, w[r]) : max(m, w[r] & 0x7fffffffu);
    if (PER == 2) { m &= 0x7fff7fffu; *(uint2*)&most_of[turn][c] = make_uint2(m << 16, m & 0xffff0000u); }
    else most_of[turn][c] = m;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        uint32_t all = 0;
#pragma unroll
        for (int i = 0; i < TEAMS; ++i) all = max(all, most_of[i][c + k]);
        const BlockScale t = block_scale(all);
        const int column = col0 + c + k;
        if (column >= a.channels) break;
        if (turn == 0) a.scale_t[(size_t)column * a.rb + tile_r] = t.scale;
        const uint32_t kept = t.bad ? 0u : 0xffffffffu;
        uint32_t o[ROWS / 4];
#pragma unroll
        for (int q = 0; q < ROWS / 4; ++q) {
            float f[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(PER == 2 ? (k ? w[4 * q + i] & 0xffff0000u : w[4 * q + i] << 16) : w[4 * q + i]);
            o[q] = __byte_perm(two_e4m3(mul2(make_float2(f[0], f[1]), both<float2>(t.inv))), two_e4m3(mul2(make_float2(f[2], f[3]), both<float2>(t.inv))), 0x5410) & kept;
        }
        uint8_t* const out = a.qt + (size_t)column * a.qt_pitch + row0;
        if (row0 >= a.rows) break;
        if constexpr (ROWS == 16) store_bytes(out, make_uint4(o[0], o[1], o[2], o[3]), a.rows - row0);
        else store_bytes(out, make_uint2(o[0], o[1]), a.rows - row0);
    }
}

// Turned, or with a scale for 128 x 128 values: a CTA has such a tile, read once.  A thread has eight columns of eight rows, which it puts into 8 bits on their way to shared memory;
// and then a column (bfloat16: two) of 64 (32) rows, which it reads from there.  WHOLE: one scale for the tile.
template <typename T, bool WIDE, bool WHOLE>
__global__ void __launch_bounds__(256) k_quantize_tile(const BlocksArgs a)
{
    constexpr int PER = 4 / (int)sizeof(T), TEAMS = 2 * PER, ROWS = 128 / TEAMS;       // columns of a thread, threads to a column, rows of each
    extern __shared__ uint4 tile4[];                          // [128][128] of the map's type
    __shared__ alignas(8) uint32_t most_of[TEAMS][128];
    __shared__ uint32_t most_of_tile;
    const int tile_c = blockIdx.x % a.kb, tile_r = blockIdx.x / a.kb, lane = threadIdx.x & 31;
    const int part = threadIdx.x & 15, team = threadIdx.x >> 4, col = tile_c * 128 + part * 8, there = a.channels - col;
    dc_pdl_wait();
    dc_pdl_release();
    if (WHOLE) {
        if (threadIdx.x == 0) most_of_tile = 0;
        __syncthreads();
    }
    if (!WIDE) {
        stage_tile(a, tile_r * 128, tile_c * 128, (T*)tile4);
        __syncthreads();
    }
    uint32_t most = 0;
#pragma unroll
    for (int i0 = 0; i0 < 8; i0 += 4) {
        Eight<T> v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = tile_r * 128 + (i0 + i) * 16 + team;
            if (!WIDE) v[i].load((const char*)(tile4 + (((i0 + i) * 16 + team) * 16 + part) * (sizeof(T) / 2)));
            else load_eight<WIDE>(v[i], (const char*)a.x + (size_t)row * a.x_pitch + (size_t)col * sizeof(T), row < a.rows ? there : 0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (i0 + i) * 16 + team, row = tile_r * 128 + r;
            if (WIDE && (WHOLE || a.qt)) v[i].keep(tile4 + (r * 16 + part) * (sizeof(T) / 2));
            const uint32_t m = v[i].most();
            if (WHOLE) most = max(most, m);
            else if (a.q) {
                const BlockScale s = block_scale(most_of_half(m, lane));
                if (row < a.rows) {
                    store_eight<WIDE>(a.q + (size_t)row * a.q_pitch + col, eight_e4m3(v[i], s), there);
                    if (part == 0) a.scale[(size_t)row * a.kb + tile_c] = s.scale;
                }
            }
        }
    }
    BlockScale s;
    if (WHOLE) {
        most = __reduce_max_sync(0xffffffffu, most);
        if (lane == 0) atomicMax(&most_of_tile, most);        // the same whatever the order
        __syncthreads();
        s = block_scale(most_of_tile);
        if (threadIdx.x == 0) {
            if (a.q) a.scale[(size_t)tile_r * a.kb + tile_c] = s.scale;
            if (a.qt) a.scale_t[(size_t)tile_c * a.rb + tile_r] = s.scale;
        }
        if (a.q && there > 0)
#pragma unroll 2
            for (int i = 0; i < 8; ++i) {
                const int r = i * 16 + team, row = tile_r * 128 + r;
                if (row >= a.rows) break;
                Eight<T> v;
                v.load((const char*)(tile4 + (r * 16 + part) * (sizeof(T) / 2)));
                store_eight<WIDE>(a.q + (size_t)row * a.q_pitch + col, eight_e4m3(v, s), there);
            }
    } else __syncthreads();
    if (!a.qt) return;
    const int c = threadIdx.x % (128 / PER) * PER, turn = threadIdx.x / (128 / PER), row0 = tile_r * 128 + turn * ROWS;
    constexpr int LINE = 128 / PER;                           // words of a row
    const uint32_t* const word = (const uint32_t*)((const char*)tile4 + ((size_t)turn * ROWS * 128 + c) * sizeof(T));
    const bool whole = tile_r * 128 + 128 <= a.rows && tile_c * 128 + 128 <= a.channels;
    uint32_t w[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) w[r] = word[r * LINE];
    BlockScale t[PER];
    if (WHOLE)
#pragma unroll
        for (int k = 0; k < PER; ++k) t[k] = s;
    else {
        uint32_t m[4] = {0, 0, 0, 0};
#pragma unroll
        for (int r = 0; r < ROWS; ++r) m[r & 3] = PER == 2 ? larger2(m[r & 3], w[r]) : max(m[r & 3], w[r] & 0x7fffffffu);
        if (PER == 2) {
            const uint32_t all = larger2(larger2(m[0], m[1]), larger2(m[2], m[3])) & 0x7fff7fffu;
            *(uint2*)&most_of[turn][c] = make_uint2(all << 16, all & 0xffff0000u);
        } else most_of[turn][c] = max(max(m[0], m[1]), max(m[2], m[3]));
        __syncthreads();
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            uint32_t all = 0;
#pragma unroll
            for (int i = 0; i < TEAMS; ++i) all = max(all, most_of[i][c + k]);
            t[k] = block_scale(all);
            if (turn == 0 && tile_c * 128 + c + k < a.channels) a.scale_t[(size_t)(tile_c * 128 + c + k) * a.rb + tile_r] = t[k].scale;
        }
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const float2 inv = both<float2>(t[k].inv);
        const uint32_t kept = t[k].bad ? 0u : 0xffffffffu;
        const int column = tile_c * 128 + c + k;
        uint8_t* const out = a.qt + (size_t)column * a.qt_pitch + row0;
#pragma unroll
        for (int g = 0; g < ROWS; g += 16) {                  // sixteen rows: 16 bytes of a column
            uint32_t o[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float f[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(PER == 2 ? (k ? w[g + 4 * q + i] & 0xffff0000u : w[g + 4 * q + i] << 16) : w[g + 4 * q + i]);
                o[q] = __byte_perm(two_e4m3(mul2(make_float2(f[0], f[1]), inv)), two_e4m3(mul2(make_float2(f[2], f[3]), inv)), 0x5410) & kept;
            }
            if (whole) *(uint4*)(out + g) = make_uint4(o[0], o[1], o[2], o[3]);
            else if (column < a.channels) store_bytes(out + g, make_uint4(o[0], o[1], o[2], o[3]), a.rows - row0 - g);
        }
    }
}

// ---------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------
struct BlocksProduct {
    const uint8_t* a; size_t a_pitch; const float* a_scale;
    const uint8_t* b; size_t b_pitch; const float* b_scale;
    const float* bias;                                        // or NULL
    int64_t m; int n, k, relu, b_block_rows;
    void* out; size_t out_pitch;
};
struct BlocksLimits {
    unsigned long long wait_ns;                               // of every wait
    uint32_t loads;                                           // blocks of K that a CTA loads before it stops: 0xffffffff, but where a test makes the waits run out
};
struct BlocksTiles {
    BlocksProduct p;
    int NB, m_tiles, stages, stage_bytes, kb, k_last;         // column tiles; blocks of K; MMAs (32 values) of the last one
    uint32_t idesc;
    int bufs;                                                 // places a warp stages its boxes in, 1 or 2
    int wide, boxes;                                          // out takes 16-byte stores; is written in boxes by TMA
    BlocksLimits limits;
};

constexpr int kAddWarps = 16, kFirstAdder = 4, kBlocksThreads = (kFirstAdder + kAddWarps) * 32;
constexpr int kBlocksMostStages = 8, kScaleSlots = 3;         // a slot: the scales of four blocks of K
constexpr int kBox = 32 * 64;                                 // a warp's 32 rows on their way out, 64 bytes each; two of them
struct BlocksCtl {
    unsigned long long full[kBlocksMostStages], empty[kBlocksMostStages], tmem_full[4], tmem_empty[4], scale_full[kScaleSlots], scale_empty[kScaleSlots];
    uint32_t tmem_base;
    volatile int abort_flag;
    unsigned long long wait_ns;
};
constexpr int kBlocksSmem = 227 * 1024;
constexpr int kRowScales = 128 * 4, kScaleBytes = kScaleSlots * (kRowScales + 8) * 4, kEachBytes = kScaleSlots * (kRowScales + 4 * 256) * 4;
constexpr int kBlocksRoom = kBlocksSmem - 1024 - (int)sizeof(BlocksCtl);

#define DC_UMMA_F8(name, group)                                                                                                                 \
    __device__ __forceinline__ void name(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, int n)                            \
    {                                                                                                                                           \
        _Pragma("unroll") for (int k = 0; k < 4; ++k)                                                                                           \
            if (k < n)                                                                                                                          \
                asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t" \
                             "tcgen05.mma." group ".kind::f8f6f4 [%0], da, db, %4, p;\n\t}"                                                     \
                             ::"r"(d), "r"(a_lo + 2u * k), "r"(b_lo + 2u * k), "r"(hi), "r"(idesc), "r"(k) : "memory");                          \
    }
DC_UMMA_F8(umma_f8, "cta_group::1")
DC_UMMA_F8(umma_f8_pair, "cta_group::2")
#undef DC_UMMA_F8

// Bounded waits, of one thread and of a whole warp.  What bounds the loops that wait is the instructions, and most of all the branches, from one block of K to the next: a wait that is over
// at once is a look (of a warp: and a vote) and nothing else; the clock is looked at after 256 more.
template <typename CTL>
__device__ __forceinline__ bool blocks_late(CTL* ctl, uint32_t spin, unsigned long long& t0)
{
    if ((spin & 255u) != 255u) return false;
    const unsigned long long t = now_ns();
    if (spin == 255u) t0 = t;
    if (ctl->abort_flag == 0 && t - t0 <= ctl->wait_ns) return false;
    ctl->abort_flag = 1;
    return true;
}
template <typename CTL>
__device__ __forceinline__ bool blocks_wait(uint32_t bar, uint32_t parity, CTL* ctl)
{
    unsigned long long t0 = 0;
#pragma unroll 1
    for (uint32_t spin = 0; !mbar_try(bar, parity); ++spin)
        if (blocks_late(ctl, spin, t0)) return false;
    return true;
}
__device__ __forceinline__ uint32_t look(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{\n\t.reg .pred p, q;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tvote.sync.all.pred q, p, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done;
}
// True: it has run out.
template <typename CTL>
__device__ __forceinline__ bool blocks_run_out(uint32_t bar, uint32_t parity, CTL* ctl)
{
    if (__builtin_expect(look(bar, parity), 1)) return false;
    unsigned long long t0 = 0;
#pragma unroll 1
    for (uint32_t spin = 0; !look(bar, parity); ++spin)
        if (__any_sync(0xffffffffu, blocks_late(ctl, spin, t0))) return true;
    return false;
}
// Behind a wait that has run out: copies and MMAs that are under way get two milliseconds to end before tensor memory is freed and the CTA leaves.
__device__ __forceinline__ void blocks_settle() { const unsigned long long t0 = now_ns(); while (now_ns() - t0 < 2000000ull) { } }
// An arrival of lane 0, without a branch.
__device__ __forceinline__ void arrive_first(uint32_t bar, int lane)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.eq.s32 p, %1, 0;\n\t@p mbarrier.arrive.relaxed.cta.shared::cta.b64 _, [%0];\n\t}" ::"r"(bar), "r"(lane) : "memory");
}
// ... after which what the warp has read from shared memory may be written over.
__device__ __forceinline__ void arrive_read(uint32_t bar, int lane)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.eq.s32 p, %1, 0;\n\t@p mbarrier.arrive.release.cta.shared::cta.b64 _, [%0];\n\t}" ::"r"(bar), "r"(lane) : "memory");
}
__device__ __forceinline__ void arrive_first_remote(uint32_t bar, int lane)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.eq.s32 p, %1, 0;\n\t@p mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];\n\t}" ::"r"(bar), "r"(lane) : "memory");
}
__device__ __forceinline__ float4 lds_floats(uint32_t at)
{
    const uint4 v = lds128(at);
    return make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
}
// Two floats in one 64-bit register, as packed arithmetic has them: as pairs of 32-bit registers the sums were moved about, an instruction for each product.
__device__ __forceinline__ uint64_t pair_of(uint32_t a, uint32_t b)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ float2 floats_of(uint64_t v)
{
    float2 f;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
    return f;
}
__device__ __forceinline__ void add_product(uint64_t& sum, uint64_t a, uint64_t b) { asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(sum) : "l"(a), "l"(b)); }
__device__ __forceinline__ uint64_t product(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ void lds_pairs(uint32_t at, uint64_t* v) { asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(v[0]), "=l"(v[1]) : "r"(at)); }
// N floats from global into shared memory; zeros where there are none (`any`: an address that is).
template <int N>
__device__ __forceinline__ void copy_floats(uint32_t dst, const float* src, const float* any, bool there)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], %3, %2;" ::"r"(dst), "l"(there ? src : any), "r"(there ? 4 * N : 0), "n"(4 * N) : "memory");
}
// Columns of tensor memory, loaded and waited for in one statement: nothing that reads them comes before they are there.
__device__ __forceinline__ void tmem_read16(uint32_t taddr, uint32_t* r)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\ttcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_read32(uint32_t taddr, uint32_t* r)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\ttcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]) : "r"(taddr) : "memory");
}

// 32 rows x 16 columns in fragments: a lane has columns 8 j + 2 (lane % 4) and the next one of rows lane / 4 + 8 i, i < 4, in r[8 (i / 2) + 4 j + 2 (i % 2)] and the next one.  Four columns' scales
// to a lane, then, in the place of sixteen: shared memory hands out 128 bytes a cycle, also of one value to all lanes of a warp.  4000 x 4096 x 2000 with a scale for each row 51.9 us, with a row to a lane 61.8.
__device__ __forceinline__ void tmem_read_fragments(uint32_t taddr, uint32_t* r)
{
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%16];\n\ttcgen05.ld.sync.aligned.16x256b.x2.b32 {%8, %9, %10, %11, %12, %13, %14, %15}, [%17];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr), "r"(taddr + (16u << 16)) : "memory");
}
__device__ __forceinline__ float lds_float(uint32_t at)
{
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at));
    return v;
}
__device__ __forceinline__ uint64_t lds_pair(uint32_t at)
{
    uint64_t v;
    asm volatile("ld.shared.b64 %0, [%1];" : "=l"(v) : "r"(at));
    return v;
}

// BN: columns of a tile.  EACH: b has a scale for each row and block, not for 128 rows.
template <bool PAIR, int BN, bool EACH, typename T>
__global__ void __launch_bounds__(kBlocksThreads, 1) k_blocks(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmC, const BlocksTiles a)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* const ring = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* const staging = ring + a.stages * a.stage_bytes;
    float* const row_scale = (float*)(staging + kAddWarps * a.bufs * kBox);  // [slots][128 rows][4 blocks]
    float* const col_scale = row_scale + kScaleSlots * kRowScales;           // EACH: [slots][4 blocks][256 columns]; else [slots][2][4 blocks]: of either 128 columns
    constexpr int kCols = EACH ? 4 * 256 : 8;
    BlocksCtl* const ctl = (BlocksCtl*)(col_scale + kScaleSlots * kCols);
    const BlocksProduct& p = a.p;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int rank = PAIR ? (int)cluster_rank() : 0, first = PAIR ? blockIdx.x >> 1 : blockIdx.x, step = PAIR ? gridDim.x >> 1 : gridDim.x;
    constexpr bool FRAG = EACH && BN > 128;                   // (with 32 columns to a warp a row to a lane is as fast or faster: 4000 x 4096 x 2000 57.5 us and 59)
    constexpr int M = PAIR ? 2 : 1, PARTS = BN < 128 ? 2 : 4; // row tiles of an item; warps that share a row's columns
    // Tiles of 256 columns are two halves with accumulators, barriers and an issuer of their own.
    constexpr int HALVES = BN > 128 ? 2 : 1, BH = BN / HALVES;
    constexpr uint32_t ACCS = HALVES == 2 ? 2 : 4, kColumns = 4 * BH;         // accumulators of a half

    if (threadIdx.x == 0) {
        for (int i = 0; i < a.stages; ++i) { mbar_init(&ctl->full[i], 1); mbar_init(&ctl->empty[i], HALVES); }
        for (int i = 0; i < 4; ++i) { mbar_init(&ctl->tmem_full[i], 1); mbar_init(&ctl->tmem_empty[i], 4 * PARTS / HALVES * M); }
        for (int i = 0; i < kScaleSlots; ++i) { mbar_init(&ctl->scale_full[i], 32); mbar_init(&ctl->scale_empty[i], 4 * PARTS); }
        ctl->abort_flag = 0;
        ctl->wait_ns = a.limits.wait_ns;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmA) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmB) : "memory");
    }
    if (warp == 1) {
        if (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(kColumns) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(kColumns) : "memory");
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
    const int n_items = (a.m_tiles + M - 1) / M * a.NB;
    // row tile `rank` of an item; an absent second tile repeats the first, and nothing of it is stored
    auto tile_of = [&](int group, bool* there) -> int {
        const int idx = group * M + rank;
        *there = idx < a.m_tiles;
        return *there ? idx : idx - rank;
    };
    const uint32_t full0 = smem_u32(&ctl->full[0]), empty0 = smem_u32(&ctl->empty[0]), ring0 = smem_u32(ring);

    if (warp < kFirstAdder) {
        if (warp == 0) {
            // ---------------- producer ----------------
            if (elect_one()) {
                const uint32_t lead_full = PAIR ? map_to_cta(&ctl->full[0], 0) : full0;
                RingPos r;
                r.start(ring0, (uint32_t)a.stages);
                uint32_t left = a.limits.loads;
                bool ok = true, there;
                for (int item = first; item < n_items && ok; item += step) {
                    const int group = item / a.NB, row = tile_of(group, &there) * kTileM, col = (item - group * a.NB) * BN + rank * (BH / 2);
                    for (int kc = 0; kc < a.kb; ++kc) {
                        ok = left-- != 0u && blocks_wait(empty0 + r.off, r.phase ^ 1u, ctl);
                        if (!ok) break;
                        if (PAIR) {
                            if (rank == 0) mbar_expect_tx(full0 + r.off, 2u * (uint32_t)a.stage_bytes);
                            load_pair(r.data, &tmA, kc * kBytesK, row, lead_full + r.off);
                            load_pair(r.data + kATile, &tmB, kc * kBytesK, col, lead_full + r.off);
                            if (HALVES == 2) load_pair(r.data + kATile + BH / 2 * kBytesK, &tmB, kc * kBytesK, col + BH, lead_full + r.off);
                        } else {
                            mbar_expect_tx(full0 + r.off, (uint32_t)a.stage_bytes);
                            tma_load_2d(r.data, &tmA, kc * kBytesK, row, full0 + r.off);
                            tma_load_2d(r.data + kATile, &tmB, kc * kBytesK, col, full0 + r.off);
                        }
                        r.next(ring0, (uint32_t)a.stages, (uint32_t)a.stage_bytes);
                    }
                }
            }
            __syncwarp();
        } else if (warp <= HALVES) {
            // ---------------- MMA issuers (of a pair: the leader's, for both CTAs) ----------------
            // What bounds a block of K is its round: MMAs, their completion's way to the adders, the reads, the release's way back, the issue.  Halves with rounds of their own take as many columns at
            // once as one issuer's, but their MMAs half as long: 8192 x 4096 x 4096 121 to 125 us, 127 as one; 25088 x 512 x 2048 40.4 and 43.
            if (rank == 0 && elect_one()) {
                const uint64_t dconst = umma_desc(0, 1024, 2);
                const uint32_t d_hi = (uint32_t)(dconst >> 32), r0 = (uint32_t)dconst + (ring0 >> 4), slot = (uint32_t)a.stage_bytes >> 4;
                const uint32_t tmem_empty0 = smem_u32(&ctl->tmem_empty[0]) + 16u * ((uint32_t)warp - 1u), tmem_full0 = smem_u32(&ctl->tmem_full[0]) + 16u * ((uint32_t)warp - 1u);
                RingPos r;
                r.start(r0, (uint32_t)a.stages);
                uint32_t acc = 0, acc_ph = 1;
                const uint32_t half = (uint32_t)warp - 1u, b_at = (kATile + half * (uint32_t)(BH / 2 * kBytesK)) >> 4;
                bool ok = true;
                for (int item = first; item < n_items && ok; item += step)
                    for (int kc = 0; kc < a.kb; ++kc) {
                        ok = blocks_wait(full0 + r.off, r.phase, ctl) && blocks_wait(tmem_empty0 + 8u * acc, acc_ph, ctl);
                        if (!ok) break;
                        tc_fence_after();
                        const int n = kc + 1 < a.kb ? 4 : a.k_last;
                        const uint32_t d = tmem_base + (half * ACCS + acc) * (uint32_t)BH;
                        if (PAIR) {
                            umma_f8_pair(d, r.data, r.data + b_at, d_hi, a.idesc, n);
                            commit_pair(tmem_full0 + 8u * acc);
                            commit_pair(empty0 + r.off);
                        } else {
                            umma_f8(d, r.data, r.data + (kATile >> 4), d_hi, a.idesc, n);
                            umma_commit_at(tmem_full0 + 8u * acc);
                            umma_commit_at(empty0 + r.off);
                        }
                        r.next(r0, (uint32_t)a.stages, slot);
                        if (++acc == ACCS) { acc = 0; acc_ph ^= 1u; }
                    }
            }
            __syncwarp();
        } else if (warp == 3) {
            // ---------------- scales ----------------
            // Copied four blocks at a time, straight into shared memory, several slots ahead.  A row's scales lie side by side: 16 bytes to a copy where they are
            // aligned.  A lane has four rows, and of EACH's columns eight at most.
            uint32_t slot = 0, phase = 0;
            bool there, dead = false;
            const bool quads = a.kb % 4 == 0 && ((uintptr_t)p.a_scale | (uintptr_t)p.b_scale) % 16 == 0;
            for (int item = first; item < n_items && !dead; item += step) {
                const int group = item / a.NB, tile = tile_of(group, &there), n0 = (item - group * a.NB) * BN;
                const float* const rows = p.a_scale + ((size_t)tile * kTileM + lane) * a.kb;
                const int n_rows = (int)min((int64_t)kTileM, p.m - (int64_t)tile * kTileM) - lane;
                const int j0 = EACH ? n0 + lane : n0 / 128 + lane, n_cols = EACH ? p.n - j0 : lane < 2 ? (p.n + 127) / 128 - j0 : 0;
                const float* const cols = p.b_scale + (size_t)j0 * a.kb;
                for (int kc = 0; kc < a.kb; kc += 4) {
                    dead = blocks_run_out(smem_u32(&ctl->scale_empty[slot]), phase ^ 1u, ctl);
                    if (dead) break;
                    const uint32_t rows_at = smem_u32(row_scale + slot * kRowScales) + 16 * lane, cols_at = smem_u32(col_scale + slot * kCols);
                    if (quads) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) copy_floats<4>(rows_at + i * 512, rows + (size_t)(32 * i) * a.kb + kc, p.a_scale, 32 * i < n_rows);
                        if (!EACH && lane < 2) copy_floats<4>(cols_at + 16 * lane, cols + kc, p.b_scale, n_cols > 0);
                    } else
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const bool on = kc + u < a.kb;
#pragma unroll
                            for (int i = 0; i < 4; ++i) copy_floats<1>(rows_at + i * 512 + 4 * u, rows + (size_t)(32 * i) * a.kb + kc + u, p.a_scale, on && 32 * i < n_rows);
                            if (!EACH && lane < 2) copy_floats<1>(cols_at + 16 * lane + 4 * u, cols + kc + u, p.b_scale, on && n_cols > 0);
                        }
                    if (EACH)
#pragma unroll
                        for (int u = 0; u < 4; ++u)
#pragma unroll
                            for (int i = 0; i < BN / 32; ++i)
                                copy_floats<1>(cols_at + u * 1024 + i * 128 + 4 * lane, cols + (size_t)(32 * i) * a.kb + kc + u, p.b_scale, kc + u < a.kb && 32 * i < n_cols);
                    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&ctl->scale_full[slot])) : "memory");
                    if (++slot == kScaleSlots) { slot = 0; phase ^= 1u; }
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
        }
    } else if (warp < kFirstAdder + 4 * PARTS) {
        // ---------------- sums of the blocks; bias, ReLU, rounding, store ----------------
        // A warp has 32 rows (the quadrant of tensor memory that it may read), one to a lane or, FRAG, in fragments, and a quarter of the columns (of 64: half, so that they make a box; the rest has nothing to do).
        constexpr int MINE = BN / PARTS;
        const int q = warp & 3, part = (warp - kFirstAdder) >> 2;
        uint32_t stage = smem_u32(staging) + (uint32_t)(warp - kFirstAdder) * kBox;
        const uint32_t both_places = a.bufs == 2 ? stage ^ (stage + kAddWarps * kBox) : 0;       // from one place to the other
        const uint32_t half = HALVES == 2 ? part / 2 : 0, lead_empty = PAIR ? map_to_cta(&ctl->tmem_empty[0], 0) + 16u * half : 0;
        const uint32_t my_rows = smem_u32(row_scale) + (uint32_t)(q * 32 + (FRAG ? lane >> 2 : lane)) * 16, my_cols = smem_u32(col_scale) + (uint32_t)(EACH ? part * MINE + (FRAG ? 2 * (lane & 3) : 0) : BN > 128 ? part / 2 * 4 : 0) * 4;
        uint32_t acc = 0, acc_ph = 0, slot = 0, phase = 0;
        bool there, dead = false;
        const uint32_t tmem_full0 = smem_u32(&ctl->tmem_full[0]) + 16u * half, tmem_empty0 = smem_u32(&ctl->tmem_empty[0]);
        const uint32_t from0 = tmem_base + half * ACCS * (uint32_t)BH + (uint32_t)(part * MINE) % (uint32_t)BH + ((uint32_t)(q * 32) << 16);
        const uint32_t scale_full0 = smem_u32(&ctl->scale_full[0]), scale_empty0 = smem_u32(&ctl->scale_empty[0]);
        for (int item = first; item < n_items; item += step) {
            const int group = item / a.NB, tile = tile_of(group, &there), n0 = (item - group * a.NB) * BN + part * MINE;
            const int64_t row0 = (int64_t)tile * kTileM + q * 32;
            const int rows = there ? (int)max((int64_t)0, min((int64_t)32, p.m - row0)) : 0;
            uint64_t sum[MINE / 2];
#pragma unroll
            for (int i = 0; i < MINE / 2; ++i) sum[i] = 0;
            // A warp whose wait has run out takes no part any more: it hands nothing back, so nothing that others still read is written over, and stores NaN.  Another one's sums are whole, or its own wait runs out.
            for (int k0 = 0; k0 < a.kb && !dead; k0 += 4) {
                if (blocks_run_out(scale_full0 + 8u * slot, phase, ctl)) { dead = true; break; }
                float s0 = 0.f, s1 = 0.f, s2 = 0.f, s3 = 0.f;
                if (!FRAG) {
                    const float4 r = lds_floats(my_rows + slot * (kRowScales * 4)), b = EACH ? make_float4(1.f, 1.f, 1.f, 1.f) : lds_floats(my_cols + slot * (kCols * 4));
                    s0 = r.x * b.x; s1 = r.y * b.y; s2 = r.z * b.z; s3 = r.w * b.w;
                }
                uint32_t cols = my_cols + slot * (kCols * 4), rows_at = my_rows + slot * (kRowScales * 4);
                const int here = min(4, a.kb - k0);
#pragma unroll 1
                for (int u = 0; u < here; ++u, cols += 1024, rows_at += 4) {
                    uint64_t s[FRAG ? 4 : 1];
                    if constexpr (FRAG) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) { const uint32_t t = __float_as_uint(lds_float(rows_at + i * 128)); s[i] = pair_of(t, t); }
                    } else {
                        s[0] = pair_of(__float_as_uint(s0), __float_as_uint(s0));
                        s0 = s1; s1 = s2; s2 = s3;
                    }
                    if (blocks_run_out(tmem_full0 + 8u * acc, acc_ph, ctl)) { dead = true; break; }
                    tc_fence_after();
                    const uint32_t from = from0 + acc * (uint32_t)BH;
#pragma unroll
                    for (int c = 0; c < MINE; c += 16) {
                        uint32_t v[16];
                        uint64_t of_cols[2];
                        if constexpr (FRAG) {
                            of_cols[0] = lds_pair(cols + (uint32_t)c * 4);   // (under way while tensor memory is read)
                            of_cols[1] = lds_pair(cols + (uint32_t)c * 4 + 32);
                            tmem_read_fragments(from + c, v);
                        } else tmem_read16(from + c, v);
                        if (c + 16 == MINE) {
                            tc_fence_before();
                            __syncwarp();
                            if (PAIR) arrive_first_remote(lead_empty + 8u * acc, lane);
                            else arrive_first(tmem_empty0 + 8u * acc, lane);
                        }
                        if constexpr (FRAG) {
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                add_product(sum[c / 2 + i], product(pair_of(v[2 * i], v[2 * i + 1]), of_cols[i >> 1 & 1]), s[2 * (i >> 2) + (i & 1)]);
                        } else
#pragma unroll
                            for (int i = 0; i < 8; i += 2) {
                                uint64_t t[2] = {pair_of(v[2 * i], v[2 * i + 1]), pair_of(v[2 * i + 2], v[2 * i + 3])};
                                if (EACH) {
                                    uint64_t w[2];
                                    lds_pairs(cols + (uint32_t)(c + 2 * i) * 4, w);
                                    t[0] = product(t[0], w[0]);
                                    t[1] = product(t[1], w[1]);
                                }
                                add_product(sum[c / 2 + i], t[0], s[0]);
                                add_product(sum[c / 2 + i + 1], t[1], s[0]);
                            }
                    }
                    acc = (acc + 1u) & (ACCS - 1u);
                    acc_ph ^= acc == 0u;
                }
                if (dead) break;
                __syncwarp();
                arrive_read(scale_empty0 + 8u * slot, lane);
                slot = slot + 1u == kScaleSlots ? 0u : slot + 1u;
                phase ^= slot == 0u;
            }
            if (dead)
#pragma unroll
                for (int i = 0; i < MINE / 2; ++i) sum[i] = 0x7fffffff7fffffffull;
            constexpr int PER = 64 / (int)sizeof(T);          // columns of a box
#pragma unroll
            for (int c = 0; c < MINE; c += PER) {
                const int c1 = n0 + c;
                if (c1 >= p.n) break;
                if (a.boxes) { if (lane == 0) store_read(a.bufs); }
                __syncwarp();
                // 32 rows of 64 bytes, the 16 bytes of a row in another order for each two rows: no bank conflicts
                if constexpr (FRAG) {
                    const uint32_t at = stage + (lane >> 2) * 64, mix = lane >> 3 & 3;
#pragma unroll
                    for (int j = 0; j < PER / 8; ++j) {
                        const int j1 = c1 + 8 * j + 2 * (lane & 3);
                        const float2 bias = make_float2(p.bias && j1 < p.n ? dc_ld(p.bias + j1) : 0.f, p.bias && j1 + 1 < p.n ? dc_ld(p.bias + j1 + 1) : 0.f);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {         // row lane / 4 + 8 i
                            const float2 f = add2(floats_of(sum[(c + 8 * j) / 16 * 8 + 4 * (i >> 1) + 2 * (j & 1) + (i & 1)]), bias);
                            if constexpr (sizeof(T) == 2)
                                asm volatile("st.shared.b32 [%0], %1;" ::"r"(at + i * 512 + ((j ^ mix) << 4) + 4 * (lane & 3)), "r"(p.relu ? two_bf16<true>(f) : two_bf16<false>(f)) : "memory");
                            else
                                asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(at + i * 512 + (((2 * j + (lane >> 1 & 1)) ^ mix) << 4) + 8 * (lane & 1)),
                                             "f"(p.relu ? clamped<true>(f.x) : f.x), "f"(p.relu ? clamped<true>(f.y) : f.y) : "memory");
                        }
                    }
                } else {
                    uint32_t w[16];
#pragma unroll
                    for (int i = 0; i < PER / 2; ++i) {
                        float2 f = floats_of(sum[c / 2 + i]);
                        const int j = c1 + 2 * i;
                        if (p.bias) f = add2(f, make_float2(j < p.n ? dc_ld(p.bias + j) : 0.f, j + 1 < p.n ? dc_ld(p.bias + j + 1) : 0.f));
                        if constexpr (sizeof(T) == 2) w[i] = p.relu ? two_bf16<true>(f) : two_bf16<false>(f);
                        else {
                            w[2 * i] = __float_as_uint(p.relu ? clamped<true>(f.x) : f.x);
                            w[2 * i + 1] = __float_as_uint(p.relu ? clamped<true>(f.y) : f.y);
                        }
                    }
#pragma unroll
                    for (int u = 0; u < 4; ++u) sts128(stage + lane * 64 + ((u ^ ((lane >> 1) & 3)) << 4), w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]);
                }
                if (a.boxes) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0 && rows > 0) store_box(&tmC, stage, c1, (int)row0);
                    stage ^= both_places;
                    continue;
                }
                __syncwarp();
                if (a.wide && c1 + PER <= p.n) {              // four lanes to 64 bytes
                    const int u = lane & 3;
#pragma unroll
                    for (int it = 0; it < 4; ++it) {
                        const int r = it * 8 + (lane >> 2);
                        if (r < rows) *(uint4*)((char*)p.out + (size_t)(row0 + r) * p.out_pitch + (size_t)c1 * sizeof(T) + u * 16) = lds128(stage + r * 64 + ((u ^ ((r >> 1) & 3)) << 4));
                    }
                } else {                                      // an element per lane, side by side
                    constexpr int AT_ONCE = 32 / PER;         // rows
                    const int e = lane & (PER - 1), u = e * (int)sizeof(T) >> 4;
#pragma unroll 4
                    for (int it = 0; it < 32 / AT_ONCE; ++it) {
                        const int r = it * AT_ONCE + lane / PER;
                        const uint32_t at = stage + r * 64 + ((u ^ ((r >> 1) & 3)) << 4) + (e * (int)sizeof(T) & 15);
                        if (r < rows && c1 + e < p.n) {
                            T* const out = (T*)((char*)p.out + (size_t)(row0 + r) * p.out_pitch) + c1 + e;
                            if constexpr (sizeof(T) == 4) { uint32_t x; asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(at) : "memory"); *(uint32_t*)out = x; }
                            else { uint16_t x; asm volatile("ld.shared.b16 %0, [%1];" : "=h"(x) : "r"(at) : "memory"); *(uint16_t*)out = x; }
                        }
                    }
                }
                __syncwarp();
            }
        }
        if (a.boxes && lane == 0) store_done();
    }
    tc_fence_before();
    __syncthreads();
    if (ctl->abort_flag) blocks_settle();
    if (PAIR) cluster_sync_all();                             // neither CTA frees tensor memory or leaves while the other may still use it
    if (warp == 1) {
        tc_fence_after();
        if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kColumns) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kColumns) : "memory");
    }
}

// ---------------------------------------------------------------------------
// products of few rows
// ---------------------------------------------------------------------------
// What bounds them are the weights, each read once: they are the side of 128 rows (tensor memory's lanes), the rows of a (16 to 128 of them) its columns, and the blocks of K are dealt to a
// cluster of CTAs, enough of them for the weights to stream at HBM's rate.  Each CTA scales and adds up its own blocks in registers; the partial sums meet in distributed shared
// memory, where CTA r finishes channels r * 128 / CS and on, in the order of the ranks.  `early`: everything older than the kernel before is complete (dc_linear_blocks: that kernel
// puts x into 8 bits), so the weights' loads start before the wait for it.
constexpr int kSplitStages = 12, kSplitScales = 32 * 1024;
template <int NT> struct SplitAdders { static constexpr int N = NT < 64 ? 4 : NT < 128 ? 8 : 16; };   // warps that add up: of wide tiles two or four to the same 32 channels, with a share of the columns each
// A CTA of it waits for its cluster, and tensor memory is given out without a limit on the wait: it takes at least this much shared memory for each 128 columns, so that what fits beside
// it has columns too (as the split product of integers, dc_quant.cu).
constexpr size_t kSplitLeast = 64 * 1024;
struct BlocksSplit {
    BlocksProduct p;
    int CS, stages, kb, k_last, m_tiles, early;
    uint32_t idesc;
    BlocksLimits limits;                                      // loads: of the first CTA of a cluster
};
struct BlocksSplitCtl {
    unsigned long long full[kSplitStages], empty[kSplitStages], tmem_full[4], tmem_empty[4];
    uint32_t tmem_base;
    volatile int abort_flag;
    unsigned long long wait_ns;
};

template <int NT, bool EACH, typename T>
__global__ void __launch_bounds__(64 + 32 * SplitAdders<NT>::N, 1) k_blocks_split(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const BlocksSplit a)
{
    constexpr uint32_t kStageBytes = kATile + NT * kBytesK, ACCS = 4, kColumns = ACCS * NT;          // accumulators
    constexpr int LD = NT < 32 ? 16 : 32, ADDERS = SplitAdders<NT>::N, kThreads = 64 + 32 * ADDERS, MINE = NT / (ADDERS / 4);
    extern __shared__ uint8_t smem_raw[];
    uint8_t* const ring = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    // [CS][NT / 4][128 / CS]: this CTA's channels, four rows' sums each, from every CTA; a warp's stores lie side by side
    float4* const red = (float4*)(ring + (size_t)a.stages * kStageBytes);
    BlocksSplitCtl* const ctl = (BlocksSplitCtl*)(red + 32 * NT);
    float* const scale = (float*)(ctl + 1);                   // [this CTA's blocks][NT]: of the rows, without EACH times the weights'
    const BlocksProduct& p = a.p;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int rank = (int)cluster_rank(), item = blockIdx.x / a.CS, mt = item % a.m_tiles, nt = item / a.m_tiles;
    const int nk = (a.kb - rank + a.CS - 1) / a.CS;           // block it * CS + rank: a cluster reads whole stretches of a row at once

    if (threadIdx.x == 0) {
        for (int i = 0; i < a.stages; ++i) { mbar_init(&ctl->full[i], 2); mbar_init(&ctl->empty[i], 1); }   // weights and rows arrive apart
        for (int i = 0; i < (int)ACCS; ++i) { mbar_init(&ctl->tmem_full[i], 1); mbar_init(&ctl->tmem_empty[i], ADDERS); }
        ctl->abort_flag = 0;
        ctl->wait_ns = a.limits.wait_ns;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmW) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmX) : "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(kColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");    // waited for before another CTA's shared memory is written
    tc_fence_after();
    const uint32_t tmem_base = ctl->tmem_base;
    const uint32_t full0 = smem_u32(&ctl->full[0]), empty0 = smem_u32(&ctl->empty[0]), ring0 = smem_u32(ring);
    const int loads = rank == 0 && a.limits.loads < (uint32_t)nk ? (int)a.limits.loads : nk, ahead = loads < a.stages ? loads : a.stages;
    auto load_weights = [&](int it, uint32_t off, uint32_t slot) {
        mbar_expect_tx(full0 + off, (uint32_t)kATile);
        tma_load_2d(slot, &tmW, (it * a.CS + rank) * kBytesK, nt * kTileM, full0 + off);
    };
    if (!a.early) { dc_pdl_wait(); dc_pdl_release(); }
    if (warp == 0 && elect_one())
        for (int it = 0; it < ahead; ++it) load_weights(it, 8u * it, ring0 + it * kStageBytes);
    __syncwarp();
    if (a.early) { dc_pdl_wait(); dc_pdl_release(); }

    bool waited = false;                                                     // for the cluster
    // the channel that this thread finishes: the threads are a multiple of a CTA's channels
    const int rows = 128 / a.CS, ch = threadIdx.x % rows, j = nt * kTileM + rank * rows + ch;
    const float bias = j < p.n && p.bias ? dc_ld(p.bias + j) : 0.f;
    if (warp == 0) {
        // ---------------- producer ----------------
        if (elect_one()) {
            RingPos r;
            r.start(ring0, (uint32_t)a.stages);
            for (int it = 0; it < loads; ++it) {
                if (it >= a.stages) {
                    if (!blocks_wait(empty0 + r.off, r.phase ^ 1u, ctl)) break;
                    load_weights(it, r.off, r.data);
                }
                mbar_expect_tx(full0 + r.off, (uint32_t)(NT * kBytesK));
                tma_load_2d(r.data + kATile, &tmX, (it * a.CS + rank) * kBytesK, mt * NT, full0 + r.off);
                r.next(ring0, (uint32_t)a.stages, kStageBytes);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        if (elect_one()) {
            const uint64_t dconst = umma_desc(0, 1024, 2);
            const uint32_t d_hi = (uint32_t)(dconst >> 32), r0 = (uint32_t)dconst + (ring0 >> 4);
            RingPos r;
            r.start(r0, (uint32_t)a.stages);
            uint32_t acc = 0, acc_ph = 1;
            for (int it = 0; it < nk; ++it) {
                if (!blocks_wait(full0 + r.off, r.phase, ctl) || !blocks_wait(smem_u32(&ctl->tmem_empty[acc]), acc_ph, ctl)) break;
                tc_fence_after();
                umma_f8(tmem_base + acc * NT, r.data, r.data + (kATile >> 4), d_hi, a.idesc, it * a.CS + rank + 1 < a.kb ? 4 : a.k_last);
                umma_commit_at(smem_u32(&ctl->tmem_full[acc]));
                umma_commit_at(empty0 + r.off);
                r.next(r0, (uint32_t)a.stages, kStageBytes >> 4);
                acc = (acc + 1u) & (ACCS - 1u);
                acc_ph ^= acc == 0;
            }
        }
        __syncwarp();
    } else {
        // ---------------- sums of this CTA's blocks, and their way to the CTA that finishes the channel ----------------
        const int q = warp & 3, m = q * 32 + lane, owner = m / rows, col0 = (warp - 2) / 4 * MINE;
        for (int i = threadIdx.x - 64; i < nk * NT; i += 32 * ADDERS) {
            const int64_t row = (int64_t)mt * NT + i % NT;
            const int at = i / NT * a.CS + rank;
            float s = row < p.m ? p.a_scale[row * a.kb + at] : 0.f;
            if (!EACH) s *= dc_ld(p.b_scale + (size_t)nt * a.kb + at);
            scale[i] = s;
        }
        const float* const weight_scale = p.b_scale + (size_t)min(nt * kTileM + m, p.n - 1) * a.kb + rank;      // EACH: of this lane's channel
        asm volatile("bar.sync 1, %0;" ::"n"(32 * ADDERS) : "memory");
        uint64_t sum[MINE / 2];
#pragma unroll
        for (int i = 0; i < MINE / 2; ++i) sum[i] = 0;
        uint32_t acc = 0, acc_ph = 0;
        const uint32_t scale0 = smem_u32(scale + col0);
        bool dead = false;
        float next = EACH && nk > 0 ? weight_scale[0] : 1.f;
        for (int it = 0; it < nk; ++it) {
            const uint32_t sw = __float_as_uint(next);
            if (EACH && it + 1 < nk) next = weight_scale[(size_t)(it + 1) * a.CS];
            dead = blocks_run_out(smem_u32(&ctl->tmem_full[acc]), acc_ph, ctl);
            if (dead) break;
            tc_fence_after();
            const uint32_t from = tmem_base + acc * NT + col0 + ((uint32_t)(q * 32) << 16);
#pragma unroll
            for (int c = 0; c < MINE; c += LD) {
                uint32_t v[LD];
                if constexpr (LD == 32) tmem_read32(from + c, v);
                else tmem_read16(from + c, v);
#pragma unroll
                for (int i = 0; i < LD / 2; i += 2) {
                    uint64_t s[2], t[2] = {pair_of(v[2 * i], v[2 * i + 1]), pair_of(v[2 * i + 2], v[2 * i + 3])};
                    lds_pairs(scale0 + (uint32_t)(it * NT + c + 2 * i) * 4, s);
                    if (EACH) { t[0] = product(t[0], pair_of(sw, sw)); t[1] = product(t[1], pair_of(sw, sw)); }
                    add_product(sum[c / 2 + i], t[0], s[0]);
                    add_product(sum[c / 2 + i + 1], t[1], s[1]);
                }
            }
            tc_fence_before();
            __syncwarp();
            arrive_first(smem_u32(&ctl->tmem_empty[acc]), lane);
            acc = (acc + 1u) & (ACCS - 1u);
            acc_ph ^= acc == 0;
        }
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        waited = true;
        if (!dead) {
            const uint32_t dst = map_to_cta(red + rank * (NT / 4) * rows + m - owner * rows, (uint32_t)owner);
            const int there = (int)min((int64_t)NT, p.m - (int64_t)mt * NT);
#pragma unroll
            for (int c = 0; c < MINE; c += 4)
                if (col0 + c < there) {
                    const float2 x = floats_of(sum[c / 2]), y = floats_of(sum[c / 2 + 1]);
                    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(dst + (uint32_t)((col0 + c) / 4 * rows * 16)), "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y) : "memory");
                }
        }
    }
    if (!waited) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    // a CTA that gave up has not sent its sums: every CTA of the cluster hears of it
    if (ctl->abort_flag != 0) {
        for (int r = 0; r < a.CS; ++r)
            asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(map_to_cta((const void*)&ctl->abort_flag, (uint32_t)r)), "r"(1) : "memory");
        blocks_settle();
    }
    cluster_sync_all();                      // this CTA's channels have arrived from every CTA
    {
        // ---------------- this CTA's channels: sums from all ranks, bias, ReLU, rounding, store ----------------
        const int there = (int)min((int64_t)NT, p.m - (int64_t)mt * NT);
        const float dead = ctl->abort_flag != 0 ? __uint_as_float(0x7fffffffu) : 0.f;        // what is stored says so
        for (int t = threadIdx.x / rows * 4; t < there && j < p.n; t += kThreads / rows * 4) {    // four rows of a
            float4 sum = make_float4(dead, dead, dead, dead);
            for (int r = 0; r < a.CS; ++r) {
                const float4 v = red[(r * (NT / 4) + t / 4) * rows + ch];
                sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
            }
            const float sums[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (t + k >= there) break;
                float f = sums[k] + bias;
                if (p.relu) f = clamped<true>(f);
                T* const out = (T*)((char*)p.out + (size_t)((int64_t)mt * NT + t + k) * p.out_pitch) + j;
                if constexpr (sizeof(T) == 4) *out = f;
                else *out = __float2bfloat16_rn(f);
            }
        }
    }
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kColumns) : "memory");
    }
}

// Clusters of so many CTAs, each with an SM of its own, that the device holds at once (none, it may be).  A query that fails is the call's error: a guess in its place would sum up in another order.
int clusters_at_once(int cs, int device, int* at_once)
{
    static std::atomic<int> known[64][4];                     // and one more
    const int at = cs == 1 ? 0 : cs == 2 ? 1 : cs == 4 ? 2 : 3;
    if (device >= 0 && device < 64)
        if (const int n = known[device][at].load(std::memory_order_relaxed)) { *at_once = n - 1; return DC_OK; }
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cs; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)cs); cfg.blockDim = dim3(192); cfg.dynamicSmemBytes = 200 * 1024; cfg.attrs = attr; cfg.numAttrs = 1;
    int n = 0;
    DC_CUDA(cudaFuncSetAttribute(k_blocks_split<16, false, float>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBlocksSmem));
    DC_CUDA(cudaOccupancyMaxActiveClusters(&n, k_blocks_split<16, false, float>, &cfg));
    if (device >= 0 && device < 64) known[device][at].store(n + 1, std::memory_order_relaxed);
    *at_once = n;
    return DC_OK;
}

// Failure detection without a fault (not part of the public header: tests declare it themselves).  The next product loads the operands of `blocks` blocks of K in each CTA (of clusters that share a
// sum: in the first one, all in the others) and bounds its waits by wait_ms in the place of 2 s: they run out, what was not summed up whole becomes NaN, and the kernel returns.  No copy and no MMA is
// under way then.  The product after it is an ordinary one.
std::atomic<uint64_t> g_stall;                                // wait_ms, blocks
BlocksLimits next_limits()
{
    if (g_stall.load(std::memory_order_relaxed))
        if (const uint64_t t = g_stall.exchange(0)) return {(t >> 32) * 1000000ull, (uint32_t)t};
    return {kWaitNs, 0xffffffffu};
}

// How a product of few tiles is split, and the cycles that it takes (as launch_product counts them).
struct SplitPlan { int NT, CS; double cost; };
int split_plan(const BlocksProduct& p, int kb, int device, SplitPlan* plan)
{
    SplitPlan& best = *plan;
    best = {};
    const int NT = p.m <= 16 ? 16 : p.m <= 32 ? 32 : p.m <= 64 ? 64 : 128;
    const long long tiles = (p.m + NT - 1) / NT * (long long)dc_div_up(p.n, kTileM);
    for (int cs = 2; cs <= 8 && cs <= kb; cs *= 2) {
        if ((size_t)dc_div_up(kb, cs) * NT * sizeof(float) > (size_t)kSplitScales) continue;
        int at_once = 0;
        const int rc = clusters_at_once(cs, device, &at_once);
        if (rc != DC_OK) return rc;
        if (at_once < 1) continue;
        const long long rounds = (tiles + at_once - 1) / at_once;
        // HBM's 3400 bytes a cycle shared by the CTAs; a block's way through tensor memory; to send the sums, join and store them
        const double load = (kATile + NT * kBytesK) / 50.0, hbm = kATile * (double)(tiles * cs < at_once * cs ? tiles * cs : at_once * cs) / 3400.0, add = 400.0 + 4.0 * NT;
        const double join = 2500.0 + NT * (cs == 8 ? 30.0 : cs == 4 ? 40.0 : 50.0);
        const double step = load > hbm ? (load > add ? load : add) : (hbm > add ? hbm : add), cost = rounds * (dc_div_up(kb, cs) * step + join);
        if (rounds <= 2 && (best.CS == 0 || cost < best.cost)) best = {NT, cs, cost};
    }
    return DC_OK;
}

template <int NT, bool EACH, typename T>
int launch_split_as(const BlocksProduct& p, const SplitPlan& s, int kb, int early, int device, cudaStream_t stream)
{
    BlocksSplit a = {};
    a.p = p; a.CS = s.CS; a.kb = kb; a.k_last = dc_div_up(p.k - (kb - 1) * kBytesK, 32); a.early = early; a.limits = next_limits();
    a.m_tiles = (int)((p.m + NT - 1) / NT);
    const int stage = kATile + NT * kBytesK, most = dc_div_up(kb, s.CS), fixed = 128 * NT * 4 + (int)sizeof(BlocksSplitCtl) + 1024 + most * NT * 4, room = (kBlocksSmem - fixed) / stage;
    a.stages = room < kSplitStages ? room : kSplitStages;
    if (a.stages > most) a.stages = most;
    a.idesc = (1u << 4) | ((uint32_t)(NT >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
    CUtensorMap tmW, tmX;
    if (!encode_rows(&tmW, p.b, p.b_pitch, p.n, p.k, kTileM) || !encode_rows(&tmX, p.a, p.a_pitch, p.m, p.k, NT)) return DC_ERR_CUDA;
    static dc_once_per_device attr_set;
    DC_CUDA(attr_set.ensure(device, [] { return cudaFuncSetAttribute(k_blocks_split<NT, EACH, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBlocksSmem); }));
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)s.CS; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.m_tiles * dc_div_up(p.n, kTileM) * s.CS)); cfg.blockDim = dim3(64 + 32 * SplitAdders<NT>::N);
    const size_t smem = (size_t)a.stages * stage + fixed, least = NT > 64 ? kBlocksSmem : kSplitLeast * (NT > 32 ? 2 : 1);
    cfg.dynamicSmemBytes = smem > least ? smem : least; cfg.stream = stream;
    cfg.attrs = attr; cfg.numAttrs = g_dc_pdl ? 2 : 1;
    DC_CUDA(cudaLaunchKernelEx(&cfg, k_blocks_split<NT, EACH, T>, tmW, tmX, a));
    return DC_OK;
}
template <bool EACH, typename T>
int launch_split(const BlocksProduct& p, const SplitPlan& s, int kb, int early, int device, cudaStream_t stream)
{
    switch (s.NT) {
    case 16: return launch_split_as<16, EACH, T>(p, s, kb, early, device, stream);
    case 32: return launch_split_as<32, EACH, T>(p, s, kb, early, device, stream);
    case 64: return launch_split_as<64, EACH, T>(p, s, kb, early, device, stream);
    default: return launch_split_as<128, EACH, T>(p, s, kb, early, device, stream);
    }
}

template <bool PAIR, int BN, bool EACH, typename T>
int launch_blocks(const CUtensorMap& tmA, const CUtensorMap& tmB, const CUtensorMap& tmC, const BlocksTiles& a, int ctas, int device, cudaStream_t stream)
{
    static dc_once_per_device attr_set;
    DC_CUDA(attr_set.ensure(device, [] {
        return cudaFuncSetAttribute(k_blocks<PAIR, BN, EACH, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBlocksSmem);
    }));
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = PAIR ? 2 : 1; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas); cfg.blockDim = dim3(kBlocksThreads); cfg.dynamicSmemBytes = kBlocksSmem; cfg.stream = stream;
    cfg.attrs = g_dc_pdl ? attr : attr + 1; cfg.numAttrs = g_dc_pdl ? 2 : 1;
    DC_CUDA(cudaLaunchKernelEx(&cfg, k_blocks<PAIR, BN, EACH, T>, tmA, tmB, tmC, a));
    return DC_OK;
}

// early: b, its scales and bias are older than the kernel before, which waits for its own predecessor.
int launch_product(const BlocksProduct& p, int dtype, bool early, int device, int num_sms, cudaStream_t stream)
{
    BlocksTiles a = {};
    a.p = p;
    a.m_tiles = (int)((p.m + kTileM - 1) / kTileM);
    const int elt = dtype == DC_BF16 ? 2 : 4;
    a.kb = dc_div_up(p.k, kBytesK);
    bool pair = false;
    int BN = 64;
    double best = 0.0;
    // The tile that takes the fewest cycles, as counted from measurements: a block of K takes so many (what bounds it is its way from the MMAs to the sums and back), an SM's share of out leaves
    // at about 24 bytes a cycle where others pause, and an item costs 500 to begin and end.
    static constexpr double kStep[4][2] = {{1040.0, 1540.0}, {635.0, 800.0}, {635.0, 780.0}, {480.0, 540.0}};     // scales for 128 rows of b, for each
    for (int c = 0; c < 4; ++c) {
        const bool two = c < 2;
        const int bn = c == 0 ? 256 : c == 3 ? 64 : 128;
        const long long n_items = (two ? (a.m_tiles + 1) / 2 : a.m_tiles) * (long long)dc_div_up(p.n, bn), at_once = two ? num_sms / 2 : num_sms, rounds = (n_items + at_once - 1) / at_once;
        const double cost = rounds * (a.kb * kStep[c][p.b_block_rows == 1] + 128.0 * bn * elt / 24.0 + 500.0);
        if (c == 0 || cost < best) { best = cost; pair = two; BN = bn; }
    }
    if (p.n <= (1 << 20) && p.m <= (1 << 20)) {
        SplitPlan s;
        const int rc = split_plan(p, a.kb, device, &s);
        if (rc != DC_OK) return rc;
        if (s.CS > 1 && s.cost < best) {
            if (p.b_block_rows == 1) return dtype == DC_BF16 ? launch_split<true, __nv_bfloat16>(p, s, a.kb, early, device, stream) : launch_split<true, float>(p, s, a.kb, early, device, stream);
            return dtype == DC_BF16 ? launch_split<false, __nv_bfloat16>(p, s, a.kb, early, device, stream) : launch_split<false, float>(p, s, a.kb, early, device, stream);
        }
    }
    a.NB = dc_div_up(p.n, BN);
    a.limits = next_limits();
    const int b_rows = pair ? BN / 2 : BN;
    a.stage_bytes = kATile + b_rows * kBytesK;
    a.bufs = a.kb <= 8 ? 2 : 1;                               // long products take the room for operands
    a.stages = (kBlocksRoom - kAddWarps * kBox * a.bufs - (p.b_block_rows == 1 ? kEachBytes : kScaleBytes)) / a.stage_bytes;
    if (a.stages > kBlocksMostStages) a.stages = kBlocksMostStages;
    a.k_last = dc_div_up(p.k - (a.kb - 1) * kBytesK, 32);
    // float32 accumulators, both operands e4m3, K-major
    a.idesc = (1u << 4) | ((uint32_t)((BN > 128 ? 128 : BN) >> 3) << 17) | ((uint32_t)((pair ? 256 : 128) >> 4) << 24);
    a.wide = (uintptr_t)p.out % 16 == 0 && p.out_pitch % 16 == 0;
    CUtensorMap tmA, tmB, tmC = {};
    if (!encode_rows(&tmA, p.a, p.a_pitch, p.m, p.k, kTileM) || !encode_rows(&tmB, p.b, p.b_pitch, p.n, p.k, BN > 128 ? b_rows / 2 : b_rows)) return DC_ERR_CUDA;
    if (a.wide && (size_t)p.n * elt % 16 == 0) a.boxes = encode_out(&tmC, p.out, p.out_pitch, p.m, p.n, elt);
    const long long items = (pair ? (a.m_tiles + 1) / 2 : a.m_tiles) * (long long)a.NB, cap = pair ? num_sms / 2 : num_sms;
    if (items >= 0x70000000) return DC_ERR_LIMIT;
    const int ctas = (int)(items < cap ? items : cap) * (pair ? 2 : 1);
#define DC_BLOCKS(PAIR, BN, EACH, T) return launch_blocks<PAIR, BN, EACH, T>(tmA, tmB, tmC, a, ctas, device, stream)
#define DC_BLOCKS_OF(EACH, T) do { if (pair && BN == 256) DC_BLOCKS(true, 256, EACH, T); if (pair) DC_BLOCKS(true, 128, EACH, T); if (BN == 128) DC_BLOCKS(false, 128, EACH, T); DC_BLOCKS(false, 64, EACH, T); } while (0)
#define DC_BLOCKS_TO(T) do { if (p.b_block_rows == 1) DC_BLOCKS_OF(true, T); DC_BLOCKS_OF(false, T); } while (0)
    if (dtype == DC_BF16) DC_BLOCKS_TO(__nv_bfloat16);
    DC_BLOCKS_TO(float);
#undef DC_BLOCKS_TO
#undef DC_BLOCKS_OF
#undef DC_BLOCKS
}

template <typename T, bool WIDE>
int launch_quantize(const BlocksArgs& a, int device, int num_sms, cudaStream_t stream)
{
    const int64_t items = ((int64_t)a.rows + 3) / 4 * a.kb;
    // n / kb = n * by.x >> (32 + by.y) for n < 2^31, by.x the next whole number above 2^(32 + by.y) / kb, 2^by.y < kb
    uint2 by = make_uint2(0, 0);
    if (a.kb > 1) {
        while ((2 << by.y) < a.kb) ++by.y;
        by.x = (uint32_t)((((uint64_t)1 << (32 + by.y)) + a.kb - 1) / a.kb);
    }
    if (!a.qt && a.block_rows == 1 && items < 0x7fffffff) {
        DC_CUDA(dc_launch_pdl(k_quantize_row_blocks<T, WIDE>, dim3((unsigned)((items + 15) / 16)), 256, 0, stream, a, by, (uint32_t)items));
        return DC_OK;
    }
    if (a.qt && a.block_rows == 1 && 2 * (int64_t)a.kb * a.rb < 5 * (int64_t)num_sms) {
        const int rows = a.q ? (int)((items + 15) / 16) : 0;
        DC_CUDA(dc_launch_pdl(k_quantize_columns<T, WIDE>, dim3((unsigned)(rows + a.rb * dc_div_up(a.channels, 32))), 256, 0, stream, a, by, (uint32_t)items, rows));
        return DC_OK;
    }
    const int64_t tiles = (int64_t)a.kb * a.rb;
    if (tiles > 0x7fffffff) return DC_ERR_LIMIT;
    const size_t smem = 128 * 128 * sizeof(T);
    auto* const kernel = a.block_rows > 1 ? k_quantize_tile<T, WIDE, true> : k_quantize_tile<T, WIDE, false>;
    static dc_once_per_device set[2];
    DC_CUDA(set[a.block_rows > 1].ensure(device, [=] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem); }));
    DC_CUDA(dc_launch_pdl(kernel, dim3((unsigned)tiles), 256, smem, stream, a));
    return DC_OK;
}

int quantize(BlocksArgs& a, int dtype, int device, int num_sms, cudaStream_t stream)
{
    a.kb = dc_div_up(a.channels, 128); a.rb = (int)(((int64_t)a.rows + 127) / 128);
    const bool wide = (uintptr_t)a.x % 16 == 0 && (a.rows < 2 || a.x_pitch % 16 == 0) && a.channels % 8 == 0;
    if (dtype == DC_BF16) return wide ? launch_quantize<__nv_bfloat16, true>(a, device, num_sms, stream) : launch_quantize<__nv_bfloat16, false>(a, device, num_sms, stream);
    return wide ? launch_quantize<float, true>(a, device, num_sms, stream) : launch_quantize<float, false>(a, device, num_sms, stream);
}

constexpr int kMostTerms = 1 << 28;                           // columns, terms of a sum

bool floats_ok(const float* p) { return (uintptr_t)p % sizeof(float) == 0; }
bool bytes_ok(const uint8_t* q, size_t pitch, const float* scale, int64_t rows, int64_t columns)
{
    return q && scale && floats_ok(scale) && (uintptr_t)q % 16 == 0 && pitch % 16 == 0 && (rows < 2 || pitch >= (size_t)columns);
}
// What both products ask of their operands.
int product_check(const uint8_t* b, size_t b_pitch, const float* b_scale, int32_t b_block_rows, const float* bias, int64_t m, int32_t n, int32_t k, int32_t dtype, const void* out, size_t out_pitch)
{
    if ((dtype != DC_FP32 && dtype != DC_BF16) || (b_block_rows != 1 && b_block_rows != 128)) return DC_ERR_CONFIG;
    const int elt = dtype == DC_BF16 ? 2 : 4;
    if (m < 0 || n < 1 || k < 1) return DC_ERR_ARG;
    if (m > DC_MOST_ROWS || n > kMostTerms || k > kMostTerms || (n > 1 && b_pitch > kMostPitch)) return DC_ERR_LIMIT;
    if (m == 0) return DC_OK;
    if (!bytes_ok(b, b_pitch, b_scale, n, k) || !out) return DC_ERR_ARG;
    if (!floats_ok(bias) || (uintptr_t)out % elt || out_pitch % elt || (m > 1 && out_pitch < (size_t)n * elt)) return DC_ERR_ARG;
    return DC_OK;
}
size_t blocks_pitch(int64_t k) { return (size_t)(k + 15) / 16 * 16; }

}  // namespace

extern "C" {

int dc_quantize_blocks(const void* x_dev, size_t x_pitch, int64_t rows, int32_t channels, int32_t dtype, int32_t block_rows, uint8_t* q_dev, size_t q_pitch, float* scale_dev,
                       uint8_t* qt_dev, size_t qt_pitch, float* scale_t_dev, void* cuda_stream)
{
    if ((dtype != DC_FP32 && dtype != DC_BF16) || (block_rows != 1 && block_rows != 128)) return DC_ERR_CONFIG;
    const int elt = dtype == DC_BF16 ? 2 : 4;
    if (rows < 0 || channels < 1 || !q_dev != !scale_dev || !qt_dev != !scale_t_dev) return DC_ERR_ARG;
    if (channels > kMostTerms || rows > DC_MOST_ROWS || (rows > 1 && x_pitch > 0xffffffffu) || (q_dev && rows > 1 && q_pitch > kMostPitch) || (qt_dev && channels > 1 && qt_pitch > kMostPitch)) return DC_ERR_LIMIT;
    if (rows == 0 || (!q_dev && !qt_dev)) return DC_OK;
    if (!x_dev || (uintptr_t)x_dev % elt || x_pitch % elt || (rows > 1 && x_pitch < (size_t)channels * elt)) return DC_ERR_ARG;
    if ((q_dev && !bytes_ok(q_dev, q_pitch, scale_dev, rows, channels)) || (qt_dev && !bytes_ok(qt_dev, qt_pitch, scale_t_dev, channels, rows))) return DC_ERR_ARG;
    BlocksArgs a = {};
    a.x = x_dev; a.x_pitch = x_pitch; a.rows = (int)rows; a.channels = channels; a.block_rows = block_rows;
    a.q = q_dev; a.q_pitch = q_pitch; a.scale = scale_dev; a.qt = qt_dev; a.qt_pitch = qt_pitch; a.scale_t = scale_t_dev;
    int device = 0, sms = 0;
    const int rc = dc_current_device(&device, &sms);
    return rc != DC_OK ? rc : quantize(a, dtype, device, sms, (cudaStream_t)cuda_stream);
}

int dc_matmul_blocks(const uint8_t* a_dev, size_t a_pitch, const float* a_scale_dev, const uint8_t* b_dev, size_t b_pitch, const float* b_scale_dev, int32_t b_block_rows,
                     const float* bias_dev, int64_t m, int32_t n, int32_t k, int32_t relu, int32_t dtype, void* out_dev, size_t out_pitch, void* cuda_stream)
{
    int rc = product_check(b_dev, b_pitch, b_scale_dev, b_block_rows, bias_dev, m, n, k, dtype, out_dev, out_pitch);
    if (rc != DC_OK || m == 0) return rc;
    if (m > 1 && a_pitch > kMostPitch) return DC_ERR_LIMIT;
    if (!bytes_ok(a_dev, a_pitch, a_scale_dev, m, k)) return DC_ERR_ARG;
    int device = 0, sms = 0;
    if ((rc = dc_current_device(&device, &sms)) != DC_OK) return rc;
    const BlocksProduct p = {a_dev, a_pitch, a_scale_dev, b_dev, b_pitch, b_scale_dev, bias_dev, m, n, k, relu, b_block_rows, out_dev, out_pitch};
    return launch_product(p, dtype, false, device, sms, (cudaStream_t)cuda_stream);
}

int dc_debug_stall_next_blocks(int wait_ms, int blocks)
{
    if (wait_ms < 1 || wait_ms > 1000 || blocks < 0) return DC_ERR_ARG;
    g_stall = (uint64_t)wait_ms << 32 | (uint32_t)blocks;
    return DC_OK;
}

int dc_linear_blocks_workspace(int64_t m, int32_t k, size_t* bytes)
{
    if (m < 0 || k < 1 || !bytes) return DC_ERR_ARG;
    if (m > DC_MOST_ROWS || k > kMostTerms) return DC_ERR_LIMIT;
    *bytes = (size_t)m * (blocks_pitch(k) + sizeof(float) * dc_div_up(k, 128)) + 256;
    return DC_OK;
}

int dc_linear_blocks(const void* x_dev, size_t x_pitch, const uint8_t* w_dev, size_t w_pitch, const float* w_scale_dev, int32_t w_block_rows, const float* bias_dev, int64_t m, int32_t n,
                     int32_t k, int32_t relu, int32_t dtype, void* out_dev, size_t out_pitch, void* workspace_dev, size_t workspace_bytes, void* cuda_stream)
{
    int rc = product_check(w_dev, w_pitch, w_scale_dev, w_block_rows, bias_dev, m, n, k, dtype, out_dev, out_pitch);
    if (rc != DC_OK || m == 0) return rc;
    const int elt = dtype == DC_BF16 ? 2 : 4;
    size_t need = 0;
    dc_linear_blocks_workspace(m, k, &need);
    if (m > 1 && x_pitch > 0xffffffffu) return DC_ERR_LIMIT;
    if (!x_dev || (uintptr_t)x_dev % elt || x_pitch % elt || (m > 1 && x_pitch < (size_t)k * elt) || !workspace_dev || workspace_bytes < need) return DC_ERR_ARG;
    int device = 0, sms = 0;
    if ((rc = dc_current_device(&device, &sms)) != DC_OK) return rc;
    const size_t pitch = blocks_pitch(k);
    uint8_t* const q = (uint8_t*)(((uintptr_t)workspace_dev + 255) & ~(uintptr_t)255);
    float* const scale = (float*)(q + (size_t)m * pitch);
    BlocksArgs a = {};
    a.x = x_dev; a.x_pitch = x_pitch; a.rows = (int)m; a.channels = k; a.block_rows = 1; a.q = q; a.q_pitch = pitch; a.scale = scale;
    if ((rc = quantize(a, dtype, device, sms, (cudaStream_t)cuda_stream)) != DC_OK) return rc;
    const BlocksProduct p = {q, pitch, scale, w_dev, w_pitch, w_scale_dev, bias_dev, m, n, k, relu, w_block_rows, out_dev, out_pitch};
    return launch_product(p, dtype, true, device, sms, (cudaStream_t)cuda_stream);
}

}  // extern "C"
