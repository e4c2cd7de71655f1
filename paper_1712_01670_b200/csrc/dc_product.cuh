// Building blocks of the products of 8-bit rows (dc_quant.cu: integers, dc_blocks.cu: floating point): operand tiles of 128 rows x 128 bytes by TMA, CTA pairs,
// output tiles as boxes.
#pragma once
#include <atomic>

#include "dc_rows.cuh"
#include "dc_tcgen05.cuh"

namespace {

constexpr unsigned long long kWaitNs = 2000000000ull;        // every wait on the device
constexpr int kBytesK = 128;                                  // a stage: 128 values of K
constexpr int kTileM = 128, kATile = kTileM * kBytesK;
constexpr size_t kMostPitch = ((size_t)1 << 40) - 16;          // of operands: what a tensor map takes

__device__ __forceinline__ void load_pair(uint32_t dst, const CUtensorMap* tm, int c0, int c1, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(tm), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void commit_pair(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
// ReLU or nothing; a NaN stays.
template <bool RELU> __device__ __forceinline__ float clamped(float v)
{
    if (RELU) asm("max.NaN.f32 %0, %0, 0f00000000;" : "+f"(v));
    return v;
}
template <bool RELU> __device__ __forceinline__ uint32_t two_bf16(float2 a)
{
    uint32_t r;
    if (RELU) asm("cvt.rn.relu.bf16x2.f32 %0, %2, %1;" : "=r"(r) : "f"(a.x), "f"(a.y));
    else asm("cvt.rn.bf16x2.f32 %0, %2, %1;" : "=r"(r) : "f"(a.x), "f"(a.y));
    return r;
}
// A warp's staged 32 rows of 64 bytes on their way to out; lane 0 issues.
__device__ __forceinline__ void store_box(const CUtensorMap* tm, uint32_t stage, int col, int row)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(tm), "r"(stage), "r"(col), "r"(row) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
__device__ __forceinline__ void store_read(int bufs)          // the place that comes next is free
{
    if (bufs == 2) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
    else asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
}
__device__ __forceinline__ void store_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                             CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encode_fn()
{
    static std::atomic<EncodeFn> known;
    EncodeFn fn = known.load(std::memory_order_relaxed);
    if (!fn) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess) known.store(fn = (EncodeFn)p, std::memory_order_relaxed);
        cudaGetLastError();
    }
    return fn;
}

// Rows of 8-bit values in boxes of box_rows x 128 bytes; zeros beyond the last row and the last value.
bool encode_rows(CUtensorMap* tm, const void* base, size_t pitch, int64_t rows, int k, int box_rows)
{
    EncodeFn enc = encode_fn();
    if (!enc) return false;
    if (rows < 2) pitch = dc_quant_pitch(k);                                   // a single row's is anything
    const cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)pitch};
    const cuuint32_t box[2] = {(cuuint32_t)kBytesK, (cuuint32_t)box_rows}, elem[2] = {1, 1};
    return enc(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, (void*)base, dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// out [m][n] in boxes of 32 rows x 64 bytes; rows of whole 16 bytes, beyond which nothing is written, nor beyond the last row.
bool encode_out(CUtensorMap* tm, void* out, size_t out_pitch, int64_t m, int n, int elt)
{
    const size_t pitch = m < 2 ? ((size_t)n * elt + 15) / 16 * 16 : out_pitch;
    const cuuint64_t dims[2] = {(cuuint64_t)n, (cuuint64_t)m}, strides[1] = {(cuuint64_t)pitch};
    const cuuint32_t box[2] = {(cuuint32_t)(64 / elt), 32}, elem[2] = {1, 1};
    return encode_fn()(tm, elt == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, out, dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B,
                       CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace
