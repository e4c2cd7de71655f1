// Rows of channels: layer normalisation, and rows in 8 bits with a scale of their own (dc_norm.cu), and the products of such
// rows (dc_quant.cu).  The layers DC_LAYER_NORM and DC_CONV_QUANT and the entry points of the same names call these.
#pragma once
#include "dc_common.cuh"

// Most rows of a call (the kernels count rows in 32 bits, a grid's step ahead).  Pitches are below 2^32 where there are two rows or more.
#define DC_MOST_ROWS 0x7ff00000

// Rows [rows][channels] to be normalised (norm), quantised (q) or both.  Pitches in bytes.
struct dc_rows_args {
    const void* x; size_t x_pitch;
    const float *gamma, *beta;          // or NULL: ones, zeros
    int64_t rows; int channels;
    float eps;
    void* y; size_t y_pitch;            // or NULL
    float *mean, *rstd;                 // or NULL
    int8_t* q; size_t q_pitch; float* scale;   // or NULL
    // Pixels of maps of `width` columns, of which each image row begins at a multiple of `padded` rows of q and scale; 0: dense
    int width, padded;
    const uint32_t* masks;              // of such pixels, those that are not wanted: a bit for each row of q, 128 to a tile; or NULL
};
// norm: false: the rows are quantised as they are.  One kernel.
int dc_launch_rows(const dc_rows_args& a, bool norm, int dtype, int num_sms, cudaStream_t stream);

// out[r][j] = relu(a_scale[r] * b_scale[j] * sum_k a[r][k] b[j][k] + bias[j])
struct dc_product_args {
    const int8_t* a; size_t a_pitch; const float* a_scale;
    const int8_t* b; size_t b_pitch; const float* b_scale;
    const float* bias;                  // or NULL
    int64_t m; int n, k, relu;
    void* out; size_t out_pitch;
    int32_t* status;                    // device status word, or NULL
    int early;                          // 1: the weights (b, b_scale, bias) are older than the kernel before, which waits for its own predecessor
    // Pixels of maps (padded > 0; else every row): tiles of 128 rows of a, `padded` rows per line of `width` pixels; tile_list, masks: of a
    // partial convolution, or NULL
    const int32_t *tile_list, *tile_count; const uint32_t* masks;
    int width, padded, max_tiles;
};
int dc_launch_product(const dc_product_args& a, int dtype, int device, int num_sms, cudaStream_t stream);

// The same for one row or a few short ones, given as the map has them (p.a and p.a_scale are not used), in one launch (dc_few.cu).
#define DC_FEW_BYTES (200 * 1024)        // shared memory for them
bool dc_few_pays(int64_t m, int n, int k);
int dc_launch_few(const dc_product_args& p, const void* x, size_t x_pitch, int dtype, int device, int num_sms, cudaStream_t stream);

static inline size_t dc_quant_pitch(int64_t k) { return (size_t)(k + 15) / 16 * 16; }
// The device that is current, and its number of SMs (looked up once per device).
int dc_current_device(int* device, int* num_sms);
