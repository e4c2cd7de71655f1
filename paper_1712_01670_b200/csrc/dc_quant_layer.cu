// Layer normalisation and 8-bit convolutions as layers of a cache: DC_LAYER_NORM, DC_CONV_QUANT (kernels: dc_norm.cu, dc_quant.cu).
//
// A pointwise 8-bit convolution is a partial convolution like any other: its pixels in rectangles come from the cached map, tiles without a
// pixel left are not in the list, and of the others only the rest is computed.  Its input's rows in 8 bits lie in lines of a multiple of
// eight pixels, so that a flat tile (16 groups of 8 pixels of one line) is 128 rows one behind another whatever the map's width, and one box
// of a TMA load.  Rows of reused pixels are not put into 8 bits, but where the layer normalisation in front writes the rows: it normalises every pixel and puts every one
// into 8 bits.
#include "dc_rows.cuh"

namespace {
template <typename T>
int layer_alloc(dc_cache* c, T** p, size_t count)
{
    if (cudaMalloc((void**)p, count * sizeof(T)) != cudaSuccess) { cudaGetLastError(); return DC_ERR_ALLOC; }
    c->bytes += count * sizeof(T);
    return DC_OK;
}
int copy_floats(dc_cache* c, float** to, const float* from, size_t n)
{
    const int rc = layer_alloc(c, to, n);
    if (rc != DC_OK) return rc;
    DC_CUDA(cudaMemcpyAsync(*to, from, n * sizeof(float), cudaMemcpyDeviceToDevice, c->stream));
    return DC_OK;
}
}  // namespace

int dc_build_norm(dc_cache* c, int layer, const float* gamma, const float* beta)
{
    dc_layer_rt& L = c->L[layer];
    if ((size_t)c->S * L.d.out_h * L.d.out_w > (size_t)DC_MOST_ROWS) return DC_ERR_CONFIG;
    L.eps = 1e-5f;
    int rc = DC_OK;
    if (gamma) rc = copy_floats(c, (float**)&L.weight, gamma, L.d.cout);
    if (rc == DC_OK && beta) rc = copy_floats(c, &L.bias, beta, L.d.cout);
    return rc;
}

int dc_build_quant(dc_cache* c, int layer, const float* w, const float* b)
{
    dc_layer_rt& L = c->L[layer];
    const bool pointwise = dc_layer_cached(c, layer);
    const int k = L.d.kh * L.d.kw * L.d.cin;
    const size_t pitch = dc_quant_pitch(k);
    const size_t rows = pointwise ? (size_t)c->S * L.d.out_h * L.gpr * DC_TILE_W : (size_t)c->S;
    if (rows > (size_t)DC_MOST_ROWS || pitch > 0xffffffffu || (size_t)k * c->elt > 0xffffffffu) return DC_ERR_CONFIG;
    int rc = copy_floats(c, &L.bias, b, L.d.cout);
    if (rc == DC_OK) rc = layer_alloc(c, (int8_t**)&L.weight, pitch * L.d.cout);
    if (rc == DC_OK) rc = layer_alloc(c, &L.w_scale, (size_t)L.d.cout);
    if (rc == DC_OK) rc = layer_alloc(c, &L.q_rows, pitch * rows);
    if (rc == DC_OK) rc = layer_alloc(c, &L.q_scale, rows);
    if (rc != DC_OK) return rc;
    DC_CUDA(cudaMemsetAsync(L.q_rows, 0, pitch * rows, c->stream));            // the gaps behind lines are multiplied too, if never stored
    DC_CUDA(cudaMemsetAsync(L.q_scale, 0, rows * sizeof(float), c->stream));
    dc_rows_args a = {};
    a.x = w; a.x_pitch = (size_t)k * sizeof(float); a.rows = L.d.cout; a.channels = k;
    a.q = (int8_t*)L.weight; a.q_pitch = pitch; a.scale = L.w_scale;
    return dc_launch_rows(a, false, DC_FP32, c->num_sms, c->stream);
}

// The rows of a pointwise 8-bit convolution's input.
static void pixel_rows(const dc_layer_rt& L, dc_rows_args* a)
{
    a->q = L.q_rows; a->q_pitch = dc_quant_pitch(L.d.cin); a->scale = L.q_scale;
    a->width = L.d.out_w; a->padded = L.gpr * DC_TILE_W;
}

int dc_launch_norm(dc_cache* c, int layer, const void* in, void* out)
{
    dc_layer_rt& L = c->L[layer];
    dc_prof_scope ps(c, DC_ST_POINTWISE);
    dc_rows_args a = {};
    a.x = in; a.x_pitch = a.y_pitch = (size_t)L.d.cout * c->elt; a.gamma = (const float*)L.weight; a.beta = L.bias;
    a.rows = (int64_t)c->S * L.d.out_h * L.d.out_w; a.channels = L.d.cout; a.eps = L.eps; a.y = out;
    if (L.norm_feeds >= 0) pixel_rows(c->L[L.norm_feeds], &a);
    c->launches += 1;
    return dc_launch_rows(a, true, c->cfg.dtype, c->num_sms, c->stream);
}

// filled: the rows are there already (dc_launch_norm).  tile_list, tile_count, masks: the pixels to compute, or NULL: all.
int dc_launch_quant(dc_cache* c, int layer, const void* in, bool filled, void* out, const int32_t* tile_list, const int32_t* tile_count, const uint32_t* masks)
{
    dc_layer_rt& L = c->L[layer];
    const bool pointwise = dc_layer_cached(c, layer);
    const int k = L.d.kh * L.d.kw * L.d.cin;
    dc_prof_scope ps(c, DC_ST_CONV);
    dc_product_args p = {};
    p.a = L.q_rows; p.a_pitch = dc_quant_pitch(k); p.a_scale = L.q_scale; p.b = (const int8_t*)L.weight; p.b_pitch = p.a_pitch; p.b_scale = L.w_scale; p.bias = L.bias;
    p.n = L.d.cout; p.k = k; p.relu = L.d.relu; p.out = out; p.out_pitch = (size_t)L.d.cout * c->elt; p.status = c->status;
    p.early = 1;                                                                // weights are older than any frame
    p.m = pointwise ? (int64_t)c->S * L.d.out_h * L.gpr * DC_TILE_W : (int64_t)c->S;
    if (!pointwise && dc_few_pays(p.m, p.n, k)) {
        c->launches += 1;
        return dc_launch_few(p, in, (size_t)k * c->elt, c->cfg.dtype, c->device, c->num_sms, c->stream);
    }
    if (!filled) {
        dc_rows_args a = {};
        a.x = in; a.x_pitch = (size_t)k * c->elt; a.channels = k;
        a.rows = pointwise ? (int64_t)c->S * L.d.out_h * L.d.out_w : (int64_t)c->S;
        if (pointwise) pixel_rows(L, &a);
        else { a.q = L.q_rows; a.q_pitch = dc_quant_pitch(k); a.scale = L.q_scale; }
        a.masks = pointwise ? masks : nullptr;
        c->launches += 1;
        const int rc = dc_launch_rows(a, false, c->cfg.dtype, c->num_sms, c->stream);
        if (rc != DC_OK) return rc;
    }
    if (pointwise && (tile_list || L.gpr * DC_TILE_W != L.d.out_w)) {
        p.width = L.d.out_w; p.padded = L.gpr * DC_TILE_W;
        p.tile_list = tile_list; p.tile_count = tile_count; p.masks = masks; p.max_tiles = tile_list ? dc_layer_tiles(c, L) : 0;
    }
    c->launches += 1;
    return dc_launch_product(p, c->cfg.dtype, c->device, c->num_sms, c->stream);
}
