// Rows into a 4-bit prefix cache and back (format in mcsd.h).
//
// Both are streams: a row of one head is 2 d bytes of bf16 on one side and d / 2 + d / 32 on the other, with a handful of
// operations per number.  Lanes take eight channels each (16 bytes of bf16, 4 of codes), so a quad holds a group of 32 and its
// maximum needs two exchanges within the quad; consecutive rows of a workgroup are consecutive tokens of one head, whose codes
// and scales are neighbours in the cache while each of them is whole lines of the source.
//
// Bound by memory: 147200 rows of 128 channels stored take 18 to 24 us and loaded 16.6 to 20, by what the last-level cache holds of
// them (95 MB each: 4 to 5.7 TB/s, a large copy runs at 4.9), in fp32 34 and 38 us (171 MB); one row for each of 16 sequences takes
// 2.4 us either way, a launch.  One row per lane: with two, all requested
// before the first is used, the pair of calls takes 44.8 us instead of 43.1 there and 5.2 instead of 4.8 for 16 sequences of 16
// rows; with four 48.2 and 7.1.  Eight wavefronts per SIMD hide what there is to wait for.
#include "fp4_format.h"

namespace {

struct StoreParams {
    const void *k, *v;
    mcsd_fp4_cache_t cache;
    const int64_t *seq_base;
    const int32_t *first, *n_rows;
    int64_t batch_stride, src_head_stride, row_stride, head_stride;
    int32_t H, max_rows, capacity;
    RowDiv rows;
};

struct LoadParams {
    mcsd_fp4_cache_t cache[MCSD_COMMIT_MAX_LAYERS];
    void *k[MCSD_COMMIT_MAX_LAYERS], *v[MCSD_COMMIT_MAX_LAYERS];
    const int64_t *seq_base;
    const int32_t *first, *n_rows;
    int64_t batch_stride, dst_head_stride, row_stride, head_stride;
    int32_t H, max_rows, capacity;
    RowDiv rows;
};

template <bool F32>
__device__ __forceinline__ void read8(const void *base, int64_t at, float (&x)[8])
{
    if constexpr (F32) {
        const float4 a = ((const float4 *)((const float *)base + at))[0], b = ((const float4 *)((const float *)base + at))[1];
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
        const uint4 a = *(const uint4 *)((const uint16_t *)base + at);
        const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
}

// grid (rows of a sequence / rows per workgroup, B); row r of a sequence is token r % max_rows of head r / max_rows
template <int D, bool F32>
__global__ __launch_bounds__(256) void store_fp4_kernel(const StoreParams p)
{
    constexpr int LANES = D / 8, ROWS = 256 / LANES;
    const int b = blockIdx.y, c = threadIdx.x % LANES;
    const int n = min(max(p.n_rows[b], 0), p.max_rows);
    const int64_t first = p.first[b], base = p.seq_base[b];
    const int64_t r = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES;
    const int h = row_div((int)r, p.rows), t = (int)r - h * p.max_rows;
    const bool live = h < p.H && t < n && first + t >= 0 && first + t < p.capacity;
    const int64_t at = base + h * p.head_stride + (first + t) * D + c * 8;
    const int64_t src = b * p.batch_stride + h * p.src_head_stride + t * p.row_stride + c * 8;
    float k[8] = {}, v[8] = {};
    if (live) {
        read8<F32>(p.k, src, k);
        read8<F32>(p.v, src, v);
    }
    unsigned kb, vb;
    const unsigned kc = fp4_quantise8(k, kb), vc = fp4_quantise8(v, vb);
    if (live) {
        *(unsigned *)((char *)p.cache.k_codes + at / 2) = kc;
        *(unsigned *)((char *)p.cache.v_codes + at / 2) = vc;
        if ((c & 3) == 0) {
            ((unsigned char *)p.cache.k_scales)[at / 32] = (unsigned char)kb;
            ((unsigned char *)p.cache.v_scales)[at / 32] = (unsigned char)vb;
        }
    }
}

template <bool F32>
__device__ __forceinline__ void write8(void *base, int64_t at, unsigned codes, float scale)
{
    if constexpr (F32) {
        const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
        const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
        float4 *to = (float4 *)((float *)base + at);
        to[0] = make_float4(a[0], a[1], b[0], b[1]);
        to[1] = make_float4(c[0], c[1], d[0], d[1]);
    } else {
        *(uint4 *)((uint16_t *)base + at) = fp4x8_to_bf16(codes, scale);
    }
}

// grid (rows of a sequence / rows per workgroup, B, layers)
template <int D, bool F32>
__global__ __launch_bounds__(256) void load_fp4_kernel(const LoadParams p)
{
    constexpr int LANES = D / 8, ROWS = 256 / LANES;
    const int b = blockIdx.y, layer = blockIdx.z, c = threadIdx.x % LANES;
    const mcsd_fp4_cache_t cache = p.cache[layer];
    void *k = p.k[layer], *v = p.v[layer];
    const int n = min(max(p.n_rows[b], 0), p.max_rows);
    const int64_t first = p.first[b], base = p.seq_base[b];
    const int64_t r = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES;
    const int h = row_div((int)r, p.rows), t = (int)r - h * p.max_rows;
    if (h >= p.H || t >= n || first + t < 0 || first + t >= p.capacity) return;
    const int64_t to = b * p.batch_stride + h * p.dst_head_stride + t * p.row_stride + c * 8;
    const int64_t at = base + h * p.head_stride + (first + t) * D + c * 8;
    const unsigned kc = *(const unsigned *)((const char *)cache.k_codes + at / 2), vc = *(const unsigned *)((const char *)cache.v_codes + at / 2);
    const float ks = fp4_scale(((const unsigned char *)cache.k_scales)[at / 32]), vs = fp4_scale(((const unsigned char *)cache.v_scales)[at / 32]);
    write8<F32>(k, to, kc, ks);
    write8<F32>(v, to, vc, vs);
}

// What both entry points refuse; `grid_x` are the workgroups for the rows of one sequence.
int check_rows(mcsd_dtype_t dtype, int32_t B, int32_t H, int32_t d, int32_t max_rows, int64_t batch_stride, int64_t other_head_stride,
               int64_t row_stride, const int32_t *first, const int32_t *n_rows, const int64_t *seq_base, int64_t head_stride, int32_t capacity,
               unsigned &grid_x)
{
    if (!first || !n_rows || !seq_base) return MCSD_EINVAL;
    if (dtype != MCSD_F32 && dtype != MCSD_BF16) return MCSD_EINVAL;
    if (B < 1 || B > 65535 || H < 1 || H > 65535 || max_rows < 0 || capacity < 0) return MCSD_EINVAL;
    if (batch_stride < 0 || other_head_stride < 0 || row_stride < 0 || head_stride < 0) return MCSD_EINVAL;
    if (((batch_stride | other_head_stride | row_stride) & 7) || (head_stride & 127)) return MCSD_EINVAL;
    if (d != 64 && d != 128) return MCSD_EUNSUPPORTED;
    const int64_t rows = (int64_t)max_rows * H, per_wg = 256 / (d / 8);
    if ((rows + per_wg - 1) / per_wg > MCSD_MAX_GRID_256) return MCSD_EUNSUPPORTED;
    grid_x = (unsigned)((rows + per_wg - 1) / per_wg);
    return MCSD_OK;
}

}  // namespace

extern "C" int mcsd_store_fp4kv(mcsd_dtype_t dtype, int32_t B, int32_t H, int32_t d, int32_t max_rows, const void *k, const void *v,
                                int64_t batch_stride, int64_t src_head_stride, int64_t row_stride, const int32_t *first_row_dev,
                                const int32_t *n_rows_dev, const mcsd_fp4_cache_t *cache, const int64_t *seq_base_dev,
                                int64_t head_stride, int32_t capacity, void *hip_stream)
{
    if (!k || !v || !fp4_cache_ok(cache) || (((uintptr_t)k | (uintptr_t)v) & 15)) return MCSD_EINVAL;
    unsigned grid_x = 0;
    const int rc = check_rows(dtype, B, H, d, max_rows, batch_stride, src_head_stride, row_stride, first_row_dev, n_rows_dev, seq_base_dev,
                              head_stride, capacity, grid_x);
    if (rc != MCSD_OK || max_rows == 0) return rc;
    StoreParams p;
    p.k = k; p.v = v; p.cache = *cache; p.seq_base = seq_base_dev; p.first = first_row_dev; p.n_rows = n_rows_dev;
    p.batch_stride = batch_stride; p.src_head_stride = src_head_stride; p.row_stride = row_stride; p.head_stride = head_stride;
    p.H = H; p.max_rows = max_rows; p.capacity = capacity; p.rows = row_div_of((uint32_t)max_rows);
    const bool f32 = dtype == MCSD_F32;
    auto kernel = d == 128 ? (f32 ? store_fp4_kernel<128, true> : store_fp4_kernel<128, false>)
                           : (f32 ? store_fp4_kernel<64, true> : store_fp4_kernel<64, false>);
    hipLaunchKernelGGL(kernel, dim3(grid_x, B), dim3(256), 0, (hipStream_t)hip_stream, p);
    return mcsd_hip_status(hipGetLastError());
}

extern "C" int mcsd_load_fp4kv(mcsd_dtype_t dtype, int32_t B, int32_t H, int32_t d, int32_t n_layers, int32_t max_rows,
                               const mcsd_fp4_cache_t *caches, const int64_t *seq_base_dev, int64_t head_stride, int32_t capacity,
                               const int32_t *first_row_dev, const int32_t *n_rows_dev, void *const *k, void *const *v,
                               int64_t batch_stride, int64_t dst_head_stride, int64_t row_stride, void *hip_stream)
{
    if (!caches || !k || !v || n_layers < 1) return MCSD_EINVAL;
    unsigned grid_x = 0;
    const int rc = check_rows(dtype, B, H, d, max_rows, batch_stride, dst_head_stride, row_stride, first_row_dev, n_rows_dev, seq_base_dev,
                              head_stride, capacity, grid_x);
    if (rc != MCSD_OK) return rc;
    // (a tensor expanded over one of its dimensions would be written by several rows at once)
    if ((B > 1 && batch_stride < d) || (H > 1 && dst_head_stride < d) || (max_rows > 1 && row_stride < d)) return MCSD_EINVAL;
    if (n_layers > MCSD_COMMIT_MAX_LAYERS) return MCSD_EUNSUPPORTED;
    LoadParams p;
    for (int l = 0; l < MCSD_COMMIT_MAX_LAYERS; ++l) {
        p.cache[l] = mcsd_fp4_cache_t();
        p.k[l] = p.v[l] = nullptr;
    }
    for (int l = 0; l < n_layers; ++l) {
        if (!k[l] || !v[l] || !fp4_cache_ok(&caches[l]) || (((uintptr_t)k[l] | (uintptr_t)v[l]) & 15)) return MCSD_EINVAL;
        p.cache[l] = caches[l]; p.k[l] = k[l]; p.v[l] = v[l];
    }
    if (max_rows == 0) return MCSD_OK;
    p.seq_base = seq_base_dev; p.first = first_row_dev; p.n_rows = n_rows_dev;
    p.batch_stride = batch_stride; p.dst_head_stride = dst_head_stride; p.row_stride = row_stride; p.head_stride = head_stride;
    p.H = H; p.max_rows = max_rows; p.capacity = capacity; p.rows = row_div_of((uint32_t)max_rows);
    const bool f32 = dtype == MCSD_F32;
    auto kernel = d == 128 ? (f32 ? load_fp4_kernel<128, true> : load_fp4_kernel<128, false>)
                           : (f32 ? load_fp4_kernel<64, true> : load_fp4_kernel<64, false>);
    hipLaunchKernelGGL(kernel, dim3(grid_x, B, n_layers), dim3(256), 0, (hipStream_t)hip_stream, p);
    return mcsd_hip_status(hipGetLastError());
}
