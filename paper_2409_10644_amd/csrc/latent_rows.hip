// Rows of a latent cache, and the rotated part of the queries that meet them (formulas in mcsd.h): norm of a token's latent vector,
// rotation by position of its last d_rope channels and of the queries', in one pass over the projections' output.
//
// A stream: every element is read and written once.  A wavefront has a latent row, eight channels a lane: the sum of squares is an
// exchange between its lanes.  Sines and cosines of a row serve the latent and all query heads; each is computed by the thread that
// needs it first and shared through LDS.  Angles are products in binary64, reduced to a fraction of a turn there, so position 10^6
// is as exact as position 1.  Squares are summed in fp32, of a scaled vector where its size asks for it.
#include "fp4_format.h"

namespace {

struct LatentRowsParams {
    const void *q, *kv;
    uint16_t *q_out, *out;               // (out: tree rows [B][out_row][D], or the cache)
    const float *inv_freq, *weight;
    const int32_t *first, *n_rows;       // tree: prefix lengths, null
    const int64_t *seq_base;             // cache: where sequences begin, else null
    int64_t q_batch, q_row, q_head, kv_batch, kv_row, out_row;    // (strides in elements; out_row: rows per sequence or head of the outputs)
    float eps;
    int32_t rotary, interleaved, H, rows, row0, max_prefix, capacity;
    int32_t gamma;                       // > 0: rows are tree nodes row0 ..
    int32_t off[MCSD_MAX_LEVELS];        // first node of every level
};

template <bool F32>
__device__ __forceinline__ void load8(const void *base, int64_t at, float (&x)[8])
{
    if constexpr (F32) {
        const float4 a = ((const float4 *)((const float *)base + at))[0], b = ((const float4 *)((const float *)base + at))[1];
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
        const uint4 a = *(const uint4 *)((const uint16_t *)base + at);
        const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
}

__device__ __forceinline__ void store8(uint16_t *dst, const float (&x)[8])
{
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(unsigned, (bf16x2){(__bf16)x[2 * i], (__bf16)x[2 * i + 1]});
    *(uint4 *)dst = make_uint4(w[0], w[1], w[2], w[3]);
}

// Over the wavefront's lanes.
__device__ __forceinline__ float wave_sum(float v)
{
    v += __uint_as_float(dpp_move<DPP_XOR1>(__float_as_uint(v)));
    v += __uint_as_float(dpp_move<DPP_XOR2>(__float_as_uint(v)));
    v += __uint_as_float(dpp_move<DPP_HALF_MIRROR>(__float_as_uint(v)));
    v += __uint_as_float(dpp_move<0x140>(__float_as_uint(v)));            // mirror of 16
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Eight rotated channels from c on of a vector of DR whose channels are at base + at (those from `rotary` on stay as they are).
template <int DR, bool F32>
__device__ __forceinline__ void rotate8(const void *base, int64_t at, int c, const float *cosines, const float *sines, const LatentRowsParams &p, float (&x)[8])
{
    load8<F32>(base, at + c, x);
    if (c >= p.rotary) return;
    if (p.interleaved) {                                                   // (which product is rounded first is written out: every build gives the same bits)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float co = cosines[c / 2 + j], si = sines[c / 2 + j], u = x[2 * j], v = x[2 * j + 1];
            x[2 * j] = fmaf(u, co, -(v * si));
            x[2 * j + 1] = fmaf(v, co, u * si);
        }
    } else {
        const int half = p.rotary / 2;
        const bool low = c < half;
        float y[8];
        load8<F32>(base, at + (low ? c + half : c - half), y);             // the pairs' other ends
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int f = (low ? c : c - half) + j;
            const float co = cosines[f], si = sines[f];
            x[j] = low ? fmaf(x[j], co, -(y[j] * si)) : fmaf(x[j], co, y[j] * si);
        }
    }
}

// grid (rows / R, B), 256 threads
template <int DL, int DR, bool F32, int R>
__global__ __launch_bounds__(256) void latent_rows_kernel(const LatentRowsParams p)
{
    constexpr int D = DL + DR;
    __shared__ float s_cos[R][DR / 2], s_sin[R][DR / 2];
    const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, t0 = blockIdx.x * R;
    const int n = p.n_rows ? min(max(p.n_rows[b], 0), p.rows) : p.rows;
    if (t0 >= n) return;
    const int first = p.first[b], half = p.rotary / 2;
    for (int i = tid; i < R * half; i += 256) {
        const int row = R == 1 ? 0 : i / half, f = i - row * half;
        int64_t pos;
        if (p.gamma > 0) {
            const int node = p.row0 + t0 + row;
            int level = 0;
            for (int l = 0; l < p.gamma; ++l) level += node >= p.off[l];
            pos = (int64_t)min(max(first, 0), p.max_prefix) + level - 1;
        } else {
            pos = (int64_t)first + t0 + row;
        }
        const double turns = (double)pos * (double)p.inv_freq[f] * 0.15915494309189533577;
        float s, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
        s_cos[row][f] = c;
        s_sin[row][f] = s;
    }
    __syncthreads();
    // the latent rows, one per wavefront at a time
    for (int row = wave; row < R && t0 + row < n; row += 4) {
        const int t = t0 + row;
        const int64_t src = b * p.kv_batch + t * p.kv_row;
        uint16_t *dst;
        if (p.seq_base) {
            const int64_t at = (int64_t)first + t;
            if (at < 0 || at >= p.capacity) continue;
            dst = p.out + p.seq_base[b] + at * D;
        } else {
            dst = p.out + ((int64_t)b * p.out_row + p.row0 + t) * D;
        }
        float x[8], y[8];
        const bool has = DL == 512 || lane < DL / 8, turns = lane < DR / 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = 0.f;
        if (has) load8<F32>(p.kv, src + lane * 8, x);
        if (turns) rotate8<DR, F32>(p.kv, src + DL, lane * 8, s_cos[row], s_sin[row], p, y);
        if (p.weight) {
            const auto mean_square = [&]() __attribute__((always_inline)) {
                float ss = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) ss = fmaf(x[j], x[j], ss);
                return wave_sum(ss) * (1.f / DL);
            };
            float mean = mean_square() + p.eps;
            // Beyond fp32, or so small that squares were below it: the same of the vector times 2^-70 (512 squares of the largest
            // number are below 2^125 then) or 2^100, which the norm takes out again.
            if (__builtin_expect(!(mean >= 0x1p-100f && mean < INFINITY), 0)) {
                const float by = mean < 1.f ? 0x1p100f : 0x1p-70f;
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] *= by;
                mean = mean_square() + p.eps * by * by;
            }
            const float inv = 1.f / sqrtf(mean);
            float wt[8];
            if (has) {
                load8<true>(p.weight, lane * 8, wt);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = x[j] * inv * wt[j];
            }
        }
        if (has) store8(dst + lane * 8, x);
        if (turns) store8(dst + DL + lane * 8, y);
    }
    // the queries' rotated channels
    if (p.q) {
        constexpr int LANES = DR / 8;
        for (int i = tid; i < R * p.H * LANES; i += 256) {
            const int c = i % LANES, v = i / LANES, row = R == 1 ? 0 : v / p.H, h = v - row * p.H, t = t0 + row;
            if (t >= n) break;
            float x[8];
            rotate8<DR, F32>(p.q, b * p.q_batch + t * p.q_row + h * p.q_head, c * 8, s_cos[row], s_sin[row], p, x);
            store8(p.q_out + (((int64_t)b * p.H + h) * p.out_row + p.row0 + t) * D + DL + c * 8, x);
        }
    }
}

template <int DL, int DR>
void launch(const LatentRowsParams &p, bool f32, int32_t B, hipStream_t st)
{
    if (p.q) {
        auto kernel = f32 ? latent_rows_kernel<DL, DR, true, 1> : latent_rows_kernel<DL, DR, false, 1>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)p.rows, B), dim3(256), 0, st, p);
    } else {
        auto kernel = f32 ? latent_rows_kernel<DL, DR, true, 4> : latent_rows_kernel<DL, DR, false, 4>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((p.rows + 3) / 4), B), dim3(256), 0, st, p);
    }
}

// What both calls check; the strides of queries are zero where there are none.
int rows_call(LatentRowsParams &p, mcsd_dtype_t dtype, int32_t B, int32_t d_latent, int32_t d_rope, const mcsd_rope_t *rope, void *hip_stream)
{
    if (!p.kv || !p.out || !rope || !p.first) return MCSD_EINVAL;
    if (dtype != MCSD_F32 && dtype != MCSD_BF16) return MCSD_EINVAL;
    if (B < 1 || B > 65535 || p.rows < 0) return MCSD_EINVAL;
    if (p.q_batch < 0 || p.q_row < 0 || p.q_head < 0 || p.kv_batch < 0 || p.kv_row < 0) return MCSD_EINVAL;
    if ((p.q_batch | p.q_row | p.q_head | p.kv_batch | p.kv_row) & 7) return MCSD_EINVAL;
    if (((uintptr_t)p.q | (uintptr_t)p.kv | (uintptr_t)p.q_out | (uintptr_t)p.out | (uintptr_t)rope->k_weight) & 15) return MCSD_EINVAL;
    if (!(rope->eps >= 0.f) || rope->eps > 3.4e38f || rope->rotary_dim < 0 || (rope->rotary_dim & 15) || rope->q_weight) return MCSD_EINVAL;
    if (rope->rotary_dim > 0 && !rope->inv_freq) return MCSD_EINVAL;
    if (!((d_latent == 512 && d_rope == 64) || (d_latent == 256 && d_rope == 32))) return MCSD_EUNSUPPORTED;
    if (rope->rotary_dim > d_rope) return MCSD_EINVAL;
    if (p.rows > MCSD_MAX_GRID_256) return MCSD_EUNSUPPORTED;
    if (p.rows == 0) return MCSD_OK;
    p.inv_freq = rope->inv_freq; p.weight = rope->k_weight; p.eps = rope->eps;
    p.rotary = rope->rotary_dim; p.interleaved = rope->interleaved != 0;
    if (d_latent == 512) launch<512, 64>(p, dtype == MCSD_F32, B, (hipStream_t)hip_stream);
    else launch<256, 32>(p, dtype == MCSD_F32, B, (hipStream_t)hip_stream);
    return mcsd_hip_status(hipGetLastError());
}

}  // namespace

extern "C" int mcsd_tree_latent_norm_rope(const mcsd_mask_view_t *mask, mcsd_dtype_t dtype, int32_t B, int32_t H, int32_t d_latent,
                                          int32_t d_rope, int32_t row_begin, const void *q_in, const void *kv_in, int64_t q_batch_stride,
                                          int64_t q_row_stride, int64_t q_head_stride, int64_t kv_batch_stride, int64_t kv_row_stride,
                                          const mcsd_rope_t *rope, const int32_t *prefix_lens_dev, int32_t max_prefix, void *q_out,
                                          void *latent_out, int64_t node_stride, void *hip_stream)
{
    if (!mask || mask->gamma < 1 || mask->gamma > MCSD_MAX_LEVELS || !mask->level_off_host || mask->n_nodes < 1) return MCSD_EINVAL;
    if (row_begin < 0 || row_begin >= mask->n_nodes || node_stride < mask->n_nodes || max_prefix < 0) return MCSD_EINVAL;
    if (!q_in || !q_out || H < 1 || H > 65535) return MCSD_EINVAL;
    LatentRowsParams p = {};
    p.q = q_in; p.kv = kv_in; p.q_out = (uint16_t *)q_out; p.out = (uint16_t *)latent_out;
    p.first = prefix_lens_dev; p.max_prefix = max_prefix;
    p.q_batch = q_batch_stride; p.q_row = q_row_stride; p.q_head = q_head_stride; p.kv_batch = kv_batch_stride; p.kv_row = kv_row_stride;
    p.out_row = node_stride; p.H = H; p.rows = mask->n_nodes - row_begin; p.row0 = row_begin;
    p.gamma = mask->gamma;
    for (int l = 0; l < mask->gamma; ++l) p.off[l] = mask->level_off_host[l];
    return rows_call(p, dtype, B, d_latent, d_rope, rope, hip_stream);
}

extern "C" int mcsd_store_latent(mcsd_dtype_t dtype, int32_t B, int32_t d_latent, int32_t d_rope, int32_t max_rows, const void *kv_in,
                                 int64_t kv_batch_stride, int64_t kv_row_stride, const mcsd_rope_t *rope, const int32_t *first_row_dev,
                                 const int32_t *n_rows_dev, void *cache, const int64_t *seq_base_dev, int32_t capacity, void *hip_stream)
{
    if (!n_rows_dev || !seq_base_dev || capacity < 0) return MCSD_EINVAL;
    LatentRowsParams p = {};
    p.kv = kv_in; p.out = (uint16_t *)cache; p.first = first_row_dev; p.n_rows = n_rows_dev; p.seq_base = seq_base_dev;
    p.kv_batch = kv_batch_stride; p.kv_row = kv_row_stride; p.rows = max_rows; p.capacity = capacity;
    return rows_call(p, dtype, B, d_latent, d_rope, rope, hip_stream);
}
