// Norm and rotation of queries and keys, from the projections' layout [B][row][head][d] to the attention's [B][head][row][d], in
// one pass (formulas in mcsd.h).
//
// A stream: every element is read and written once.  A vector (one row's head) is held by d / 16 lanes, 16 channels each in two
// pieces of eight: the pieces are chosen so that a lane holds both ends of the pairs it rotates, and the sum of squares takes two
// or three exchanges between neighbouring lanes.  The sines and cosines of a row serve all its heads: they are computed once per
// workgroup, one angle per lane, and shared through LDS.  Angles are products in binary64, reduced to a fraction of a turn there,
// so position 10^6 is as exact as position 1.  Squares are summed in fp32, of a scaled vector where its size asks for it.
//
// Bound by memory: prompts of 500 to 2000 tokens of 48 heads of 128 channels in bf16 (123 MB read and written) take 26 to 28 us,
// 4.4 to 4.7 TB/s where a large copy runs at 4.9; the 44 tree nodes of one sequence take 4.3 us, a launch and two trips to memory.
#include "fp4_format.h"

namespace {

struct QkParams {
    const void *q, *k, *v;
    void *q_out, *k_out, *v_out;
    const float *inv_freq, *wq, *wk;
    const int32_t *first, *n_rows;       // tree: prefix lengths, null
    int64_t q_batch, q_row, kv_batch, kv_row, out_row;    // (strides in elements; out_row: rows per head of the outputs)
    float eps;
    int32_t rotary, interleaved;
    int32_t H_q, H_kv, heads;            // heads: H_q + H_kv, and H_kv more where there are values to move
    int32_t rows, row0, max_prefix;
    int32_t gamma;                       // > 0: rows are tree nodes row0 ..
    int32_t off[MCSD_MAX_LEVELS];        // first node of every level
    RowDiv by_heads;
};

template <bool F32>
struct Piece {                           // eight channels as they are in memory
    uint4 a, b;
    __device__ __forceinline__ void load(const void *base, int64_t at)
    {
        if constexpr (F32) { a = ((const uint4 *)((const float *)base + at))[0]; b = ((const uint4 *)((const float *)base + at))[1]; }
        else a = *(const uint4 *)((const uint16_t *)base + at);
    }
    __device__ __forceinline__ void store(void *base, int64_t at) const
    {
        if constexpr (F32) { ((uint4 *)((float *)base + at))[0] = a; ((uint4 *)((float *)base + at))[1] = b; }
        else *(uint4 *)((uint16_t *)base + at) = a;
    }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
        const unsigned w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x[i] = F32 ? __uint_as_float(w[i]) : __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
    __device__ __forceinline__ void set(const float (&x)[8])
    {
        unsigned w[8];
        if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(x[i]);
            b = make_uint4(w[4], w[5], w[6], w[7]);
        } else {
            typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(unsigned, (bf16x2){(__bf16)x[2 * i], (__bf16)x[2 * i + 1]});
        }
        a = make_uint4(w[0], w[1], w[2], w[3]);
    }
};

// grid (rows / R, B): R rows per workgroup
template <int D, bool F32, int R>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(const QkParams p)
{
    constexpr int LANES = D / 16, VECS = 256 / LANES;
    __shared__ __align__(16) float s_cos[R][D / 2], s_sin[R][D / 2], s_w[2][D];
    const int b = blockIdx.y, tid = threadIdx.x, t0 = blockIdx.x * R;
    const int n = p.n_rows ? min(max(p.n_rows[b], 0), p.rows) : p.rows;
    if (t0 >= n) return;
    const int first = p.first[b], half = p.rotary / 2;
    if (tid < D) {
        if (p.wq) s_w[0][tid] = p.wq[tid];
        if (p.wk) s_w[1][tid] = p.wk[tid];
    }
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
    const int c = tid % LANES, pairs = p.rotary / 16;
    // pieces of eight channels: a lane of the rotated part holds piece c and the one half the rotated part further on
    const int pa = c < pairs ? c : 2 * pairs + 2 * (c - pairs), pb = c < pairs ? c + pairs : pa + 1;
    for (int i = tid / LANES; i < R * p.heads; i += VECS) {
        const int row = R == 1 ? 0 : row_div(i, p.by_heads), h = i - row * p.heads, t = t0 + row;
        if (t >= n) break;
        const bool is_q = h < p.H_q, is_v = h >= p.H_q + p.H_kv;
        const int head = is_q ? h : is_v ? h - p.H_q - p.H_kv : h - p.H_q;
        const void *in = is_q ? p.q : is_v ? p.v : p.k;
        void *out = is_q ? p.q_out : is_v ? p.v_out : p.k_out;
        const int64_t src = is_q ? b * p.q_batch + t * p.q_row + head * D : b * p.kv_batch + t * p.kv_row + head * D;
        const int64_t dst = (((int64_t)b * (is_q ? p.H_q : p.H_kv) + head) * p.out_row + p.row0 + t) * D;
        Piece<F32> A, B;
        A.load(in, src + pa * 8);
        B.load(in, src + pb * 8);
        if (!is_v) {
            float x[8], y[8];
            A.get(x);
            B.get(y);
            const float *w = is_q ? p.wq : p.wk;
            if (w) {
                const float *sw = s_w[is_q ? 0 : 1];
                const auto mean_square = [&]() __attribute__((always_inline)) {
                    float ss = 0.f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) ss = fmaf(x[j], x[j], fmaf(y[j], y[j], ss));
                    ss += __uint_as_float(dpp_move<DPP_XOR1>(__float_as_uint(ss)));
                    ss += __uint_as_float(dpp_move<DPP_XOR2>(__float_as_uint(ss)));
                    if (LANES == 8) ss += __uint_as_float(dpp_move<DPP_HALF_MIRROR>(__float_as_uint(ss)));
                    return ss * (1.f / D);
                };
                float mean = mean_square() + p.eps;
                // Beyond fp32, or so small that squares were below it: the same of the vector times 2^-68 (128 squares of the largest
                // number are below 2^128 then) or 2^100, which the norm takes out again.  (The condition is that of all the vector's
                // lanes.)
                if (__builtin_expect(!(mean >= 0x1p-100f && mean < INFINITY), 0)) {
                    const float by = mean < 1.f ? 0x1p100f : 0x1p-68f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        x[j] *= by;
                        y[j] *= by;
                    }
                    mean = mean_square() + p.eps * by * by;
                }
                const float inv = 1.f / sqrtf(mean);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    x[j] = x[j] * inv * sw[pa * 8 + j];
                    y[j] = y[j] * inv * sw[pb * 8 + j];
                }
            }
            if (c < pairs) {                                           // (which product is rounded first is written out: every build gives the same bits)
                if (!p.interleaved) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float co = s_cos[row][pa * 8 + j], si = s_sin[row][pa * 8 + j], u = x[j], v = y[j];
                        x[j] = fmaf(u, co, -(v * si));
                        y[j] = fmaf(v, co, u * si);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float co = s_cos[row][pa * 4 + j], si = s_sin[row][pa * 4 + j], u = x[2 * j], v = x[2 * j + 1];
                        x[2 * j] = fmaf(u, co, -(v * si));
                        x[2 * j + 1] = fmaf(v, co, u * si);
                        co = s_cos[row][pb * 4 + j], si = s_sin[row][pb * 4 + j], u = y[2 * j], v = y[2 * j + 1];
                        y[2 * j] = fmaf(u, co, -(v * si));
                        y[2 * j + 1] = fmaf(v, co, u * si);
                    }
                }
            }
            A.set(x);
            B.set(y);
        }
        A.store(out, dst + pa * 8);
        B.store(out, dst + pb * 8);
    }
}

template <int R>
void launch(const QkParams &p, int32_t d, bool f32, int32_t B, hipStream_t st)
{
    auto kernel = d == 128 ? (f32 ? qk_norm_rope_kernel<128, true, R> : qk_norm_rope_kernel<128, false, R>)
                           : (f32 ? qk_norm_rope_kernel<64, true, R> : qk_norm_rope_kernel<64, false, R>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)((p.rows + R - 1) / R), B), dim3(256), 0, st, p);
}

int qk_call(const mcsd_mask_view_t *mask, mcsd_dtype_t dtype, int32_t B, int32_t H_q, int32_t H_kv, int32_t d, int32_t rows,
            int32_t row_begin, const void *q_in, const void *k_in, const void *v_in, int64_t q_batch_stride, int64_t q_row_stride,
            int64_t kv_batch_stride, int64_t kv_row_stride, const mcsd_rope_t *rope, const int32_t *first, const int32_t *n_rows,
            int32_t max_prefix, void *q_out, void *k_out, void *v_out, int64_t out_row_stride, void *hip_stream)
{
    if (!q_in || !k_in || !q_out || !k_out || !rope || !first || (v_in == nullptr) != (v_out == nullptr)) return MCSD_EINVAL;
    if (dtype != MCSD_F32 && dtype != MCSD_BF16) return MCSD_EINVAL;
    if (B < 1 || B > 65535 || H_q < 1 || H_kv < 1 || rows < 0 || max_prefix < 0 || out_row_stride < (int64_t)row_begin + rows) return MCSD_EINVAL;
    if (q_batch_stride < 0 || q_row_stride < 0 || kv_batch_stride < 0 || kv_row_stride < 0) return MCSD_EINVAL;
    if ((q_batch_stride | q_row_stride | kv_batch_stride | kv_row_stride) & 7) return MCSD_EINVAL;
    if (((uintptr_t)q_in | (uintptr_t)k_in | (uintptr_t)v_in | (uintptr_t)q_out | (uintptr_t)k_out | (uintptr_t)v_out) & 15) return MCSD_EINVAL;
    if (!(rope->eps >= 0.f) || rope->eps > 3.4e38f || rope->rotary_dim < 0 || rope->rotary_dim > d || (rope->rotary_dim & 15)) return MCSD_EINVAL;
    if (rope->rotary_dim > 0 && !rope->inv_freq) return MCSD_EINVAL;
    if (d != 64 && d != 128) return MCSD_EUNSUPPORTED;
    if ((int64_t)H_q + 2 * (int64_t)H_kv > 65535 || rows > 4 * MCSD_MAX_GRID_256) return MCSD_EUNSUPPORTED;
    if (rows == 0) return MCSD_OK;

    QkParams p = {};
    p.q = q_in; p.k = k_in; p.v = v_in; p.q_out = q_out; p.k_out = k_out; p.v_out = v_out;
    p.inv_freq = rope->inv_freq; p.wq = rope->q_weight; p.wk = rope->k_weight; p.eps = rope->eps;
    p.rotary = rope->rotary_dim; p.interleaved = rope->interleaved != 0;
    p.first = first; p.n_rows = n_rows;
    p.q_batch = q_batch_stride; p.q_row = q_row_stride; p.kv_batch = kv_batch_stride; p.kv_row = kv_row_stride; p.out_row = out_row_stride;
    p.H_q = H_q; p.H_kv = H_kv; p.heads = H_q + H_kv + (v_in ? H_kv : 0);
    p.rows = rows; p.row0 = row_begin; p.max_prefix = max_prefix;
    if (mask) {
        p.gamma = mask->gamma;
        for (int l = 0; l < mask->gamma; ++l) p.off[l] = mask->level_off_host[l];
    }
    p.by_heads = row_div_of((uint32_t)p.heads);
    // Four rows per workgroup where one leaves lanes idle (64000 rows of 12 heads: 73 us, one by one 101; 8000 of 12: 11.0, 13.3),
    // unless there are so few that the workgroups count (2000 rows of 12: 5.5, one by one 4.9).  With whole rows of lanes one by
    // one is the faster (5000 rows of 48 heads: 27.0 us, four at a time 28.9; 44 of 96: 4.3, 9.4), as long as one launch holds them.
    if ((p.heads * (d / 16) < 256 && (int64_t)rows * B > 2048) || rows > MCSD_MAX_GRID_256) launch<4>(p, d, dtype == MCSD_F32, B, (hipStream_t)hip_stream);
    else launch<1>(p, d, dtype == MCSD_F32, B, (hipStream_t)hip_stream);
    return mcsd_hip_status(hipGetLastError());
}

}  // namespace

extern "C" int mcsd_tree_qk_norm_rope(const mcsd_mask_view_t *mask, mcsd_dtype_t dtype, int32_t B, int32_t H_q, int32_t H_kv, int32_t d,
                                      int32_t row_begin, const void *q_in, const void *k_in, const void *v_in, int64_t q_batch_stride,
                                      int64_t q_row_stride, int64_t kv_batch_stride, int64_t kv_row_stride, const mcsd_rope_t *rope,
                                      const int32_t *prefix_lens_dev, int32_t max_prefix, void *q_out, void *k_out, void *v_out,
                                      int64_t node_stride, void *hip_stream)
{
    if (!mask || mask->gamma < 1 || mask->gamma > MCSD_MAX_LEVELS || !mask->level_off_host || mask->n_nodes < 1) return MCSD_EINVAL;
    if (row_begin < 0 || row_begin >= mask->n_nodes) return MCSD_EINVAL;
    return qk_call(mask, dtype, B, H_q, H_kv, d, mask->n_nodes - row_begin, row_begin, q_in, k_in, v_in, q_batch_stride, q_row_stride,
                   kv_batch_stride, kv_row_stride, rope, prefix_lens_dev, nullptr, max_prefix, q_out, k_out, v_out, node_stride, hip_stream);
}

extern "C" int mcsd_prompt_qk_norm_rope(mcsd_dtype_t dtype, int32_t B, int32_t H_q, int32_t H_kv, int32_t d, int32_t max_rows,
                                        const void *q_in, const void *k_in, const void *v_in, int64_t q_batch_stride,
                                        int64_t q_row_stride, int64_t kv_batch_stride, int64_t kv_row_stride, const mcsd_rope_t *rope,
                                        const int32_t *first_pos_dev, const int32_t *n_rows_dev, void *q_out, void *k_out, void *v_out,
                                        int64_t out_row_stride, void *hip_stream)
{
    if (!n_rows_dev) return MCSD_EINVAL;
    return qk_call(nullptr, dtype, B, H_q, H_kv, d, max_rows, 0, q_in, k_in, v_in, q_batch_stride, q_row_stride, kv_batch_stride,
                   kv_row_stride, rope, first_pos_dev, n_rows_dev, 0, q_out, k_out, v_out, out_row_stride, hip_stream);
}
