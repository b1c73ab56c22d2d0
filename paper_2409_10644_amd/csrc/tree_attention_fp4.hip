// Tree attention over a prefix cache in 4 bits (formulas and format in mcsd.h).
//
// One wavefront per query row: lanes take 64 keys at a time for the scores and the row's channels for the output.
#include <math.h>

#include "fp4_format.h"

namespace {

struct Fp4AttnParams {
    const uint16_t *q, *kt, *vt;
    uint16_t *out;
    mcsd_fp4_cache_t cache;
    const int64_t *seq_base;
    const int32_t *lens;
    const uint64_t *mask_bits;
    int64_t node_stride, head_stride;
    int32_t mask_words, H_q, H_kv, n, row0, max_prefix;
    float c;                         // softmax scale * log2(e)
};

__device__ __forceinline__ float bf16_number(uint16_t v) { return __uint_as_float((unsigned)v << 16); }
__device__ __forceinline__ float fp4_number(unsigned code, unsigned byte)
{
    return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code & 15u, fp4_scale(byte), 0)[0];
}

// grid (rows, H_q, B)
template <int D>
__global__ __launch_bounds__(64) void tree_attn_fp4_row_kernel(const Fp4AttnParams p)
{
    __shared__ float s_q[D], s_p[64];
    const int lane = threadIdx.x, node = p.row0 + blockIdx.x, h = blockIdx.y, b = blockIdx.z, hk = h / (p.H_q / p.H_kv);
    const uint16_t *q = p.q + (((int64_t)b * p.H_q + h) * p.node_stride + node) * D;
    for (int c = lane; c < D; c += 64) s_q[c] = bf16_number(q[c]);
    __syncthreads();
    const int L = min(max(p.lens[b], 0), p.max_prefix);
    const int64_t pre = p.seq_base[b] + hk * p.head_stride, tree = ((int64_t)b * p.H_kv + hk) * p.node_stride * D;
    float m = -INFINITY, l = 0.f, o[D / 64] = {};
    for (int64_t j0 = 0; j0 < (int64_t)L + p.n; j0 += 64) {
        const int64_t j = j0 + lane;
        const int t = (int)(j - L);
        float s = -INFINITY;
        if (j < L) {
            s = 0.f;
            for (int c = 0; c < D; ++c) {
                const int64_t at = pre + j * D + c;
                s = fmaf(s_q[c], fp4_number(((const unsigned char *)p.cache.k_codes)[at / 2] >> (4 * (c & 1)), ((const unsigned char *)p.cache.k_scales)[at / 32]), s);
            }
        } else if (t < p.n && (p.mask_bits[(int64_t)node * p.mask_words + (t >> 6)] >> (t & 63)) & 1) {
            s = 0.f;
            for (int c = 0; c < D; ++c) s = fmaf(s_q[c], bf16_number(p.kt[tree + (int64_t)t * D + c]), s);
        }
        float top = s;
        for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
        const float m_new = fmaxf(m, top);
        const float ref = m_new == -INFINITY ? 0.f : m_new, alpha = exp2f((m - ref) * p.c), e = exp2f((s - ref) * p.c);
        float sum = e;
        for (int x = 32; x; x >>= 1) sum += __shfl_xor(sum, x);
        l = l * alpha + sum;
        m = m_new;
        s_p[lane] = e;
        __syncthreads();
        for (int i = 0; i < D / 64; ++i) o[i] *= alpha;
        for (int k = 0; k < 64 && j0 + k < (int64_t)L + p.n; ++k) {
            const int64_t jk = j0 + k;
            for (int i = 0; i < D / 64; ++i) {
                const int c = i * 64 + lane;
                float v;
                if (jk < L) {
                    const int64_t at = pre + jk * D + c;
                    v = fp4_number(((const unsigned char *)p.cache.v_codes)[at / 2] >> (4 * (c & 1)), ((const unsigned char *)p.cache.v_scales)[at / 32]);
                } else {
                    const int tk = (int)(jk - L);
                    if (!((p.mask_bits[(int64_t)node * p.mask_words + (tk >> 6)] >> (tk & 63)) & 1)) continue;
                    v = bf16_number(p.vt[tree + (int64_t)tk * D + c]);
                }
                o[i] = fmaf(s_p[k], v, o[i]);
            }
        }
        __syncthreads();
    }
    for (int i = 0; i < D / 64; ++i)
        p.out[(((int64_t)b * p.H_q + h) * p.node_stride + node) * D + i * 64 + lane] = __builtin_bit_cast(uint16_t, (__bf16)(o[i] / l));
}

}  // namespace

extern "C" size_t mcsd_tree_attention_fp4kv_workspace(int32_t, int32_t, int32_t, int32_t, int32_t, int32_t, int32_t) { return 0; }

extern "C" int mcsd_tree_attention_fp4kv(const mcsd_mask_view_t *mask, int32_t B, int32_t H_q, int32_t H_kv, int32_t d,
                                         int32_t row_begin, const void *q, const void *k_tree, const void *v_tree,
                                         int64_t node_stride, const mcsd_fp4_cache_t *cache, const int64_t *seq_base_dev,
                                         const int32_t *prefix_lens_dev, int64_t head_stride, int32_t max_prefix,
                                         float softmax_scale, void *out, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (H_kv < 1 || H_q < 1 || H_q % H_kv != 0) return MCSD_EINVAL;
    if (!mask || !mask->bits_dev || !q || !k_tree || !v_tree || !out || !cache || !seq_base_dev || !prefix_lens_dev) return MCSD_EINVAL;
    if (B < 1 || B > 65535 || H_q > 65535 || max_prefix < 0) return MCSD_EINVAL;
    if (max_prefix > 0 && !fp4_cache_ok(cache)) return MCSD_EINVAL;
    const int32_t n = mask->n_nodes;
    if (n < 1 || node_stride < n || head_stride < 0 || row_begin < 0 || row_begin >= n) return MCSD_EINVAL;
    if (!(softmax_scale > 0.f) || !isfinite(softmax_scale)) return MCSD_EINVAL;
    if (d != 64 && d != 128) return MCSD_EUNSUPPORTED;
    if (n > MCSD_ATTN_MAX_NODES) return MCSD_EUNSUPPORTED;
    if (((uintptr_t)q | (uintptr_t)k_tree | (uintptr_t)v_tree | (uintptr_t)out) & 15) return MCSD_EINVAL;
    if (((node_stride * d) & 7) || (head_stride & 127)) return MCSD_EINVAL;
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev != mask->device) return MCSD_EINVAL;

    Fp4AttnParams p;
    p.q = (const uint16_t *)q; p.kt = (const uint16_t *)k_tree; p.vt = (const uint16_t *)v_tree; p.out = (uint16_t *)out;
    p.cache = *cache; p.seq_base = seq_base_dev; p.lens = prefix_lens_dev; p.mask_bits = mask->bits_dev;
    p.node_stride = node_stride; p.head_stride = head_stride; p.mask_words = mask->words_per_row;
    p.H_q = H_q; p.H_kv = H_kv; p.n = n; p.row0 = row_begin; p.max_prefix = max_prefix;
    p.c = softmax_scale * 1.4426950408889634f;
    auto kernel = d == 128 ? tree_attn_fp4_row_kernel<128> : tree_attn_fp4_row_kernel<64>;
    mcsd_launch(MCSD_KERNEL_ATTN_SWEEP, kernel, dim3(n - row_begin, H_q, B), dim3(64), (hipStream_t)hip_stream, p);
    return mcsd_hip_status(hipGetLastError());
}
