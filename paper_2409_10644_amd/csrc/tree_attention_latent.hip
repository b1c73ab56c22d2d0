// Tree attention over a prefix cache of one latent vector per token, shared by all heads (formulas in mcsd.h).
//
// All H * rows query rows of a sequence look at the same keys, so they are cut into chunks of 64 whichever heads they belong to,
// and a workgroup of 4 wavefronts serves one chunk.  A tile is 64 keys; a row of it is key (all d_latent + d_rope channels) and
// value (the first d_latent) at once, so it comes from memory and into LDS once.
//   S^T = X Q^T   each wavefront has 16 of the tile's keys and all 64 query rows, whose operands stay in its registers
//   P             exp2(S - reference), bf16, through LDS: every wavefront needs all of it
//   O^T += X^T P^T  each wavefront has a quarter of the value channels, all 64 rows and all keys
// so of a tile every number is read from LDS twice, once as key and once as value, whatever the number of rows.
#include <math.h>

#include <atomic>

#include "fp4_format.h"

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4_t;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2_t;

struct LatentHeader {                // what to fold: the unit that begins in a piece and goes on in others
    int32_t pieces;                  // 0: none
    int32_t b, chunk;
    int32_t first, second, stride;   // slots of its parts: first, second, second + stride, ...
    int32_t pad[2];
};

struct LatentParams {
    const uint16_t *q, *tree, *cache;
    uint16_t *out;
    const int64_t *seq_base;
    const int32_t *lens;
    const uint64_t *mask_bits;
    int64_t node_stride;
    int32_t mask_words, B, H, n, row0, max_prefix;
    int32_t rows, chunks;            // query rows of a sequence: H * (n - row0), and chunks of 64 of them
    int32_t workgroups, slot_rows;
    RowDiv by_nrows;
    float c;                         // softmax scale * log2(e)
    LatentHeader *header;            // [workgroups]
    float *part_m, *part_l, *part_o; // slots of slot_rows rows: reference maximum (log2 units), sum, output
};

constexpr size_t WS_HEADER = 256, WS_CTR_BYTES = 64 * 1024;      // what other calls keep at the head of a workspace stays as it is
constexpr float SLACK = 6.f;         // log2 of what a score may exceed the running reference by before the output is rescaled
constexpr int ROWS = 64, KEYS = 64;  // query rows of a chunk, keys of a tile
constexpr int MIN_TILES = 2, CROSS = 6;

__device__ __align__(64) const unsigned char no_row[128] = {};

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ const unsigned char *uniform(const unsigned char *a)
{
    const uint64_t v = (uint64_t)a;
    return (const unsigned char *)((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v));
}
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Over the four lanes that hold the same query row (16 apart).
__device__ __forceinline__ float row_max(float v)
{
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float row_sum(float v)
{
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// A tile in LDS: panels of 64 channels, 128 bytes a row, 64 rows each (the last panel has the d_rope channels).  The 16-byte chunk c of row
// r stands at c ^ swz(r): 16 rows read at one chunk, and rows 0-3 and 8-11 read at two neighbouring ones by the transpose loads, hit
// 16 different places of a bank row.  The weights have the same form, a row's 64 keys as its 64 channels.
__device__ __forceinline__ int swz(int r) { return ((r >> 1) & 1) << 2 | ((r >> 2) & 3); }
// A last panel of 32 channels: 64 bytes a row.
__device__ __forceinline__ int swz_half(int r) { return (r >> 2) & 3; }

template <int DL_, int DR_>
struct Cfg {
    static constexpr int DL = DL_, DR = DR_, D = DL + DR, ROWB = 2 * D;
    static constexpr int KS = D / 32;                // matrix steps of S^T
    static constexpr int CB = DL / 64;               // blocks of 16 value channels of a wavefront
    static constexpr int PANELS = DL / 64, PANEL = KEYS * 128;
    static constexpr int TILE = KEYS * ROWB;
    static constexpr int P_AT = 2 * TILE, P_BYTES = ROWS * KEYS * 2;
    static constexpr int MAX_AT = P_AT + P_BYTES, FLAG_AT = MAX_AT + 4 * ROWS * 4, LDS = FLAG_AT + 32;
    static_assert(LDS <= 160 * 1024 && (DR == 64 || DR == 32), "");
};

__device__ __forceinline__ int wave_sum(int v)
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
    return uniform(v);
}
__device__ __forceinline__ int wave_max(int v)
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v = max(v, __shfl_xor(v, o));
    return uniform(v);
}
__device__ __forceinline__ int wave_scan(int v, int lane)        // inclusive
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(v, o);
        if (lane >= o) v += u;
    }
    return v;
}

template <int DL, int DR>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) void tree_attn_latent_kernel(const LatentParams args)
{
    const LatentParams &p = args;
    using C = Cfg<DL, DR>;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[C::LDS];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int G = p.workgroups;
    // Neighbours in the order of the work share an L2: the hardware deals workgroups to the eight dies in turn.
    const int w = (G & 7) == 0 ? ((int)blockIdx.x & 7) * (G >> 3) + ((int)blockIdx.x >> 3) : (int)blockIdx.x;
    const int tree_tiles = (p.n + KEYS - 1) / KEYS;
    auto tiles_of = [&](int b) { return tree_tiles + (int)(((unsigned)min(max(p.lens[b], 0), p.max_prefix) + KEYS - 1) / KEYS); };

    // ---- this workgroup's piece of the work
    const int t_first = lane < p.B ? tiles_of(lane) : 0;
    auto tiles_at = [&](int b0) { return b0 == 0 ? t_first : b0 + lane < p.B ? tiles_of(b0 + lane) : 0; };      // of sequence b0 + lane
    int total = 0, most = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        const int t = tiles_at(b0);
        total += wave_sum(t);
        most = max(most, wave_max(t));
    }
    const int pairs = p.B * p.chunks, least = max(MIN_TILES, (int)(0.5f * __builtin_amdgcn_sqrtf((float)most)));
    int per = max((int)(((int64_t)total * p.chunks + G - 1) / G), least), aligned = 0;
    if (pairs <= G) {
        if (per >= most) {
            aligned = per;
        } else {
            auto fits = [&](int size) {
                int sum = 0;
                for (int b0 = 0; b0 < p.B; b0 += 64) sum += wave_sum((tiles_at(b0) + size - 1) / size);
                return sum * p.chunks <= G;
            };
            int lo = per, hi = per + CROSS;
            if (fits(hi)) {
                while (lo < hi) {
                    const int mid = (lo + hi) >> 1;
                    if (fits(mid)) hi = mid;
                    else lo = mid + 1;
                }
                aligned = hi;
            }
        }
    }
    // b, chunk: where the piece begins; tile: its first tile there; left: its tiles in all
    int b = -1, chunk = 0, tile = 0, left = 0, n_pieces = 1, number = 0, each = 0;
    if (aligned) {
        int before = 0;
        for (int b0 = 0; b0 < p.B && b < 0; b0 += 64) {
            const int t = tiles_at(b0), e = (t + aligned - 1) / aligned, s = wave_scan(e * p.chunks, lane);
            const int last = before + s;
            const uint64_t beyond = __builtin_amdgcn_ballot_w64(w < last);
            if (beyond) {
                const int l = __builtin_ctzll(beyond);
                b = b0 + l;
                n_pieces = __builtin_amdgcn_readlane(e, l);
                const int tiles = __builtin_amdgcn_readlane(t, l), k = w - (__builtin_amdgcn_readlane(last, l) - n_pieces * p.chunks);
                number = k / p.chunks;                               // (the same keys of all chunks next to each other)
                chunk = k - number * p.chunks;
                each = (tiles + n_pieces - 1) / n_pieces;
                tile = number * each;
                left = min(each, tiles - tile);
            }
            before = __builtin_amdgcn_readlane(last, 63);
        }
    } else {
        const int64_t from = (int64_t)w * per, all = (int64_t)total * p.chunks;
        int64_t before = 0;
        left = (int)min((int64_t)per, all - from);
        for (int b0 = 0; b0 < p.B && b < 0 && left > 0; b0 += 64) {
            const int t = tiles_at(b0), s = wave_scan(t, lane);
            const uint64_t beyond = __builtin_amdgcn_ballot_w64(from < before + (int64_t)s * p.chunks);
            if (beyond) {
                const int l = __builtin_ctzll(beyond);
                b = b0 + l;
                const int tiles = __builtin_amdgcn_readlane(t, l);
                const int k = (int)(from - (before + (int64_t)(__builtin_amdgcn_readlane(s, l) - tiles) * p.chunks));
                chunk = k / tiles;
                tile = k - chunk * tiles;
            }
            before += (int64_t)__builtin_amdgcn_readlane(s, 63) * p.chunks;
        }
    }
    if (b < 0 || left <= 0) {
        if (p.header && tid == 0) p.header[w].pieces = 0;
        return;
    }

    // ---- places of this lane
    const int krow = 16 * wave + col;                                      // its key of the tile (operand rows), for all chunks of channels
    const int k_at = krow * 128 + ((grp ^ swz(krow)) << 4);                // panel's chunk grp; the other half of a panel: ^ 64
    const int k_half = C::PANELS * C::PANEL + krow * 64 + ((grp ^ swz_half(krow)) << 4);
    const int jr = col >> 2;                                               // of the 16 lanes of a transpose load: row, 4 channels
    const int v_row = 8 * grp + jr;                                        // + 4 for the second load, + 32 for the second step
    const int v_at = v_row * 128 + ((((col & 3) >> 1) ^ swz(v_row)) << 4) + (col & 1) * 8 + wave * (DL / 4) * 128;
    const int pw_at = C::P_AT + col * 128 + (((2 * wave + (grp >> 1)) ^ swz(col)) << 4) + (grp & 1) * 8;     // + 16 rows * 128 (weights written)
    const int pr_at = C::P_AT + col * 128 + ((grp ^ swz(col)) << 4);       // (weights read; second step: ^ 64)
    // Tile loads: 8 rows of a panel per instruction, a wavefront brings rows 16 wave .. + 15.
    const int lrow = lane >> 3, lchunk = lane & 7;
    const uint32_t load_even = (uint32_t)(lrow * C::ROWB + ((lchunk ^ swz(lrow)) << 4));
    const uint32_t load_odd = (uint32_t)(lrow * C::ROWB + ((lchunk ^ swz(lrow + 8)) << 4));
    const uint32_t load_half = (uint32_t)((lane >> 2) * C::ROWB + (((lane & 3) ^ swz_half(lane >> 2)) << 4));

    // (begins, goes on): whether the piece's part of the unit has its first and its last tile
    for (bool begun = false;; begun = true) {
        b = uniform(b);
        chunk = uniform(chunk);
        tile = uniform(tile);
        left = uniform(left);
        const int len = uniform(min(max(p.lens[b], 0), p.max_prefix)), tiles = tree_tiles + (int)(((unsigned)len + KEYS - 1) / KEYS);
        const int from = tile, count = min(left, tiles - tile);
        const unsigned char *past = uniform((const unsigned char *)(p.cache + p.seq_base[b]));
        const unsigned char *nodes = uniform((const unsigned char *)(p.tree + (int64_t)b * p.node_stride * C::D));

        auto request = [&](int t, int stage) __attribute__((always_inline)) {
            const unsigned char *src = t < tree_tiles ? nodes + (int64_t)t * C::TILE : past + (int64_t)(t - tree_tiles) * C::TILE;
            const int here = t < tree_tiles ? p.n - t * KEYS : len - (t - tree_tiles) * KEYS;      // keys of this tile (or more)
            unsigned char *dst = lds + stage * C::TILE;
            if (here >= KEYS) {
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int x = 0; x < C::PANELS + (DR == 64); ++x)
                        load_to_lds16<false>(src + (16 * wave + 8 * k) * C::ROWB + x * 128, k ? load_odd : load_even,
                                             dst + x * C::PANEL + (16 * wave + 8 * k) * 128);
                if constexpr (DR == 32)
                    load_to_lds16<false>(src + 16 * wave * C::ROWB + C::PANELS * 128, load_half, dst + C::PANELS * C::PANEL + 16 * wave * 64);
            } else {                                                       // rows behind the last: zeros
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int x = 0; x < C::PANELS + (DR == 64); ++x) {
                        const int row = 16 * wave + 8 * k;
                        load_to_lds16_at(row + lrow < here ? src + row * C::ROWB + x * 128 + (k ? load_odd : load_even) : no_row + (lane & 7) * 16,
                                         dst + x * C::PANEL + row * 128);
                    }
                if constexpr (DR == 32)
                    load_to_lds16_at(16 * wave + (lane >> 2) < here ? src + 16 * wave * C::ROWB + C::PANELS * 128 + load_half : no_row + (lane & 3) * 16,
                                     dst + C::PANELS * C::PANEL + 16 * wave * 64);
            }
        };
        request(from, 0);

        // Query operands: rows col + 16 rg of the chunk (behind the last: that one), channels 32 ks + 8 grp .. + 7.  And which tree nodes
        // the rows see among this lane's 4 keys: 4 bits per row and tree tile.
        bf16x8_t q[4][C::KS];
        unsigned seen[2] = {0, 0};
#pragma unroll
        for (int rg = 0; rg < 4; ++rg) {
            const int r = min(chunk * ROWS + 16 * rg + col, p.rows - 1), h = row_div(r, p.by_nrows), i = p.row0 + r - h * (p.n - p.row0);
            const uint16_t *src = p.q + (((int64_t)b * p.H + h) * p.node_stride + i) * C::D + 8 * grp;
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks) q[rg][ks] = *(const bf16x8_t *)(src + 32 * ks);
            const uint64_t *bits = p.mask_bits + (int64_t)i * p.mask_words;
            seen[0] |= (unsigned)((bits[0] >> (16 * wave + 4 * grp)) & 15) << (4 * rg);
            if (tree_tiles > 1) seen[1] |= (unsigned)((bits[1] >> (16 * wave + 4 * grp)) & 15) << (4 * rg);
        }
        f32x4_t o[4][C::CB];
        float ref[4], l[4];
#pragma unroll
        for (int rg = 0; rg < 4; ++rg) {
            ref[rg] = -INFINITY;
            l[rg] = 0.f;
#pragma unroll
            for (int cb = 0; cb < C::CB; ++cb) o[rg][cb] = (f32x4_t){0, 0, 0, 0};
        }

        for (int t = 0; t < count; ++t) {
            const int at = from + t, stage = t & 1, st = stage * C::TILE;
            MCSD_WAIT_VMCNT(0);
            meet();                                                        // the tile is here, and the one before is done with
            if (t + 1 < count) request(at + 1, stage ^ 1);

            f32x4_t s[4];
#pragma unroll
            for (int rg = 0; rg < 4; ++rg) s[rg] = (f32x4_t){0, 0, 0, 0};
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks) {
                const int a = DR == 32 && ks == C::KS - 1 ? k_half : (k_at ^ ((ks & 1) << 6)) + (ks >> 1) * C::PANEL;
                const bf16x8_t k = *(const bf16x8_t *)(lds + st + a);
#pragma unroll
                for (int rg = 0; rg < 4; ++rg) s[rg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[rg][ks], s[rg], 0, 0, 0);
            }
            const bool tree = at < tree_tiles;
            const int here = tree ? KEYS : len - (at - tree_tiles) * KEYS;
#pragma unroll
            for (int rg = 0; rg < 4; ++rg) s[rg] *= p.c;
            if (tree || here < KEYS) {
                unsigned bits;
                if (tree) {
                    bits = at ? seen[1] : seen[0];
                } else {
                    const int mine = min(max(here - 16 * wave - 4 * grp, 0), 4);
                    bits = ((1u << mine) - 1) * 0x1111u;
                }
#pragma unroll
                for (int rg = 0; rg < 4; ++rg)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[rg][i] = (bits >> (4 * rg + i)) & 1 ? s[rg][i] : -INFINITY;
            }
            float mx[4];
            bool grow = false;
#pragma unroll
            for (int rg = 0; rg < 4; ++rg) {
                mx[rg] = fmaxf(fmaxf(s[rg][0], s[rg][1]), fmaxf(s[rg][2], s[rg][3]));
                grow |= mx[rg] > ref[rg] + SLACK;
            }
            // weights, and whether a row of this wavefront outgrows its reference
            float part[4];
            auto weigh = [&]() __attribute__((always_inline)) {
#pragma unroll
                for (int rg = 0; rg < 4; ++rg) {
                    const float zero = ref[rg] == -INFINITY ? 0.f : ref[rg];
                    float e[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) e[i] = fast_exp2(s[rg][i] - zero);
                    part[rg] = (e[0] + e[1]) + (e[2] + e[3]);
                    const u32x2_t pk = {__builtin_bit_cast(unsigned, (bf16x2_t){(__bf16)e[0], (__bf16)e[1]}),
                                        __builtin_bit_cast(unsigned, (bf16x2_t){(__bf16)e[2], (__bf16)e[3]})};
                    *(u32x2_t *)(lds + pw_at + rg * 16 * 128) = pk;
                }
            };
            weigh();
            const bool wave_grows = __builtin_amdgcn_ballot_w64(grow) != 0;
            if (lane == 0) *(int *)(lds + C::FLAG_AT + 4 * wave) = wave_grows;
            meet();
            const u32x4_t flags = *(const u32x4_t *)(lds + C::FLAG_AT);
            if (__builtin_expect(uniform((int)(flags[0] | flags[1] | flags[2] | flags[3])) != 0, 0)) {
                // all wavefronts: the maxima of all keys, new references, the weights again
#pragma unroll
                for (int rg = 0; rg < 4; ++rg) {
                    const float m = row_max(mx[rg]);
                    if (grp == 0) *(float *)(lds + C::MAX_AT + (wave * ROWS + 16 * rg + col) * 4) = m;
                }
                meet();
#pragma unroll
                for (int rg = 0; rg < 4; ++rg) {
                    float m = -INFINITY;
#pragma unroll
                    for (int k = 0; k < 4; ++k) m = fmaxf(m, *(const float *)(lds + C::MAX_AT + (k * ROWS + 16 * rg + col) * 4));
                    const float next = m > ref[rg] + SLACK ? m : ref[rg];
                    const float alpha = next == ref[rg] ? 1.f : fast_exp2(ref[rg] - next);
                    ref[rg] = next;
                    l[rg] *= alpha;
#pragma unroll
                    for (int cb = 0; cb < C::CB; ++cb) o[rg][cb] *= alpha;
                }
                weigh();
                meet();
            }
#pragma unroll
            for (int rg = 0; rg < 4; ++rg) l[rg] += part[rg];

#pragma unroll
            for (int k2 = 0; k2 < 2; ++k2) {
                bf16x8_t pf[4];
#pragma unroll
                for (int rg = 0; rg < 4; ++rg) pf[rg] = *(const bf16x8_t *)(lds + (pr_at ^ (k2 << 6)) + rg * 16 * 128);
#pragma unroll
                for (int cb = 0; cb < C::CB; ++cb) {
                    const int a = st + (v_at ^ ((cb & 3) << 5)) + (cb >> 2) * C::PANEL + k2 * 32 * 128;
                    const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4_t __attribute__((address_space(3))) *)(lds + a));
                    const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4_t __attribute__((address_space(3))) *)(lds + ((a + 512) ^ 16)));
                    const bf16x8_t v = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                    for (int rg = 0; rg < 4; ++rg) o[rg][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pf[rg], o[rg][cb], 0, 0, 0);
                }
            }
        }

        // ---- sums of all wavefronts; the rows' output, or this part of it
        meet();
#pragma unroll
        for (int rg = 0; rg < 4; ++rg) {
            const float sum = row_sum(l[rg]);
            if (grp == 0) *(float *)(lds + C::MAX_AT + (wave * ROWS + 16 * rg + col) * 4) = sum;
        }
        meet();
        const bool whole = from == 0 && count == tiles, first = from == 0, last = from + count == tiles;
        const int slot = aligned ? 2 * w : 2 * w + (begun ? 1 : 0);
#pragma unroll
        for (int rg = 0; rg < 4; ++rg) {
            const int row = 16 * rg + col, r = chunk * ROWS + row;
            float sum = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) sum += *(const float *)(lds + C::MAX_AT + (k * ROWS + row) * 4);
            if (r < p.rows) {
                if (whole) {
                    const int h = row_div(r, p.by_nrows), i = p.row0 + r - h * (p.n - p.row0);
                    uint16_t *dst = p.out + (((int64_t)b * p.H + h) * p.node_stride + i) * DL + wave * (DL / 4) + 4 * grp;
                    const float inv = 1.f / sum;
#pragma unroll
                    for (int cb = 0; cb < C::CB; ++cb) {
                        const f32x4_t x = o[rg][cb] * inv;
                        const u32x2_t pk = {__builtin_bit_cast(unsigned, (bf16x2_t){(__bf16)x[0], (__bf16)x[1]}),
                                            __builtin_bit_cast(unsigned, (bf16x2_t){(__bf16)x[2], (__bf16)x[3]})};
                        *(u32x2_t *)(dst + 16 * cb) = pk;
                    }
                } else {
                    const int64_t at = (int64_t)slot * p.slot_rows + row;
                    if (wave == 0 && grp == 0) {
                        p.part_m[at] = ref[rg];
                        p.part_l[at] = sum;
                    }
                    float *dst = p.part_o + at * DL + wave * (DL / 4) + 4 * grp;
#pragma unroll
                    for (int cb = 0; cb < C::CB; ++cb) *(f32x4_t *)(dst + 16 * cb) = o[rg][cb];
                }
            }
        }
        left -= count;
        const bool more = !aligned && left > 0;
        if (!more) {
            if (p.header && tid == 0) {
                LatentHeader h = {};
                if (first && !last) {                                      // it begins here: who goes on with it
                    h.b = b;
                    h.chunk = chunk;
                    h.first = slot;
                    if (aligned) {
                        h.pieces = n_pieces;
                        h.stride = 2 * p.chunks;
                        h.second = slot + h.stride;
                    } else {
                        h.pieces = 1 + (tiles - count + per - 1) / per;
                        h.stride = 2;
                        h.second = 2 * (w + 1);
                    }
                }
                p.header[w] = h;
            }
            return;
        }
        meet();                                                            // the sums are read before the next unit's are written
        tile = 0;
        if (++chunk == p.chunks) {
            chunk = 0;
            if (++b == p.B) return;
        }
    }
}

// grid (pieces, slot_rows / 8): eight rows of the unit that begins in a piece, its parts added up in order.
template <int DL>
__global__ __launch_bounds__(256) void tree_attn_latent_fold_kernel(const LatentParams p)
{
    const LatentHeader h = p.header[blockIdx.x];
    constexpr int PER = DL / 128;                    // pieces of four channels per thread
    const int row = blockIdx.y * 8 + (threadIdx.x >> 5), r = h.chunk * ROWS + row, c = (threadIdx.x & 31) * 4;
    if (h.pieces == 0 || row >= p.slot_rows || r >= p.rows) return;
    float m = -INFINITY, sum = 0.f;
    f32x4_t acc[PER];
#pragma unroll
    for (int x = 0; x < PER; ++x) acc[x] = (f32x4_t){0, 0, 0, 0};
    for (int k = 0; k < h.pieces; ++k) {
        const int64_t at = (int64_t)(k == 0 ? h.first : h.second + (k - 1) * h.stride) * p.slot_rows + row;
        const float pm = p.part_m[at], pl = p.part_l[at], next = fmaxf(m, pm);
        const float a = m == next ? 1.f : fast_exp2(m - next), e = pm == next ? 1.f : fast_exp2(pm - next);
        m = next;
        sum = sum * a + pl * e;
#pragma unroll
        for (int x = 0; x < PER; ++x) acc[x] = acc[x] * a + *(const f32x4_t *)(p.part_o + at * DL + c + 128 * x) * e;
    }
    const int head = row_div(r, p.by_nrows), i = p.row0 + r - head * (p.n - p.row0);
    uint16_t *dst = p.out + (((int64_t)h.b * p.H + head) * p.node_stride + i) * DL + c;
    const float inv = 1.f / sum;
#pragma unroll
    for (int x = 0; x < PER; ++x) {
        const f32x4_t y = acc[x] * inv;
        const u32x2_t pk = {__builtin_bit_cast(unsigned, (bf16x2_t){(__bf16)y[0], (__bf16)y[1]}),
                            __builtin_bit_cast(unsigned, (bf16x2_t){(__bf16)y[2], (__bf16)y[3]})};
        *(u32x2_t *)(dst + 128 * x) = pk;
    }
}

// ---------------------------------------------------------------------------------------------------- host
struct LatentPlan {
    int chunks, workgroups, slot_rows;
    size_t bytes;                    // workspace; 0: no unit is ever cut
};

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

int compute_units()
{
    static std::atomic<int> cus_of_device[64];
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) {
        (void)hipGetLastError();
        return 256;                  // no device to ask: the whole chip
    }
    int v = cus_of_device[dev].load(std::memory_order_relaxed);
    if (v == 0) {
        if (hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || v < 1) v = 256;
        cus_of_device[dev].store(v, std::memory_order_relaxed);
    }
    return v;
}

// False where the work has more tiles than the kernel's numbers hold.
bool make_plan(int B, int H, int dl, int n_rows, int n, int max_prefix, LatentPlan &pl)
{
    const int64_t rows = (int64_t)H * n_rows, chunks = (rows + ROWS - 1) / ROWS, pairs = chunks * B;
    const int64_t tiles = (n + KEYS - 1) / KEYS + ((int64_t)max_prefix + KEYS - 1) / KEYS;
    if (rows > 0x3fffffff || pairs > 0x3fffffff || pairs * tiles > 0x3fffffff) return false;
    const int64_t pieces = pairs * ((tiles + MIN_TILES - 1) / MIN_TILES);
    const int cus = compute_units();
    pl.chunks = (int)chunks;
    pl.workgroups = (int)(pieces < cus ? pieces : cus);
    pl.slot_rows = rows < ROWS ? (int)rows : ROWS;
    pl.bytes = 0;
    if (pieces > pairs || pairs > cus) {
        const size_t slots = (size_t)2 * pl.workgroups, slot_rows = slots * pl.slot_rows;
        pl.bytes = WS_HEADER + WS_CTR_BYTES + align256(pl.workgroups * sizeof(LatentHeader)) + 2 * align256(slot_rows * 4) + slot_rows * dl * 4;
    }
    return true;
}

bool sizes_ok(int32_t dl, int32_t dr) { return (dl == 512 && dr == 64) || (dl == 256 && dr == 32); }

}  // namespace

extern "C" size_t mcsd_tree_attention_latent_workspace(int32_t B, int32_t H, int32_t d_latent, int32_t d_rope, int32_t n_nodes,
                                                       int32_t row_begin, int32_t max_prefix)
{
    if (B < 1 || H < 1 || !sizes_ok(d_latent, d_rope) || n_nodes < 1 || n_nodes > MCSD_ATTN_MAX_NODES || max_prefix < 0 || row_begin < 0 ||
        row_begin >= n_nodes)
        return 0;
    size_t most = 0;                 // of any number of rows up to this one
    for (int rows = 1; rows <= n_nodes - row_begin; ++rows) {
        LatentPlan pl;
        if (make_plan(B, H, d_latent, rows, n_nodes, max_prefix, pl) && pl.bytes > most) most = pl.bytes;
    }
    return most;
}

extern "C" int mcsd_tree_attention_latent(const mcsd_mask_view_t *mask, int32_t B, int32_t H, int32_t d_latent, int32_t d_rope,
                                          int32_t row_begin, const void *q, const void *latent_tree, int64_t node_stride,
                                          const void *latent_prefix, const int64_t *seq_base_dev, const int32_t *prefix_lens_dev,
                                          int32_t max_prefix, float softmax_scale, void *out, void *workspace, size_t workspace_bytes,
                                          void *hip_stream)
{
    if (!mask || !mask->bits_dev || !q || !latent_tree || !out || !seq_base_dev || !prefix_lens_dev) return MCSD_EINVAL;
    if (B < 1 || B > 65535 || H < 1 || H > 65535 || max_prefix < 0 || (max_prefix > 0 && !latent_prefix)) return MCSD_EINVAL;
    const int32_t n = mask->n_nodes;
    if (n < 1 || node_stride < n || row_begin < 0 || row_begin >= n) return MCSD_EINVAL;
    if (!(softmax_scale > 0.f) || !isfinite(softmax_scale)) return MCSD_EINVAL;
    if (!sizes_ok(d_latent, d_rope) || n > MCSD_ATTN_MAX_NODES) return MCSD_EUNSUPPORTED;
    if (((uintptr_t)q | (uintptr_t)latent_tree | (uintptr_t)latent_prefix | (uintptr_t)out) & 15) return MCSD_EINVAL;
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev != mask->device) {
        (void)hipGetLastError();
        return MCSD_EINVAL;
    }
    LatentPlan pl;
    if (!make_plan(B, H, d_latent, n - row_begin, n, max_prefix, pl)) return MCSD_EUNSUPPORTED;
    if (pl.bytes > 0 && (!workspace || workspace_bytes < pl.bytes || ((uintptr_t)workspace & 255))) return MCSD_EWORKSPACE;

    LatentParams p = {};
    p.q = (const uint16_t *)q; p.tree = (const uint16_t *)latent_tree; p.cache = (const uint16_t *)latent_prefix; p.out = (uint16_t *)out;
    p.seq_base = seq_base_dev; p.lens = prefix_lens_dev; p.mask_bits = mask->bits_dev;
    p.node_stride = node_stride; p.mask_words = mask->words_per_row;
    p.B = B; p.H = H; p.n = n; p.row0 = row_begin; p.max_prefix = max_prefix;
    p.rows = H * (n - row_begin); p.chunks = pl.chunks;
    p.workgroups = pl.workgroups; p.slot_rows = pl.slot_rows;
    p.by_nrows = row_div_of((uint32_t)(n - row_begin));
    p.c = softmax_scale * 1.4426950408889634f;
    if (pl.bytes > 0) {
        char *ws = (char *)workspace + WS_HEADER + WS_CTR_BYTES;
        const size_t slot_rows = (size_t)2 * pl.workgroups * pl.slot_rows;
        p.header = (LatentHeader *)ws;
        ws += align256(pl.workgroups * sizeof(LatentHeader));
        p.part_m = (float *)ws;
        ws += align256(slot_rows * 4);
        p.part_l = (float *)ws;
        ws += align256(slot_rows * 4);
        p.part_o = (float *)ws;
    }
    hipStream_t st = (hipStream_t)hip_stream;
    auto kernel = d_latent == 512 ? tree_attn_latent_kernel<512, 64> : tree_attn_latent_kernel<256, 32>;
    mcsd_launch(MCSD_KERNEL_ATTN_SWEEP, kernel, dim3(pl.workgroups), dim3(256), st, p);
    if (hipGetLastError() != hipSuccess) return MCSD_EHIP;
    if (pl.bytes > 0) {
        auto fold = d_latent == 512 ? tree_attn_latent_fold_kernel<512> : tree_attn_latent_fold_kernel<256>;
        mcsd_launch(MCSD_KERNEL_ATTN_MERGE, fold, dim3(pl.workgroups, (pl.slot_rows + 7) / 8), dim3(256), st, p);
        return mcsd_hip_status(hipGetLastError());
    }
    return MCSD_OK;
}
