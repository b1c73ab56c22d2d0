// Tree attention over a prefix cache of one latent vector per token, shared by all heads (formulas in mcsd.h).
//
// All H * rows query rows of a sequence look at the same keys, so they are cut into chunks of 64 whichever heads they belong to, and a
// workgroup serves one chunk.  A tile is 32 keys; a row of it is key (all d_latent + d_rope channels) and value (the first d_latent) at
// once, so it comes from memory and into LDS once, into a ring of four tiles.
//   S^T = X Q^T   four wavefronts, each with 16 of the tile's keys and 32 query rows, whose operands stay in its registers; then
//   P             2^(S - reference) in bf16, through LDS
//   O^T += X^T P^T  four others, one tile behind, each with a quarter of the value channels, all 64 rows and all keys
// A SIMD has one wavefront of each kind: the soft-max of the one runs in the shadow of the other's products, and they meet once a tile.
// (The same work by four wavefronts that take turns at both, alone on their SIMDs: every instruction between the products then
// stands alone, 4500 cycles per 64 keys, of which the products are 2176.)
#include <math.h>

#include "fp4_format.h"
#include "wave_ops.h"

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4_t;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2_t;

struct LatentHeader {                // what to fold: a unit (a chunk of a sequence) whose keys several workgroups shared
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
    LatentHeader *header;            // [workgroups, or units where these are fewer]
    float *part_m, *part_l, *part_o; // slots of slot_rows rows: reference maximum (log2 units), sum, output
};

constexpr size_t WS_HEADER = 256, WS_CTR_BYTES = 64 * 1024;      // what other calls keep at the head of a workspace stays as it is
constexpr float SLACK = 16.f;        // log2 of what a score may exceed the running reference by before the output is rescaled
constexpr int ROWS = 64, KEYS = 32;  // query rows of a chunk, keys of a tile
constexpr int MIN_TILES = 4, UNCUT = 16;
constexpr int CROSS = 12;            // tiles that a piece within one sequence may have beyond an equal share (both sides at its use)
constexpr int THREADS = 512;
constexpr int GROWN = 1, WRONG = 2;  // of a tile: scores beyond a reference; scores of tree nodes, seen or not, that are not finite

__device__ __align__(64) const unsigned char no_row[128] = {};

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ const unsigned char *uniform(const unsigned char *a)
{
    const uint64_t v = (uint64_t)a;
    return (const unsigned char *)((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v));
}
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ float max4(const f32x4_t &v)
{
    float m;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(v[0]), "v"(v[1]), "v"(v[2]));
    asm("v_max_f32 %0, %1, %2" : "=v"(m) : "v"(m), "v"(v[3]));
    return m;
}

// A value that the compiler knows nothing about: what is made of it is made here, not kept in registers from before the loops.
__device__ __forceinline__ int anew(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}

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

// Matrix products with the accumulator in its place (the builtin's result may stand elsewhere, and across a loop's branches it then
// does: twice the registers).  The wait states that vector instructions need behind the results are the caller's, settle(), and so are the
// two between a vector instruction and a product that reads what it wrote.
__device__ __forceinline__ void mfma(f32x4_t &c, const bf16x8_t &a, const bf16x8_t &b) { asm("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(c) : "v"(a), "v"(b)); }
__device__ __forceinline__ void settle() { asm volatile("s_nop 15\n\ts_nop 3" ::: "memory"); }
__device__ __forceinline__ int lds_at(const void *p) { return (int)(uintptr_t)(__attribute__((address_space(3))) const void *)p; }
// load_to_lds16 where `ask` (uniform) is not 0, with the branch inside: in two ways around it the compiler would hold the output twice.
template <bool NT>
__device__ __forceinline__ void load_if(int ask, const void *gbase, uint32_t voff, void *lds_base)
{
    if constexpr (NT)
        asm volatile("s_cmp_eq_u32 %3, 0\n\ts_cbranch_scc1 .Lnone%=\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt\n.Lnone%=:"
                     : : "s"(lds_at(lds_base)), "v"(voff), "s"(gbase), "s"(ask) : "memory", "scc");
    else
        asm volatile("s_cmp_eq_u32 %3, 0\n\ts_cbranch_scc1 .Lnone%=\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n.Lnone%=:"
                     : : "s"(lds_at(lds_base)), "v"(voff), "s"(gbase), "s"(ask) : "memory", "scc");
}
// Where `on` (uniform) is not 0, all accumulators of a lane times the numbers at LDS bytes a, a + 64, a + 128, a + 192 (one per group of 16
// rows), each through 16 bytes of LDS of the lane's own.  One block with its branch inside, so that for the compiler every accumulator
// stays in its registers: written as ordinary multiplications behind a branch, it kept the output twice, and copied it from one place
// to the other every turn.
// (LDS serves a wavefront in order: what it wrote it reads without a wait.)
#define MCSD_TIMES(C) "ds_write_b128 %[own], " C "\n\tds_read_b32 %[t0], %[own]\n\tds_read_b32 %[t1], %[own] offset:4\n\t" \
                      "ds_read_b32 %[t2], %[own] offset:8\n\tds_read_b32 %[t3], %[own] offset:12\n\ts_waitcnt lgkmcnt(0)\n\tv_mul_f32 %[t0], %[t0], %[f]\n\t" \
                      "v_mul_f32 %[t1], %[t1], %[f]\n\tv_mul_f32 %[t2], %[t2], %[f]\n\tv_mul_f32 %[t3], %[t3], %[f]\n\tds_write_b32 %[own], %[t0]\n\t" \
                      "ds_write_b32 %[own], %[t1] offset:4\n\tds_write_b32 %[own], %[t2] offset:8\n\tds_write_b32 %[own], %[t3] offset:12\n\t" \
                      "ds_read_b128 " C ", %[own]\n\t"
#define MCSD_FACTOR(AT) "ds_read_b32 %[f], %[a] offset:" AT "\n\ts_waitcnt lgkmcnt(0)\n\t"
#define MCSD_SKIP "s_cmp_eq_u32 %[on], 0\n\ts_cbranch_scc1 .Lkept%=\n\ts_nop 15\n\ts_nop 3\n\t"
#define MCSD_TIMES4(A, B, C, D) MCSD_TIMES(A) MCSD_TIMES(B) MCSD_TIMES(C) MCSD_TIMES(D)
__device__ __forceinline__ void multiply(int on, f32x4_t (&o)[4][4], int a, int own)
{
    float f, t0, t1, t2, t3;
    asm volatile(MCSD_SKIP MCSD_FACTOR("0") MCSD_TIMES4("%0", "%1", "%2", "%3") MCSD_FACTOR("64") MCSD_TIMES4("%4", "%5", "%6", "%7")
                 MCSD_FACTOR("128") MCSD_TIMES4("%8", "%9", "%10", "%11") MCSD_FACTOR("192") MCSD_TIMES4("%12", "%13", "%14", "%15") "s_waitcnt lgkmcnt(0)\n.Lkept%=:"
                 : "+v"(o[0][0]), "+v"(o[0][1]), "+v"(o[0][2]), "+v"(o[0][3]), "+v"(o[1][0]), "+v"(o[1][1]), "+v"(o[1][2]), "+v"(o[1][3]),
                   "+v"(o[2][0]), "+v"(o[2][1]), "+v"(o[2][2]), "+v"(o[2][3]), "+v"(o[3][0]), "+v"(o[3][1]), "+v"(o[3][2]), "+v"(o[3][3]),
                   [f] "=&v"(f), [t0] "=&v"(t0), [t1] "=&v"(t1), [t2] "=&v"(t2), [t3] "=&v"(t3)
                 : [a] "v"(a), [own] "v"(own), [on] "s"(on)
                 : "memory", "scc");
}
__device__ __forceinline__ void multiply(int on, f32x4_t (&o)[1][4], int a, int own)
{
    float f, t0, t1, t2, t3;
    asm volatile(MCSD_SKIP MCSD_FACTOR("0") MCSD_TIMES4("%0", "%1", "%2", "%3") "s_waitcnt lgkmcnt(0)\n.Lkept%=:"
                 : "+v"(o[0][0]), "+v"(o[0][1]), "+v"(o[0][2]), "+v"(o[0][3]), [f] "=&v"(f), [t0] "=&v"(t0), [t1] "=&v"(t1), [t2] "=&v"(t2), [t3] "=&v"(t3)
                 : [a] "v"(a), [own] "v"(own), [on] "s"(on)
                 : "memory", "scc");
}
__device__ __forceinline__ void multiply(int on, f32x4_t (&o)[1][8], int a, int own)
{
    float f, t0, t1, t2, t3;
    asm volatile(MCSD_SKIP MCSD_FACTOR("0") MCSD_TIMES4("%0", "%1", "%2", "%3") MCSD_TIMES4("%4", "%5", "%6", "%7") "s_waitcnt lgkmcnt(0)\n.Lkept%=:"
                 : "+v"(o[0][0]), "+v"(o[0][1]), "+v"(o[0][2]), "+v"(o[0][3]), "+v"(o[0][4]), "+v"(o[0][5]), "+v"(o[0][6]), "+v"(o[0][7]),
                   [f] "=&v"(f), [t0] "=&v"(t0), [t1] "=&v"(t1), [t2] "=&v"(t2), [t3] "=&v"(t3)
                 : [a] "v"(a), [own] "v"(own), [on] "s"(on)
                 : "memory", "scc");
}
__device__ __forceinline__ void multiply(int on, f32x4_t (&o)[4][8], int a, int own)
{
    float f, t0, t1, t2, t3;
    asm volatile(MCSD_SKIP MCSD_FACTOR("0") MCSD_TIMES4("%0", "%1", "%2", "%3") MCSD_TIMES4("%4", "%5", "%6", "%7")
                 MCSD_FACTOR("64") MCSD_TIMES4("%8", "%9", "%10", "%11") MCSD_TIMES4("%12", "%13", "%14", "%15")
                 MCSD_FACTOR("128") MCSD_TIMES4("%16", "%17", "%18", "%19") MCSD_TIMES4("%20", "%21", "%22", "%23")
                 MCSD_FACTOR("192") MCSD_TIMES4("%24", "%25", "%26", "%27") MCSD_TIMES4("%28", "%29", "%30", "%31") "s_waitcnt lgkmcnt(0)\n.Lkept%=:"
                 : "+v"(o[0][0]), "+v"(o[0][1]), "+v"(o[0][2]), "+v"(o[0][3]), "+v"(o[0][4]), "+v"(o[0][5]), "+v"(o[0][6]), "+v"(o[0][7]),
                   "+v"(o[1][0]), "+v"(o[1][1]), "+v"(o[1][2]), "+v"(o[1][3]), "+v"(o[1][4]), "+v"(o[1][5]), "+v"(o[1][6]), "+v"(o[1][7]),
                   "+v"(o[2][0]), "+v"(o[2][1]), "+v"(o[2][2]), "+v"(o[2][3]), "+v"(o[2][4]), "+v"(o[2][5]), "+v"(o[2][6]), "+v"(o[2][7]),
                   "+v"(o[3][0]), "+v"(o[3][1]), "+v"(o[3][2]), "+v"(o[3][3]), "+v"(o[3][4]), "+v"(o[3][5]), "+v"(o[3][6]), "+v"(o[3][7]),
                   [f] "=&v"(f), [t0] "=&v"(t0), [t1] "=&v"(t1), [t2] "=&v"(t2), [t3] "=&v"(t3)
                 : [a] "v"(a), [own] "v"(own), [on] "s"(on)
                 : "memory", "scc");
}

// Values of a tree tile that are not finite become zeros, in the panels that one wavefront of O^T reads (the scores are made by then).
// Rows that do not see such a node have a weight of zero for it, and the product with its values would be NaN; a row that sees it is NaN by
// its score.
__device__ __forceinline__ void clear_wrong(unsigned char *panels, int lane, int bytes)
{
#pragma unroll 1
    for (int k = lane * 16; k < bytes; k += 1024) {
        u32x4_t v = *(const u32x4_t *)(panels + k);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if ((v[i] & 0x7f80u) == 0x7f80u) v[i] &= 0xffff0000u;
            if ((v[i] & 0x7f800000u) == 0x7f800000u) v[i] &= 0xffffu;
        }
        *(u32x4_t *)(panels + k) = v;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// A tile in LDS: panels of 64 channels, 128 bytes a row (the last panel has the d_rope channels).  The 16-byte chunk c of row r stands at
// c ^ swz(r), so that lanes served together hit different places of a bank row: 16-byte reads of 16 rows (served as lanes 0-3 with
// 20-23, 4-7 with 16-19 and so on: four rows at one chunk with the next four at its neighbour; with bits 2 and 3 of the row in plain
// order half of the cycles of these reads were conflicts) and transpose loads (rows 0-3 and 8-11 at two neighbouring chunks).
__device__ __forceinline__ int swz(int r) { return ((r >> 1) & 1) << 2 | ((r >> 3 ^ r >> 2) & 1) << 1 | ((r >> 2) & 1); }
// Rows of 64 bytes: a last panel of 32 channels, and the weights (a row's 32 keys).
__device__ __forceinline__ int swz_half(int r) { return ((r >> 2) & 1) << 1 | ((r >> 3) & 1); }

template <int DL_, int DR_>
struct Cfg {
    static constexpr int DL = DL_, DR = DR_, D = DL + DR, ROWB = 2 * D;
    static constexpr int KS = D / 32;                // matrix steps of S^T
    static constexpr int CB = DL / 64;               // blocks of 16 value channels of a wavefront
    static constexpr int PANELS = DL / 64, PANEL = KEYS * 128;
    static constexpr int TILE = KEYS * ROWB, STAGES = 4;
    static constexpr int LOADS = PANELS + 1;         // per wavefront and tile
    static constexpr int P_AT = STAGES * TILE, P_BYTES = ROWS * KEYS * 2;              // two of them
    static constexpr int MAX_AT = P_AT + 2 * P_BYTES;                                  // two words per row: maxima, or sums
    static constexpr int ALPHA_AT = MAX_AT + 2 * ROWS * 4, FLAG_AT = ALPHA_AT + ROWS * 4, LDS = FLAG_AT + 2 * 16;
    static_assert(LDS <= 160 * 1024 && (DR == 64 || DR == 32), "");
};

template <int DL, int DR, bool NT>
__global__ __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(2, 2))) void tree_attn_latent_kernel(const LatentParams args)
{
    constexpr int RG = 4;
#include "tree_attention_latent_body.h"
}
// (32 sequences of 192 keys, 16 heads, one node: 12.6 -> 10.0 us; of 777 to 8191 keys 40.4 -> 38.2.)
template <int DL, int DR>
__global__ __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(2, 2))) void tree_attn_latent_few_kernel(const LatentParams args)
{
    constexpr int RG = 1;
    constexpr bool NT = true;
#include "tree_attention_latent_body.h"
}

// grid (headers, slot_rows * DL / 1024): four channels of a row per thread, the unit's parts added up in order, eight of them asked for at
// once (one after the other each is a trip to memory).
template <int DL>
__global__ __launch_bounds__(256) void tree_attn_latent_fold_kernel(const LatentParams p)
{
    const LatentHeader h = p.header[blockIdx.x];
    constexpr int LANES = DL / 4;
    const int row = blockIdx.y * (256 / LANES) + threadIdx.x / LANES, r = h.chunk * ROWS + row, c = threadIdx.x % LANES * 4;
    if (h.pieces == 0 || row >= p.slot_rows || r >= p.rows) return;
    float m = -INFINITY, sum = 0.f;
    f32x4_t acc = {0, 0, 0, 0};
    for (int k0 = 0; k0 < h.pieces; k0 += 8) {
        float pm[8], pl[8], now = m;
        f32x4_t po[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int k = min(k0 + i, h.pieces - 1);
            const int64_t at = (int64_t)(k == 0 ? h.first : h.second + (k - 1) * h.stride) * p.slot_rows + row;
            pm[i] = p.part_m[at];
            pl[i] = p.part_l[at];
            po[i] = *(const f32x4_t *)(p.part_o + at * DL + c);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) now = fmaxf(now, pm[i]);
        const float a = m == now ? 1.f : fast_exp2(m - now);               // (equal: also where no part has seen a key)
        m = now;
        sum *= a;
        acc *= a;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (k0 + i >= h.pieces) break;
            const float e = pm[i] == now ? 1.f : fast_exp2(pm[i] - now);
            sum = fmaf(pl[i], e, sum);
            acc += po[i] * e;
        }
    }
    const int head = row_div(r, p.by_nrows), i = p.row0 + r - head * (p.n - p.row0);
    const f32x4_t y = acc * (1.f / sum);
    const u32x2_t pk = {__builtin_bit_cast(unsigned, (bf16x2_t){(__bf16)y[0], (__bf16)y[1]}),
                        __builtin_bit_cast(unsigned, (bf16x2_t){(__bf16)y[2], (__bf16)y[3]})};
    *(u32x2_t *)(p.out + (((int64_t)h.b * p.H + head) * p.node_stride + i) * DL + c) = pk;
}

// ---------------------------------------------------------------------------------------------------- host
struct LatentPlan {
    int chunks, workgroups, slot_rows;
    size_t bytes;                    // workspace; 0: no unit is ever cut.  (By the sizes alone, so that it serves smaller calls.)
    bool cut;                        // whether units may be cut
};

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// False where the work has more tiles than the kernel's numbers hold.
bool make_plan(int B, int H, int dl, int n_rows, int n, int max_prefix, LatentPlan &pl)
{
    const int64_t rows = (int64_t)H * n_rows, chunks = (rows + ROWS - 1) / ROWS, pairs = chunks * B;
    const int64_t tiles = (n + KEYS - 1) / KEYS + ((int64_t)max_prefix + KEYS - 1) / KEYS;
    if (rows > 0x3fffffff || pairs > 0x3fffffff || pairs * tiles > 0x3fffffff) return false;
    const int64_t pieces = pairs * ((tiles + MIN_TILES - 1) / MIN_TILES);
    const int cus = mcsd_compute_units();
    pl.chunks = (int)chunks;
    pl.workgroups = (int)(pieces < cus ? pieces : cus);
    pl.slot_rows = rows < ROWS ? (int)rows : ROWS;
    pl.bytes = 0;
    pl.cut = pieces > pairs || pairs > cus;
    if (pl.cut) {
        const size_t slots = (size_t)2 * pl.workgroups, slot_rows = slots * pl.slot_rows;
        pl.bytes = WS_HEADER + WS_CTR_BYTES + align256(pl.workgroups * sizeof(LatentHeader)) + 2 * align256(slot_rows * 4) + slot_rows * dl * 4;
    }
    // Cutting the longest unit saves (tiles - tiles of a piece) turns of 0.94 us (0.69 with 256 channels) and costs the plan and a second
    // launch, 4.5 us, and the parts' way out and back at 5.5 TB/s.  Two sequences x 128 heads x 14 nodes of 448 keys: whole 23.6 us, cut 26.2;
    // 8 x 16 heads x 44 nodes of 256 keys (256 channels): 13.7, cut 20.2; 4 x 16 heads x 1 node of 320 keys: cut 15.2, whole 16.7.  Of sequences
    // that differ, which the host does not know, more can be saved: of longer ones (16 x 512..4096 keys: 108 us, whole 134) all are planned.
    if (pl.cut && pairs <= cus && tiles <= UNCUT) {
        const int64_t at_once = cus / pairs, wanted = (tiles + MIN_TILES - 1) / MIN_TILES, n_pieces = at_once < wanted ? at_once : wanted;
        const double saved = (double)(tiles - (tiles + n_pieces - 1) / n_pieces) * (dl == 512 ? 0.94 : 0.69);
        if (saved <= 4.5 + (double)(pairs * n_pieces) * pl.slot_rows * dl * 8 / 5.5e6) {
            pl.cut = false;
            pl.workgroups = (int)pairs;
        }
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
    if (pl.cut) {
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
    // (non-temporal where a sequence's keys are read once)
    auto kernel = p.rows <= 16     ? (d_latent == 512 ? tree_attn_latent_few_kernel<512, 64> : tree_attn_latent_few_kernel<256, 32>)
                  : d_latent == 512 ? (pl.chunks == 1 ? tree_attn_latent_kernel<512, 64, true> : tree_attn_latent_kernel<512, 64, false>)
                                  : (pl.chunks == 1 ? tree_attn_latent_kernel<256, 32, true> : tree_attn_latent_kernel<256, 32, false>);
    mcsd_launch(MCSD_KERNEL_ATTN_SWEEP, kernel, dim3(pl.workgroups), dim3(THREADS), st, p);
    if (hipGetLastError() != hipSuccess) return MCSD_EHIP;
    if (pl.cut) {
        auto fold = d_latent == 512 ? tree_attn_latent_fold_kernel<512> : tree_attn_latent_fold_kernel<256>;
        const int64_t units = (int64_t)B * pl.chunks;
        const unsigned headers = (unsigned)(units < pl.workgroups ? units : pl.workgroups), rows = 1024u / d_latent;
        mcsd_launch(MCSD_KERNEL_ATTN_MERGE, fold, dim3(headers, (pl.slot_rows + rows - 1) / rows), dim3(256), st, p);
        return mcsd_hip_status(hipGetLastError());
    }
    return MCSD_OK;
}
