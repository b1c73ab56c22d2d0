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
constexpr int MIN_TILES = 4, CROSS = 12, UNCUT = 16;
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
    const LatentParams &p = args;
    using C = Cfg<DL, DR>;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[C::LDS];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int G = p.workgroups;
    // Neighbours in the order of the work share an L2: the hardware deals workgroups to the eight dies in turn.
    const int w = (G & 7) == 0 ? ((int)blockIdx.x & 7) * (G >> 3) + ((int)blockIdx.x >> 3) : (int)blockIdx.x;
    const int tree_tiles = (p.n + KEYS - 1) / KEYS;
    // ---- this workgroup's piece of the work.  Lengths and places of 64 sequences, one per lane (in most calls all of them: one trip to
    // memory).
    int b_lanes = 0, len_l = 0;
    int64_t base_l = 0;
    auto fetch = [&](int b0) __attribute__((always_inline)) {
        b_lanes = b0;
        len_l = -1;
        if (b0 + lane < p.B) {
            len_l = min(max(p.lens[b0 + lane], 0), p.max_prefix);
            base_l = p.seq_base[b0 + lane];
        }
    };
    const bool uncut = !p.header;                                          // one workgroup for every unit: nothing to plan
    if (!uncut) fetch(0);
    auto tiles_at = [&](int b0) __attribute__((always_inline)) {           // of sequence b0 + lane
        if (b0 != b_lanes) fetch(b0);
        return len_l >= 0 ? tree_tiles + (int)(((unsigned)len_l + KEYS - 1) / KEYS) : 0;
    };
    int total = 0, most = 0;
    for (int b0 = 0; b0 < p.B && !uncut; b0 += 64) {
        const int t = tiles_at(b0);
        total += wave_last(wave_scan(t));
        most = max(most, wave_max(t));
    }
    const int pairs = p.B * p.chunks, least = max(MIN_TILES, (int)(0.5f * __builtin_amdgcn_sqrtf((float)most)));
    int per = max((int)(((int64_t)total * p.chunks + G - 1) / G), least), aligned = 0;
    if (pairs <= G && !uncut) {
        if (per >= most) {
            aligned = per;
        } else {
            auto fits = [&](int size) {
                int sum = 0;
                for (int b0 = 0; b0 < p.B; b0 += 64) sum += wave_last(wave_scan(small_div(tiles_at(b0) + size - 1, size)));
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
    // Else as many teams as the chunks leave room for, one workgroup for every chunk, that go through all sequences' tiles in step: a tile
    // is read from memory once for all of its chunks then, and from the L2 by the others.  (Equal pieces of everything, where that would
    // leave too many workgroups without work, each at a place of its own: the ragged batch of 16 sequences of 512 to 4096 keys, 15 chunks
    // each, took 150 us, at 7 TB/s from behind the L2.)
    bool in_step = false;
    if (!aligned && !uncut && p.chunks <= G) {
        const int teams = G / p.chunks, of_team = max((total + teams - 1) / teams, least);
        in_step = (int64_t)of_team * 4 <= (int64_t)per * 5;
        if (in_step) per = of_team;
    }
    // b, chunk: where the piece begins; tile: its first tile there; left: its tiles in all
    int b = -1, chunk = 0, tile = 0, left = 0, n_pieces = 1, number = 0, each = 0;
    if (uncut) {
        b = small_div(w, p.chunks);
        chunk = w - b * p.chunks;
        left = 0x7fffffff;
        aligned = 1;
        fetch(b & ~63);
    } else if (aligned) {
        int before = 0;
        for (int b0 = 0; b0 < p.B && b < 0; b0 += 64) {
            const int t = tiles_at(b0), e = small_div(t + aligned - 1, aligned), s = wave_scan(e * p.chunks);
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
        const int64_t all = (int64_t)total * (in_step ? 1 : p.chunks), from = (int64_t)(in_step ? w / p.chunks : w) * per;
        const int each_seq = in_step ? 1 : p.chunks;
        int64_t before = 0;
        left = (int)max((int64_t)0, min((int64_t)per, all - from));
        for (int b0 = 0; b0 < p.B && b < 0 && left > 0; b0 += 64) {
            const int t = tiles_at(b0), s = wave_scan(t);
            const uint64_t beyond = __builtin_amdgcn_ballot_w64(from < before + (int64_t)s * each_seq);
            if (beyond) {
                const int l = __builtin_ctzll(beyond);
                b = b0 + l;
                const int tiles = __builtin_amdgcn_readlane(t, l);
                const int k = (int)(from - (before + (int64_t)(__builtin_amdgcn_readlane(s, l) - tiles) * each_seq));
                chunk = in_step ? w % p.chunks : k / tiles;
                tile = in_step ? k : k - chunk * tiles;
            }
            before += (int64_t)__builtin_amdgcn_readlane(s, 63) * each_seq;
        }
    }
    if (b < 0 || left <= 0) {
        if (tid == 0 && pairs > G) p.header[w].pieces = 0;
        return;
    }

    // ---- places of this lane
    const bool scorer = wave < 4;                                          // S^T and weights, else O^T
    const int part = wave & 3, rh = part & 1, kg = part >> 1;              // a scorer's rows 32 rh .. and keys 16 kg ..; else the channels DL / 4 part ..
    const int krow = 16 * kg + col;
    const int k_at = krow * 128 + ((grp ^ swz(krow)) << 4);                // panel's chunk grp; the other half of a panel: ^ 64
    const int k_half = C::PANELS * C::PANEL + krow * 64 + ((grp ^ swz_half(krow)) << 4);
    const int pw_at = C::P_AT + (32 * rh + col) * 64 + (((2 * kg + (grp >> 1)) ^ swz_half(col)) << 4) + (grp & 1) * 8;       // weights written; + 16 rows * 64
    const int pr_at = C::P_AT + col * 64 + ((grp ^ swz_half(col)) << 4);   // weights read
    const int jr = col >> 2, v_row = 8 * grp + jr;                         // of the 16 lanes of a transpose load: row (+ 4 for the second load), 4 channels
    const int v_at = v_row * 128 + ((((col & 3) >> 1) ^ swz(v_row)) << 4) + (col & 1) * 8 + part * (DL / 4) * (2 * KEYS);
    // Tile loads, by those of O^T: 8 rows of a panel per instruction.
    const int lrow = 8 * part + (lane >> 3);
    const uint32_t load_at = (uint32_t)(lrow * C::ROWB + (((lane & 7) ^ swz(lrow)) << 4));
    const int hrow = 16 * (part & 1) + (lane >> 2);                        // (half panels: 16 rows, two wavefronts bring the same)
    const uint32_t load_half = (uint32_t)(hrow * C::ROWB + C::PANELS * 128 + (((lane & 3) ^ swz_half(hrow)) << 4));

    for (bool begun = false;; begun = true) {
        b = uniform(b);
        chunk = uniform(chunk);
        tile = uniform(tile);
        left = uniform(left);
        if (b >= b_lanes + 64) fetch(b & ~63);
        const int len = __builtin_amdgcn_readlane(len_l, b - b_lanes), tiles = tree_tiles + (int)(((unsigned)len + KEYS - 1) / KEYS);
        const int from = tile, count = min(left, tiles - tile);
        const bool whole = from == 0 && count == tiles, first = from == 0, last = from + count == tiles;
        const int slot = aligned ? 2 * w : 2 * w + (begun ? 1 : 0);

        if (scorer) {
            // Query operands: rows col + 16 rg of this half of the chunk (behind the last: that one), channels 32 ks + 8 grp .. + 7.  They come by
            // way of the places of tiles 2 and 3, whole cache lines, once for both wavefronts that
            // share them (each by itself, 16 rows an instruction and half a line of each, waited 11500 cycles for them: 16 heads under 14 nodes and 128
            // keys 18.5 us instead of 15.9, 16 x 512..4096 keys under 60 nodes 115 instead of 108).
            // And which tree nodes the rows see among this lane's 4 keys: 4 bits per row and tree tile.
            bf16x8_t q[2][C::KS];
            uint64_t bits[2][2];
            unsigned char *const queries = lds + 2 * C::TILE;
            auto query_row = [&](int row, int &i) __attribute__((always_inline)) {                 // of the chunk: its place, its node
                const int r = min(chunk * ROWS + row, p.rows - 1), h = row_div(r, p.by_nrows);
                i = p.row0 + r - h * (p.n - p.row0);
                return (const unsigned char *)(p.q + (((int64_t)b * p.H + h) * p.node_stride + i) * C::D);
            };
#pragma unroll
            for (int half = 0; half < 2; ++half) {                         // 8 rows of a panel per instruction
                const int row = 16 * wave + 8 * half + (lane >> 3);
                int i;
                const unsigned char *src = query_row(row, i) + (((lane & 7) ^ swz(row & 15)) << 4);
#pragma unroll
                for (int x = 0; x < C::PANELS + (DR == 64); ++x) load_to_lds16_at(src + x * 128, queries + x * 2 * C::PANEL + (16 * wave + 8 * half) * 128);
            }
            if constexpr (DR == 32) {
                const int row = 16 * wave + (lane >> 2);
                int i;
                const unsigned char *src = query_row(row, i) + C::PANELS * 128 + (((lane & 3) ^ swz_half(row & 15)) << 4);
                load_to_lds16_at(src, queries + C::PANELS * 2 * C::PANEL + 16 * wave * 64);
            }
#pragma unroll
            for (int rg = 0; rg < 2; ++rg) {
                int i;
                query_row(32 * rh + 16 * rg + col, i);
                const uint64_t *row = p.mask_bits + (int64_t)i * p.mask_words;
                bits[rg][0] = row[0];
                bits[rg][1] = tree_tiles > 2 ? row[1] : 0;
            }
            MCSD_WAIT_VMCNT(0);
            meet();                                                        // the queries are here
#pragma unroll
            for (int rg = 0; rg < 2; ++rg)
#pragma unroll
                for (int ks = 0; ks < C::KS; ++ks) {
                    const int row = 32 * rh + 16 * rg + col;
                    q[rg][ks] = *(const bf16x8_t *)(queries + (DR == 32 && ks == C::KS - 1 ? C::PANELS * 2 * C::PANEL + row * 64 + ((grp ^ swz_half(col)) << 4)
                                                                                            : (ks >> 1) * 2 * C::PANEL + row * 128 + (((grp + 4 * (ks & 1)) ^ swz(col)) << 4)));
                }
            unsigned seen = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) seen |= (unsigned)((bits[k & 1][k >> 2] >> (32 * (k >> 1 & 1) + 16 * kg + 4 * grp)) & 15) << (4 * k);      // tile k / 2, rows k % 2
            float ref[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, start[2] = {0.f, 0.f};      // (start: minus the reference, 0 while no key has been seen)
            f32x4_t s[2];
            // Of tile t, whose scores s holds: its maxima over all keys, new references, its weights again; what O^T has of the tiles before is
            // multiplied by alpha.
            auto weigh = [&](int t, float (&sum)[2]) __attribute__((always_inline)) {
                unsigned char *pw = lds + pw_at + (t & 1) * C::P_BYTES;
#pragma unroll
                for (int rg = 0; rg < 2; ++rg) {
                    float e[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) e[i] = fast_exp2(fmaf(s[rg][i], p.c, start[rg]));
                    sum[rg] = (e[0] + e[1]) + (e[2] + e[3]);
                    const u32x2_t pk = {__builtin_bit_cast(unsigned, (bf16x2_t){(__bf16)e[0], (__bf16)e[1]}),
                                        __builtin_bit_cast(unsigned, (bf16x2_t){(__bf16)e[2], (__bf16)e[3]})};
                    *(u32x2_t *)(pw + rg * 16 * 64) = pk;
                }
            };
            float sum[2] = {0.f, 0.f};                                     // of the last tile's weights
            auto outgrown = [&](int t) __attribute__((always_inline)) {
#pragma unroll
                for (int rg = 0; rg < 2; ++rg) {
                    const float m = row_max(max4(s[rg]) * p.c);
                    if (grp == 0) *(float *)(lds + C::MAX_AT + (kg * ROWS + 32 * rh + 16 * rg + col) * 4) = m;
                }
                meet();
#pragma unroll
                for (int rg = 0; rg < 2; ++rg) {
                    const int row = 32 * rh + 16 * rg + col;
                    const float m = fmaxf(*(const float *)(lds + C::MAX_AT + row * 4), *(const float *)(lds + C::MAX_AT + (ROWS + row) * 4));
                    const float now = m > ref[rg] + SLACK ? m : ref[rg];
                    const float alpha = now == ref[rg] ? 1.f : fast_exp2(ref[rg] - now);
                    ref[rg] = now;
                    start[rg] = now == -INFINITY ? 0.f : -now;
                    l[rg] *= alpha;
                    if (kg == 0 && grp == 0) *(float *)(lds + C::ALPHA_AT + row * 4) = alpha;
                }
                weigh(t, sum);
                meet();
                meet();                                                    // (O^T uses the other place for weights until then)
            };
            auto flagged = [&](int t) __attribute__((always_inline)) { return *(const u32x4_t *)(lds + C::FLAG_AT + (t & 1) * 16); };
            meet();                                                        // the first tile is here
            for (int t = 0; t < count; ++t) {
                const int at = from + t, st = (t & 3) * C::TILE, k0 = anew(k_at) + st;
                auto key_of = [&](int ks) __attribute__((always_inline)) {
                    return *(const bf16x8_t *)(lds + (DR == 32 && ks == C::KS - 1 ? k_half + st : (k0 ^ ((ks & 1) << 6)) + (ks >> 1) * C::PANEL));
                };
                const u32x4_t flags = flagged(t - 1);                      // (looked at behind the products)
                f32x4_t n[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
                constexpr int AHEAD = 8;                                   // steps that key operands are read ahead
                bf16x8_t kf[AHEAD];
#pragma unroll
                for (int ks = 0; ks < AHEAD; ++ks) kf[ks] = key_of(ks);
                asm volatile("s_nop 1" : "+v"(n[0]), "+v"(n[1]));          // (two wait states from a vector instruction to a product that reads its result)
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int ks = 0; ks < C::KS; ++ks) {
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int rg = 0; rg < 2; ++rg) mfma(n[rg], kf[ks % AHEAD], q[rg][ks]);
                    if (ks + AHEAD < C::KS) kf[ks % AHEAD] = key_of(ks + AHEAD);
                }
                __builtin_amdgcn_sched_barrier(0);
                if (t > 0 && __builtin_expect((uniform((int)(flags[0] | flags[1] | flags[2] | flags[3])) & GROWN) != 0, 0)) outgrown(t - 1);
                settle();
#pragma unroll
                for (int rg = 0; rg < 2; ++rg) {
                    asm volatile("" : "+v"(n[rg]));
                    s[rg] = n[rg];
                    l[rg] += sum[rg];
                }
                const bool tree = at < tree_tiles;
                const int here = tree ? KEYS : len - (at - tree_tiles) * KEYS;
                bool wrong = false;
                if (tree || here < KEYS) {
                    unsigned bits;
                    if (tree) {
                        bits = seen >> (8 * at);
#pragma unroll
                        for (int rg = 0; rg < 2; ++rg)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                s[rg][i] += s[rg][i] - s[rg][i];           // (infinities as well are NaN)
                                wrong |= s[rg][i] != s[rg][i];
                            }
                    } else {
                        const int mine = min(max(here - 16 * kg - 4 * grp, 0), 4);
                        bits = ((1u << mine) - 1) * 0x11u;
                    }
#pragma unroll
                    for (int rg = 0; rg < 2; ++rg)
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[rg][i] = (bits >> (4 * rg + i)) & 1 ? s[rg][i] : -INFINITY;
                }
                weigh(t, sum);
                bool grow = false;
#pragma unroll
                for (int rg = 0; rg < 2; ++rg) grow |= max4(s[rg]) * p.c > ref[rg] + SLACK;
                const int flag = (__builtin_amdgcn_ballot_w64(grow) != 0 ? GROWN : 0) | (__builtin_amdgcn_ballot_w64(wrong) != 0 ? WRONG : 0);
                if (lane == 0) *(int *)(lds + C::FLAG_AT + (t & 1) * 16 + 4 * wave) = flag;
                __builtin_amdgcn_s_setprio(0);
                meet();
            }
            {
                const u32x4_t flags = flagged(count - 1);
                if (__builtin_expect((uniform((int)(flags[0] | flags[1] | flags[2] | flags[3])) & GROWN) != 0, 0)) outgrown(count - 1);
                l[0] += sum[0];
                l[1] += sum[1];
            }
            // sums and references of the rows, while O^T takes the last tile
#pragma unroll
            for (int rg = 0; rg < 2; ++rg) {
                const float sum = row_sum(l[rg]);
                const int row = 32 * rh + 16 * rg + col;
                if (grp == 0) *(float *)(lds + C::MAX_AT + (kg * ROWS + row) * 4) = sum;
                if (kg == 0 && grp == 0) *(float *)(lds + C::ALPHA_AT + row * 4) = ref[rg];
            }
            meet();
        } else {
            const int64_t base = (int64_t)__builtin_amdgcn_readlane((int)(base_l >> 32), b - b_lanes) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)base_l, b - b_lanes);
            const unsigned char *past = uniform((const unsigned char *)(p.cache + base));
            const unsigned char *nodes = uniform((const unsigned char *)(p.tree + (int64_t)b * p.node_stride * C::D));
            auto request = [&](int t) __attribute__((always_inline)) {     // tile t of this part, LOADS loads
                const int at = from + t, here = at < tree_tiles ? p.n - at * KEYS : len - (at - tree_tiles) * KEYS;      // keys of the tile (or more)
                const unsigned char *src = at < tree_tiles ? nodes + (int64_t)at * C::TILE : past + (int64_t)(at - tree_tiles) * C::TILE;
                unsigned char *dst = lds + (t & 3) * C::TILE + 8 * part * 128;
                const int row = anew(lrow);
                if (here >= KEYS) {
#pragma unroll
                    for (int x = 0; x < C::PANELS + (DR == 64); ++x) load_to_lds16<NT>(src + x * 128, load_at, dst + x * C::PANEL);
                    if constexpr (DR == 32) load_to_lds16<NT>(src, load_half, lds + (t & 3) * C::TILE + C::PANELS * C::PANEL + 16 * (part & 1) * 64);
                } else {                                                   // rows behind the last: zeros
#pragma unroll
                    for (int x = 0; x < C::PANELS + (DR == 64); ++x)
                        load_to_lds16_at(row < here ? src + x * 128 + load_at : no_row + (anew(lane) & 7) * 16, dst + x * C::PANEL);
                    if constexpr (DR == 32)
                        load_to_lds16_at(hrow < here ? src + load_half : no_row + (lane & 3) * 16, lds + (t & 3) * C::TILE + C::PANELS * C::PANEL + 16 * (part & 1) * 64);
                }
            };
            f32x4_t o[4][C::CB];
#pragma unroll
            for (int rg = 0; rg < 4; ++rg)
#pragma unroll
                for (int cb = 0; cb < C::CB; ++cb) o[rg][cb] = (f32x4_t){0, 0, 0, 0};
            request(0);
            if (count > 1) request(1);
            meet();                                                        // the queries are here
            if (count > 1) MCSD_WAIT_VMCNT(C::LOADS);
            else MCSD_WAIT_VMCNT(0);
            meet();                                                        // the first tile is here
            // In turn t, while the scores of tile t are made, tile t - 1 is added up, tile t + 2 requested into the place of tile t - 2, and
            // behind it tile t + 1 is here.
            if (count > 2) request(2);
            if (count > 2) MCSD_WAIT_VMCNT(C::LOADS);
            else MCSD_WAIT_VMCNT(0);
            meet();
            for (int t = 1;; ++t) {
                const int vb = anew(v_at) + ((t - 1) & 3) * C::TILE, pb = anew(pr_at) + ((t - 1) & 1) * C::P_BYTES;
                auto value_of = [&](int cb) __attribute__((always_inline)) {
                    const int a = vb ^ ((cb & 3) << 5), at = (cb >> 2) * C::PANEL;
                    const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4_t __attribute__((address_space(3))) *)(lds + a + at));
                    const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4_t __attribute__((address_space(3))) *)(lds + (a ^ 48) + at + 512));
                    return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                };
                const u32x4_t flags = *(const u32x4_t *)(lds + C::FLAG_AT + ((t - 1) & 1) * 16);
                constexpr int AHEAD = C::CB;                               // value operands read ahead
                bf16x8_t pf[4], vf[AHEAD];
#pragma unroll
                for (int rg = 0; rg < 4; ++rg) pf[rg] = *(const bf16x8_t *)(lds + pb + rg * 16 * 64);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int cb = 0; cb < AHEAD; ++cb) vf[cb] = value_of(cb);
                __builtin_amdgcn_sched_barrier(0);
                asm volatile("" : "+v"(pf[0]), "+v"(pf[1]), "+v"(pf[2]), "+v"(pf[3]));       // (one wait for weights and flags)
                const int flag = uniform((int)(flags[0] | flags[1] | flags[2] | flags[3])), on = flag & GROWN;
                if (__builtin_expect((flag & WRONG) != 0, 0)) {
                    clear_wrong(lds + ((t - 1) & 3) * C::TILE + part * (DL / 4) * (2 * KEYS), lane, DL / 4 * (2 * KEYS));
#pragma unroll
                    for (int cb = 0; cb < AHEAD; ++cb) vf[cb] = value_of(cb);
                }
                if (__builtin_expect(on != 0, 0)) {                        // a reference was outgrown by that tile
                    meet();
                    meet();
#pragma unroll
                    for (int rg = 0; rg < 4; ++rg) pf[rg] = *(const bf16x8_t *)(lds + pb + rg * 16 * 64);
                }
                const int own = lds_at(lds + C::P_AT) + (t & 1) * C::P_BYTES + part * 1024 + anew(lane) * 16;      // (weights that are done with)
                const int alpha = lds_at(lds + C::ALPHA_AT) + anew(col) * 4;
                multiply(t > 1 ? on : 0, o, alpha, own);                   // (before that it is zero)
                if (on) meet();
                const int next = t + 2, at = from + next, here = at < tree_tiles ? p.n - at * KEYS : len - (at - tree_tiles) * KEYS;
                const unsigned char *src = at < tree_tiles ? nodes + (int64_t)at * C::TILE : past + (int64_t)(at - tree_tiles) * C::TILE;
                unsigned char *dst = lds + (next & 3) * C::TILE;
                int ask = uniform(next < count && here >= KEYS ? 1 : 0);
                asm volatile("" : "+s"(ask));
                if (next < count && !ask) request(next);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int cb = 0; cb < C::CB; ++cb) {
#pragma unroll
                    for (int rg = 0; rg < 4; ++rg) mfma(o[rg][cb], vf[cb % AHEAD], pf[rg]);
                    if (cb + AHEAD < C::CB) vf[cb % AHEAD] = value_of(cb + AHEAD);
                    // (a load takes as long as the products of a block)
                    load_if<NT>(ask, src + cb * 128, load_at, dst + 8 * part * 128 + cb * C::PANEL);
                    if (cb == C::CB - 1) {
                        if constexpr (DR == 64) load_if<NT>(ask, src + C::PANELS * 128, load_at, dst + 8 * part * 128 + C::PANELS * C::PANEL);
                        else load_if<NT>(ask, src, load_half, dst + C::PANELS * C::PANEL + 16 * (part & 1) * 64);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (next < count) MCSD_WAIT_VMCNT(C::LOADS);
                else MCSD_WAIT_VMCNT(0);
                meet();
                if (t == count) break;
            }
            // ---- the rows' output, or this part of it: 16 rows x 128 bytes at a time by way of LDS (where weights were), so that a store
            // writes whole cache lines (8 bytes a lane from the registers, 32 a row, took 8200 cycles: 2 x 128 heads under 14 nodes and 192 keys 16.1 us
            // instead of 14.9).
#pragma unroll
            for (int rg = 0; rg < 4; ++rg) {
                settle();
                __builtin_amdgcn_sched_barrier(0);
                if (chunk * ROWS + 16 * rg >= p.rows) break;
                unsigned char *const own = lds + C::P_AT + part * 2048;
                const int at = anew(lane), own_row = at >> 3, own_at = own_row * 128 + (((at & 7) ^ own_row) << 4);
#pragma unroll
                for (int cb = 0; cb < C::CB; ++cb) asm volatile("" : "+v"(o[rg][cb]));
                const int c = at & 15, g = at >> 4, row = 16 * rg + c;
                const float sum = *(const float *)(lds + C::MAX_AT + row * 4) + *(const float *)(lds + C::MAX_AT + (ROWS + row) * 4);
                const float ref = *(const float *)(lds + C::ALPHA_AT + row * 4);
                unsigned char *dst[2];                                     // of rows own_row and own_row + 8
                bool there[2];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int row = 16 * rg + 8 * half + own_row, r = chunk * ROWS + row;
                    there[half] = r < p.rows;
                    if (whole) {
                        const int h = row_div(r, p.by_nrows), i = p.row0 + r - h * (p.n - p.row0);
                        dst[half] = (unsigned char *)(p.out + (((int64_t)b * p.H + h) * p.node_stride + i) * DL + part * (DL / 4) + (at & 7) * 8);
                    } else {
                        dst[half] = (unsigned char *)(p.part_o + ((int64_t)slot * p.slot_rows + row) * DL + part * (DL / 4) + (at & 7) * 4);
                    }
                }
                auto store = [&](int x) __attribute__((always_inline)) {
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const u32x4_t v = *(const u32x4_t *)(own + own_at + half * 1024);
                        if (there[half]) *(u32x4_t *)(dst[half] + x * 128) = v;
                    }
                };
                unsigned char *const to = own + c * 128;
                if (whole) {
                    const float inv = 1.f / sum;
#pragma unroll
                    for (int x = 0; x < C::CB / 4; ++x) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const f32x4_t y = o[rg][4 * x + k] * inv;
                            const u32x2_t pk = {__builtin_bit_cast(unsigned, (bf16x2_t){(__bf16)y[0], (__bf16)y[1]}),
                                                __builtin_bit_cast(unsigned, (bf16x2_t){(__bf16)y[2], (__bf16)y[3]})};
                            *(u32x2_t *)(to + (((2 * k + (g >> 1)) ^ (c & 7)) << 4) + (g & 1) * 8) = pk;
                        }
                        store(x);
                    }
                } else {
                    if (part == 0 && g == 0 && chunk * ROWS + row < p.rows) {
                        const int64_t of = (int64_t)slot * p.slot_rows + row;
                        p.part_m[of] = ref;
                        p.part_l[of] = sum;
                    }
#pragma unroll
                    for (int x = 0; x < C::CB / 2; ++x) {
#pragma unroll
                        for (int k = 0; k < 2; ++k) *(f32x4_t *)(to + (((4 * k + g) ^ (c & 7)) << 4)) = o[rg][2 * x + k];
                        store(x);
                    }
                }
            }
        }
        left -= count;
        const bool more = !aligned && left > 0;
        // What to fold: one word for every unit where no more of them than workgroups, else for every piece (only the last unit that begins
        // in it can go on in others).
        if (p.header && tid == 0 && (pairs <= G ? first : !more)) {
            LatentHeader h = {};
            if (first && !last) {                                          // it begins here: who goes on with it
                h.b = b;
                h.chunk = chunk;
                h.first = slot;
                h.stride = aligned || in_step ? 2 * p.chunks : 2;
                h.second = 2 * w + h.stride;
                h.pieces = aligned ? n_pieces : 1 + (tiles - count + per - 1) / per;
            }
            p.header[pairs <= G ? b * p.chunks + chunk : w] = h;
        }
        if (!more) return;
        tile = 0;
        if (in_step) {
            ++b;
        } else if (++chunk == p.chunks) {
            chunk = 0;
            ++b;
        }
    }
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
    auto kernel = d_latent == 512 ? (pl.chunks == 1 ? tree_attn_latent_kernel<512, 64, true> : tree_attn_latent_kernel<512, 64, false>)
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
