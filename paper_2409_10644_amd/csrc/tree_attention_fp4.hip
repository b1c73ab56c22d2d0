// Tree attention over a prefix cache in 4 bits (formulas and format in mcsd.h).
//
// A workgroup of 4 wavefronts serves up to 128 query rows of one (sequence, key/value head): the rows of the query heads that share
// the head, cut into blocks of 32, one block per wavefront; with fewer blocks the wavefronts of a block share its keys.  Scores are
// computed transposed, S^T = K Q^T, so a lane holds 16 keys of one query, the soft-max needs one exchange between half wavefronts,
// and the weights are the B operand of O^T += V^T P^T as they stand.
//
// K never leaves its 4 bits: gfx950 multiplies E2M1 operands with E8M0 scales per 32 contraction elements, which is a cache row as
// it is in memory (a lane's operand is 16 bytes of codes and a scale byte).  The other operand, the query times the soft-max scale
// and log2 e, is given as three E2M3 (6-bit) terms per group of 32 channels, each 2^-4 of the one before: 12 bits below the group's
// maximum, at 3/4 of the matrix time of bf16 operands and without a conversion of K.  The accumulators start at minus the running
// maximum, so that they come out as the exponents.
// V is converted once per tile: each wavefront turns its share of the rows into bf16 in LDS, from where the transpose load
// delivers V^T operands to all of them.
//
// Codes and scales stream from HBM straight into a ring of LDS stages.  The work is the tiles of all (sequence, head) pairs laid
// end to end, the tree's own keys first in each, cut into equal pieces for the workgroups that are resident at once, or, where
// that is as even, into equal pieces of each pair.  A pair's pieces leave their unnormalised output, maximum and sum in the
// workspace, and the workgroup that is last to do so folds them.
#include <math.h>

#include <atomic>

#include "fp4_format.h"

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(32))) float f32x32_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4_t;
typedef __attribute__((ext_vector_type(4))) int i32x4_t;
typedef __attribute__((ext_vector_type(6))) int i32x6_t;
typedef __attribute__((ext_vector_type(8))) int i32x8_t;

struct Fp4AttnParams {
    const uint16_t *q, *kt, *vt;
    uint16_t *out;
    mcsd_fp4_cache_t cache;
    const int64_t *seq_base;
    const int32_t *lens;
    const uint64_t *mask_bits;
    int64_t node_stride, head_stride;
    int32_t mask_words, B, H_q, H_kv, grp, n, row0, max_prefix;
    int32_t rows;                    // query rows per key/value head: grp * (n - row0)
    int32_t chunks;                  // workgroup units per key/value head
    int32_t units;                   // per sequence: H_kv * chunks
    RowDiv by_units, by_chunks, by_nrows;
    int32_t workgroups;              // of the launch: pieces that can be
    float c;                         // softmax scale * log2(e)
    const uint32_t *ws_tag;
    unsigned long long *ctr;         // arrivals of the pair that begins in piece w: ctr[w * CTR_STRIDE], zero before and after every launch
    float *part_m, *part_l, *part_o; // slots of 32 QBP rows: reference maximum (log2 units), sum, output
};

// Workspace: [tag word, 256 bytes] [arrival counters, 64 KiB], as mcsd_workspace_init prepares it, then [part_m] [part_l] [part_o].
constexpr uint32_t WS_TAG = 0x4d435344u;
constexpr size_t WS_HEADER = 256, WS_CTR_BYTES = 64 * 1024;
constexpr int CTR_STRIDE = 16;                       // a counter per 128-byte line: atomics on one line queue
constexpr int MAX_PIECES = (int)(WS_CTR_BYTES / 8 / CTR_STRIDE);
constexpr int MAX_SPLITS = 32;                       // pieces of one (sequence, head): one workgroup folds them

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float half_max(float v)
{
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v)
{
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ s16x4_t lds_read_tr16(const unsigned char *p)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4_t __attribute__((address_space(3))) *)(p));
}

template <int D_, int QBP_>
struct Cfg {
    static constexpr int D = D_, QBP = QBP_;
    static constexpr int KG = 4 / QBP;               // wavefronts that share a query block
    static constexpr int U = QBP == 4 ? 2 : 1;       // 32-key blocks per wavefront and tile
    static constexpr int T = 32 * KG * U;            // keys per tile: 64, 64, 128 for QBP = 4, 2, 1
    static constexpr int RW = T / 4;                 // rows that a wavefront brings and converts
    static constexpr bool OWN = QBP == 1;            // ... which are the ones it uses, and no one else
    static constexpr int ST = D / 64;                // matrix steps of S^T
    static constexpr int CB = D / 32;                // 32-row blocks of O^T
    static constexpr int RB = D / 2, SB = D / 32;    // bytes of codes and of scales per row
    static constexpr int GR = RB / 16;               // 16-byte pieces (groups) per row
    static constexpr int KB = RW * RB;               // a wavefront's K codes in a stage; V codes and 256 bytes for scales follow
    static constexpr int WB = 2 * KB + 256, STAGE = 4 * WB;
    static constexpr int LPT = (KB >= 1024 ? 2 * KB / 1024 : 1) + 1;   // loads per wavefront and tile
    static constexpr int VROWS = OWN ? 4 * 16 : T, VCOLS = VROWS * 64;   // V in LDS: rows, bytes of 32 columns
    static constexpr int VBUF = CB * VCOLS, NV = OWN ? 1 : 2;
    static constexpr int NS = OWN ? (D == 128 ? 3 : 4) : 5;            // stages; two workgroups per compute unit have 80 KB each
    static constexpr int RING = NS * STAGE;
    static constexpr int PP = CB * 4 / KG;           // pieces (four columns of a row per lane) that a wavefront ends up with
    static constexpr int XCHG = (KG - 1) * QBP * 32 * D * 4;
    static constexpr int LDS = RING + NV * VBUF > XCHG + 4 * 256 + 16 ? RING + NV * VBUF : XCHG + 4 * 256 + 16;
    static_assert(LDS <= 80 * 1024, "two workgroups per compute unit");
};

// V in LDS: 32 columns of all rows, 64 bytes each, then the next 32 columns (so that a transpose load takes the columns as an
// immediate offset).  Chunk c of row r stands at c ^ vswz(r): 16 consecutive rows written at one chunk hit 16 different places of a
// bank row; a transpose load reads 8 whole rows.
__device__ __forceinline__ int vswz(int r) { return (r >> 2) & 3; }
// Order of the groups of a row of codes, to the same end.
template <int D>
__device__ __forceinline__ int swz4(int r) { return D == 128 ? (r >> 2) & 3 : (r >> 3) & 1; }

// Log2 of what a score may exceed the running reference by before the accumulators are rescaled (exact either way).
constexpr float SLACK = 6.f;

template <int D>
struct Block {                       // a wavefront's 32 query rows
    i32x6_t term[D / 64][3];         // B operands: the lane's query, channels 64 st + 32 g .. +31, times c
    int scale[D / 64];               // their E8M0 scales in bytes 0, 1, 2
    f32x16_t start;                  // minus the reference maximum: what the accumulators of a tile start from
    f32x16_t o[D / 32];              // O^T
    float m_ref, l;                  // reference maximum in log2 units, the lane's part of the sum
};

__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// 32 numbers as three terms of E2M3 under scales 2^-4 apart.
__device__ __forceinline__ void query_terms(const float (&x)[32], i32x6_t (&term)[3], int &scale)
{
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
    int e = max((int)((m + 0x0fffffu) >> 23) - 2, 9);                  // so that no number is beyond 7.5 * 2^(e - 127)
    f32x16_t a, b;
#pragma unroll
    for (int i = 0; i < 16; ++i) { a[i] = x[2 * i]; b[i] = x[2 * i + 1]; }
#pragma unroll
    for (int t = 0; t < 3; ++t) {
        const float s = __uint_as_float((unsigned)(e - 4 * t) << 23);
        term[t] = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(a, b, s);   // (elements of the two operands in turn)
        if (t == 2) break;
        const f32x32_t back = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(term[t], s);
#pragma unroll
        for (int i = 0; i < 16; ++i) { a[i] -= back[2 * i]; b[i] -= back[2 * i + 1]; }
    }
    scale = m < 0x7f800000u ? e | (e - 4) << 8 | (e - 8) << 16 : 0xffffff;   // a NaN or an infinity: all of the row's scores are NaN
}

template <int T>
__device__ __forceinline__ f32x16_t mfma_fp4(const u32x4_t k, const i32x6_t q, f32x16_t c, int ks, int qs, int st)
{
    const i32x8_t a = {(int)k[0], (int)k[1], (int)k[2], (int)k[3], 0, 0, 0, 0}, b = {q[0], q[1], q[2], q[3], q[4], q[5], 0, 0};
    return st == 0 ? __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 2, 0, ks, T, qs)
                   : __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 2, 2, ks, T, qs);
}

// A value that the compiler knows nothing about: what is made of it is made here, not kept in registers from before the loops.
__device__ __forceinline__ int anew(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// Weights of a pair of scores, added to the sum and packed.
__device__ __forceinline__ void weigh2(const f32x16_t &s, int r, float &sum, u32x4_t *pb)
{
    const float p0 = fast_exp2(s[r]), p1 = fast_exp2(s[r + 1]);
    sum += p0 + p1;
    unsigned u = __builtin_bit_cast(unsigned, (bf16x2_t){(__bf16)p0, (__bf16)p1});
    asm volatile("" : "+v"(u));      // (stays where it is written, between two matrix instructions)
    pb[r / 8][(r % 8) / 2] = u;
}

// Soft-max and O^T += V^T P^T for the wavefront's U blocks of 32 scores (accumulators in log2 units, minus the reference).
// Where masked (uniform) bit k of bits[u] says whether key k of block u is seen.  read(i, vf) reads the V^T operands of 16 keys,
// number i of the wavefront's.
template <class C, typename Read>
__device__ __forceinline__ void absorb(f32x16_t (&sacc)[C::U], Block<C::D> &qs, const int g, const bool masked, const uint32_t *bits, Read read)
{
    constexpr int U = C::U, CB = C::CB;
    bf16x8_t vf[2][CB];
    read(0, vf[0]);
    read(1, vf[1]);
    float mx = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (masked) {
            const uint32_t own = bits[u] >> (4 * g);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const uint32_t seen = (uint32_t)__builtin_amdgcn_sbfe((int)own, 8 * (r / 4) + r % 4, 1);
                sacc[u][r] = __uint_as_float((__float_as_uint(sacc[u][r]) & seen) | (0xff800000u & ~seen));
            }
        }
#pragma unroll
        for (int r = 0; r < 16; r += 2) mx = fmaxf(fmaxf(mx, sacc[u][r]), sacc[u][r + 1]);
    }
    mx = half_max(mx);
    const bool none = qs.m_ref == -INFINITY;                           // no key seen yet: the accumulators started from zero
    const bool grow = none ? mx > -INFINITY : mx > SLACK;
    if (__builtin_amdgcn_ballot_w64(grow) != 0) {
        const float by = grow ? mx : 0.f, alpha = none ? 0.f : fast_exp2(-by);
        if (grow) qs.m_ref = (none ? 0.f : qs.m_ref) + mx;
        qs.l *= alpha;
        const float start = qs.m_ref == -INFINITY ? 0.f : -qs.m_ref;
#pragma unroll
        for (int r = 0; r < 16; ++r) qs.start[r] = start;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int r = 0; r < 16; ++r) qs.o[cb][r] *= alpha;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) sacc[u][r] -= by;
    }
    u32x4_t pb[U][2];
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < (U == 1 ? 8 : 16); r += 2) weigh2(sacc[0], r, sum, pb[0]);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (U == 2) __builtin_amdgcn_s_setprio(2);
    // 16 keys after 16 keys, the next ones' operands read and the weights of what is to come made in the shadow of the products
#pragma unroll
    for (int i = 0; i < 2 * U; ++i) {
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            qs.o[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i & 1][cb], __builtin_bit_cast(bf16x8_t, pb[i / 2][i & 1]), qs.o[cb], 0, 0, 0);
#pragma unroll
            for (int x = 0; x < 4 / CB; ++x) {
                const int k = cb * (4 / CB) + x;
                if (U == 1 && i == 0) weigh2(sacc[0], 8 + 2 * k, sum, pb[0]);
                if (U == 2 && i < 2) weigh2(sacc[U - 1], 8 * i + 2 * k, sum, pb[U - 1]);
            }
            if (i + 2 < 2 * U || U == 1) __builtin_amdgcn_sched_barrier(0);
        }
        if (i + 2 < 2 * U) {
            read(i + 2, vf[i & 1]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if constexpr (U == 2) __builtin_amdgcn_s_setprio(0);
    qs.l += sum;
}

// Inclusive sum over the wavefront.
__device__ __forceinline__ int wave_scan(int v, int lane)
{
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
        const int o = __shfl_up(v, x);
        if (lane >= x) v += o;
    }
    return v;
}
__device__ __forceinline__ int wave_last(int v) { return __builtin_amdgcn_readlane(v, 63); }
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Tiles of a sequence: the tree's, then the prefix's.
template <class C>
__device__ __forceinline__ int prefix_len(const Fp4AttnParams &p, int b) { return min(max(p.lens[b], 0), p.max_prefix); }

template <int D, int QBP>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void tree_attn_fp4_kernel(const Fp4AttnParams args, const int min_tiles)
{
    const Fp4AttnParams &p = args;
    using C = Cfg<D, QBP>;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[C::LDS];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int qb = wave % QBP, kg = wave / QBP, w = blockIdx.x;
    const int tree_tiles = (p.n + C::T - 1) / C::T;
    auto tiles_of = [&](int len) { return tree_tiles + (int)((unsigned)(len + C::T - 1) / C::T); };

    // ---- this workgroup's piece of the work: tiles [at, end) of the whole, or one split of one pair ----
    int total = 0, most = 0;                                           // tiles of one unit of every sequence
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        const int t = b0 + lane < p.B ? tiles_of(prefix_len<C>(p, b0 + lane)) : 0;
        total += wave_last(wave_scan(t, lane));
        int m = t;
#pragma unroll
        for (int x = 32; x; x >>= 1) m = max(m, __shfl_xor(m, x));
        most = max(most, uniform(m));
    }
    int per = max((total * p.units + p.workgroups - 1) / p.workgroups, min_tiles);       // tiles of a piece
    per = max(per, (most + MAX_SPLITS - 1) / MAX_SPLITS);
    int aligned = 0;                                                   // > 0: splits of that many tiles, no piece crosses a pair
    if (p.B * p.units <= p.workgroups && per >= most) {
        aligned = per;
    } else if (p.B * p.units <= p.workgroups && p.B <= 64) {
        // the smallest size whose splits fit the grid; lanes try one each
        const int cand = per + lane * (1 + per / 64);
        const int len_l = lane < p.B ? tiles_of(prefix_len<C>(p, lane)) : 0;
        int splits = 0;
        for (int b = 0; b < p.B; ++b) splits += (__builtin_amdgcn_readlane(len_l, b) + cand - 1) / cand;
        const unsigned long long fits = __builtin_amdgcn_ballot_w64(splits * p.units <= p.workgroups);
        if (fits) aligned = uniform(__shfl(cand, __builtin_ctzll(fits)));
        if (aligned > per + per / 8 + 2) aligned = 0;
    }
    if (aligned) per = aligned;
    // the sequence and unit in which the piece begins, and the tile of theirs; first piece of the unit
    int b = 0, unit = 0, tile = 0, n_pieces = 1, first_piece = 0, left = 0;
    {
        int before = 0;
        bool found = false;
        for (int b0 = 0; b0 < p.B && !found; b0 += 64) {
            const int t = b0 + lane < p.B ? tiles_of(prefix_len<C>(p, b0 + lane)) : 0;
            const int each = aligned ? (t + per - 1) / per : t;        // per unit: splits, or tiles
            const int upto = before + wave_scan(each * p.units, lane), here = aligned ? w : w * per;
            const unsigned long long mine = __builtin_amdgcn_ballot_w64(upto > here);
            if (mine) {
                const int l = __builtin_ctzll(mine);
                const int start = __builtin_amdgcn_readlane(upto - each * p.units, l), e = __builtin_amdgcn_readlane(each, l), t_l = __builtin_amdgcn_readlane(t, l);
                b = b0 + l;
                unit = (here - start) / e;
                const int in = here - start - unit * e;
                tile = aligned ? in * per : in;
                left = aligned ? min(per, t_l - tile) : per;
                if (aligned) { n_pieces = e; first_piece = w - in; }
                found = true;
            }
            before = wave_last(upto);
        }
        if (!found) return;
    }
    b = uniform(b); unit = uniform(unit); tile = uniform(tile); left = uniform(left); n_pieces = uniform(n_pieces); first_piece = uniform(first_piece);
    int64_t done = (int64_t)w * per;                                   // flat: tiles before this one

    // ---- what stays the same for all pairs ----
    const int chunk_rows = 32 * QBP, n_rows = p.n - p.row0;
    while (left > 0) {
        // (addresses made anew for every piece: kept over the fold they would be in memory in the loops)
        const int lane = anew(tid) & 63, g = lane >> 5, ln = lane & 31;
        // offsets of this lane's pieces of a tile: its own rows of codes, 16 bytes at a time, in the order that swz4 says
        const int f_row = lane / C::GR, f_grp = (lane % C::GR) ^ swz4<D>(f_row);
        const int f_rows_per = 64 / C::GR;                                 // rows covered by a load
        const int sc_idx = min(lane & 31, C::RW * C::SB / 4 - 1);
        unsigned char *const stage0 = lds + wave * C::WB;
        // operand addresses: the lane's K row in its first block (the second is two wavefronts' rows on) and its scales, V^T pieces
        int k_at[C::ST], ks_at, v_lo, v_hi;
        {
            const int r = kg * C::U * 32 + ln, rr = r % C::RW, from = (r / C::RW) * C::WB;
#pragma unroll
            for (int st = 0; st < C::ST; ++st) k_at[st] = from + rr * C::RB + (((2 * st + g) ^ swz4<D>(rr)) * 16);
            ks_at = from + 2 * C::KB + rr * C::SB;
            const int j = ln & 15, chunk = (ln >> 4) * 2 + ((j & 3) >> 1), row = (C::OWN ? wave * 16 : kg * C::U * 32) + 4 * g + (j >> 2);
            v_lo = C::RING + row * 64 + ((chunk ^ vswz(row)) * 16) + (j & 1) * 8;
            v_hi = C::RING + (row + 8) * 64 + ((chunk ^ vswz(row + 8)) * 16) + (j & 1) * 8;
        }
        constexpr int K_BLOCK = 32 / C::RW * C::WB;
        const int d_row = lane & 15, d_unit = lane >> 4;                   // the lane's quarter row when V is converted
        // ---- a piece of one pair: tiles [tile, tile + n) of sequence b, unit ----
        const int L = uniform(prefix_len<C>(p, b)), all = tiles_of(L);
        const int n = min(left, all - tile), end = tile + n;
        const int kvh = row_div(unit, p.by_chunks), chunk = unit - kvh * p.chunks;
        const int64_t pre = p.seq_base[b] + kvh * p.head_stride, tree = ((int64_t)b * p.H_kv + kvh) * p.node_stride * D;
        // the lane's query row: its node, and where it is in q and out
        auto row_of = [&](int ln, int &node) __attribute__((always_inline)) {
            const int row_c = min(chunk * chunk_rows + qb * 32 + ln, p.rows - 1), hq = row_div(row_c, p.by_nrows);
            node = p.row0 + row_c - hq * n_rows;
            return (((int64_t)b * p.H_q + kvh * p.grp + hq) * p.node_stride + node) * D;
        };
        const int t0 = max(tile - tree_tiles, 0), t1 = max(end - tree_tiles, 0), n_pre = t1 - t0;     // prefix tiles
        const int n_tree = max(min(end, tree_tiles) - tile, 0);
        const unsigned char *kc = (const unsigned char *)p.cache.k_codes + pre / 2, *vc = (const unsigned char *)p.cache.v_codes + pre / 2;
        const unsigned char *ksc = (const unsigned char *)p.cache.k_scales + pre / 32, *vsc = (const unsigned char *)p.cache.v_scales + pre / 32;

        // a tile's codes and scales into stage s; rows beyond the last key repeat it
        auto issue = [&](int x, int s) __attribute__((always_inline)) {
            const int r0 = (t0 + x) * C::T + wave * C::RW, last = L - 1 - r0;        // (may be negative: a wavefront without keys)
            unsigned char *to = stage0 + s * C::STAGE;
            const int64_t base = (int64_t)r0 * C::RB;
            if constexpr (C::KB >= 1024) {
#pragma unroll
                for (int i = 0; i < C::KB / 1024; ++i) {
                    const int64_t off = base + (int64_t)min(f_row + i * f_rows_per, last) * C::RB + f_grp * 16;
                    load_to_lds16_at(kc + off, to + i * 1024);
                    load_to_lds16_at(vc + off, to + C::KB + i * 1024);
                }
            } else {
                // half a load each: the upper lanes bring V
                const int l = lane & 31, fr = l / C::GR, fg = (l % C::GR) ^ swz4<D>(fr);
                const int64_t off = base + (int64_t)min(fr, last) * C::RB + fg * 16;
                load_to_lds16_at((g ? vc : kc) + off, to);
            }
            const int64_t sb = (int64_t)r0 * C::SB + min(sc_idx * 4, (last * C::SB) & ~3);
            load_to_lds4_at((g ? vsc : ksc) + sb, to + 2 * C::KB);
        };
        // 16 of this wavefront's V rows as bf16: rows `half` * 16 .. of its stage, of which `valid` exist
        auto convert = [&](int s, int half, int vbuf, int valid) __attribute__((always_inline)) {
            const unsigned char *from = stage0 + s * C::STAGE + C::KB;
            const int r = half * 16 + d_row;
            unsigned code[D / 32];
            if constexpr (D == 128) {
                const uint4 c4 = *(const uint4 *)(from + r * C::RB + ((d_unit ^ swz4<D>(r)) * 16));
                code[0] = c4.x; code[1] = c4.y; code[2] = c4.z; code[3] = c4.w;
            } else {
                const uint2 c2 = *(const uint2 *)(from + r * C::RB + (((d_unit >> 1) ^ swz4<D>(r)) * 16) + (d_unit & 1) * 8);
                code[0] = c2.x; code[1] = c2.y;
            }
            unsigned byte = from[C::KB + 128 + r * C::SB + (D == 128 ? d_unit : d_unit >> 1)];
            if (valid < C::RW) {                                       // (uniform) beyond the last key: zeros, whatever stands there
                byte = r < valid ? byte : 127u;
#pragma unroll
                for (int i = 0; i < D / 32; ++i) code[i] = r < valid ? code[i] : 0u;
            }
            const float scale = fp4_scale(byte);
            unsigned char *to = lds + C::RING + vbuf + (wave * 16 + d_row) * 64 + (D == 128 ? d_unit : d_unit >> 1) * C::VCOLS;
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
                *(uint4 *)(to + (((D == 128 ? i : (d_unit & 1) * 2 + i) ^ vswz(d_row)) * 16)) = fp4x8_to_bf16(code[i], scale);
        };
        // V^T operands of 16 keys from row `rows` of the wavefront's on
        auto read16 = [&](int vbuf, int rows, bf16x8_t (&vf)[C::CB]) __attribute__((always_inline)) {
#pragma unroll
            for (int cb = 0; cb < C::CB; ++cb) {
                const s16x4_t lo = lds_read_tr16(lds + (v_lo + vbuf) + rows * 64 + cb * C::VCOLS);
                const s16x4_t hi = lds_read_tr16(lds + (v_hi + vbuf) + rows * 64 + cb * C::VCOLS);
                vf[cb] = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            }
        };
        auto wait_for = [&](int later) __attribute__((always_inline)) {  // all loads but those of `later` tiles
            if (later >= 3) MCSD_WAIT_VMCNT(3 * C::LPT);
            else if (later == 2) MCSD_WAIT_VMCNT(2 * C::LPT);
            else if (later == 1) MCSD_WAIT_VMCNT(C::LPT);
            else MCSD_WAIT_VMCNT(0);
            asm volatile("" ::: "memory");
        };

        __syncthreads();                                               // (LDS is free: the piece before may have folded in it)
        Block<D> qs;
#pragma unroll
        for (int x = 0; x < C::NS - 1; ++x)
            if (x < n_pre) issue(x, x);
        // ---- the queries as terms ----
        if (n_pre > 0) {
            int node;
            const int64_t q_row = row_of(anew(ln), node);
#pragma unroll
            for (int st = 0; st < C::ST; ++st) {
                float x[32];
                const uint4 *qp = (const uint4 *)(p.q + q_row + st * 64 + g * 32);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint4 v = qp[i];
                    const unsigned wv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        x[8 * i + 2 * y] = __uint_as_float(wv[y] << 16) * p.c;
                        x[8 * i + 2 * y + 1] = __uint_as_float(wv[y] & 0xffff0000u) * p.c;
                    }
                }
                query_terms(x, qs.term[st], qs.scale[st]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int cb = 0; cb < C::CB; ++cb) qs.o[cb] = (f32x16_t){0};
        qs.start = (f32x16_t){0};
        qs.m_ref = -INFINITY;
        qs.l = 0.f;

        // ---- the tree's own keys: bf16 operands straight from memory, values through LDS ----
        for (int t = 0; t < n_tree; ++t) {
            const int key0 = (tile + t) * C::T, lane = anew(tid) & 63, g = lane >> 5, ln = lane & 31;
            int node;
            const int64_t q_row = row_of(ln, node);
            const uint64_t *mrow = p.mask_bits + (int64_t)node * p.mask_words;
            f32x16_t sacc[C::U];
            uint32_t bits[C::U];
#pragma unroll
            for (int u = 0; u < C::U; ++u) {
                const int k0 = key0 + (kg * C::U + u) * 32;
                bits[u] = (k0 >> 6) < p.mask_words && k0 < p.n ? (uint32_t)(mrow[k0 >> 6] >> (k0 & 63)) : 0u;
                sacc[u] = (f32x16_t){0};
                const uint16_t *kr = p.kt + tree + (int64_t)min(k0 + ln, p.n - 1) * D + g * 8, *qr = p.q + q_row + g * 8;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    sacc[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8_t *)(kr + ks * 16), *(const bf16x8_t *)(qr + ks * 16), sacc[u], 0, 0, 0);
                    if (ks % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) sacc[u][r] = fmaf(sacc[u][r], p.c, qs.start[0]);
                __builtin_amdgcn_sched_barrier(0);
            }
            // values: rows beyond the tree are zeros, and so is what is no number: a weight of zero would make it NaN for rows
            // that do not see it, so those are added below where they are seen
            bool odd = false;
            auto bring = [&](int r_tile) {                             // 16 rows, to where this wavefront converts them otherwise
                constexpr int CH = D / 8;
#pragma unroll
                for (int i = 0; i < CH / 4; ++i) {                     // 16 rows of CH chunks
                    const int x = i * 64 + lane, r = x / CH, ch = x % CH, key = key0 + r_tile + r;
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (key < p.n) v = *(const uint4 *)(p.vt + tree + (int64_t)key * D + ch * 8);
                    unsigned wv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const bool lo = (wv[y] & 0x7f80u) == 0x7f80u, hi = (wv[y] & 0x7f800000u) == 0x7f800000u;
                        odd |= lo | hi;
                        wv[y] &= (lo ? 0xffff0000u : 0xffffffffu) & (hi ? 0xffffu : 0xffffffffu);
                    }
                    *(uint4 *)(lds + C::RING + (ch / 4) * C::VCOLS + (wave * 16 + r) * 64 + (((ch % 4) ^ vswz(r)) * 16)) = make_uint4(wv[0], wv[1], wv[2], wv[3]);
                }
            };
            if constexpr (C::OWN) {
                absorb<C>(sacc, qs, g, true, bits, [&](int i, bf16x8_t (&vf)[C::CB]) {
                    bring(wave * 32 + i * 16);
                    read16(0, 0, vf);
                });
            } else {
                bring(wave * 16);
                meet();
                absorb<C>(sacc, qs, g, true, bits, [&](int i, bf16x8_t (&vf)[C::CB]) { read16(0, i * 16, vf); });
            }
            if (__syncthreads_or(odd)) {                               // (rare)
                for (int u = 0; u < C::U; ++u)
                    for (int k = 0; k < 32; ++k) {
                        const int key = key0 + (kg * C::U + u) * 32 + k;
                        if (key >= p.n || !((bits[u] >> k) & 1)) continue;
#pragma unroll
                        for (int cb = 0; cb < C::CB; ++cb) {
                            const uint16_t *vr = p.vt + tree + (int64_t)key * D + cb * 32 + 4 * g;
#pragma unroll
                            for (int r = 0; r < 16; ++r) {
                                const unsigned v = vr[8 * (r / 4) + r % 4];
                                qs.o[cb][r] += (v & 0x7f80u) == 0x7f80u ? __uint_as_float(v << 16) : 0.f;
                            }
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
            }
        }
        // ---- the prefix ----
        if constexpr (!C::OWN) {
            if (n_pre > 0) {
                wait_for(min(n_pre, C::NS - 1) - 1);
                convert(0, 0, 0, L - t0 * C::T - wave * C::RW);
            }
        }
        int s = 0;                                                     // stage of tile x
        for (int x = 0; x < n_pre; ++x) {
            const int s1 = s + 1 == C::NS ? 0 : s + 1, s_free = s == 0 ? C::NS - 1 : s - 1;
            const int vbuf = C::OWN ? 0 : (x & 1) * C::VBUF;
            if constexpr (!C::OWN) meet();                             // tile x is here and converted; everyone is done with the one before
            if (C::OWN) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (x + C::NS - 1 < n_pre) issue(x + C::NS - 1, s_free);
            if constexpr (C::OWN) wait_for(min(n_pre - 1 - x, C::NS - 1));
            const unsigned char *stage = lds + s * C::STAGE;
            f32x16_t sacc[C::U];
#pragma unroll
            for (int u = 0; u < C::U; ++u) {
                u32x4_t k[C::ST];
#pragma unroll
                for (int st = 0; st < C::ST; ++st) k[st] = *(const u32x4_t *)(stage + k_at[st] + u * K_BLOCK);
                int ks;
                if constexpr (D == 128) ks = *(const int *)(stage + ks_at + u * K_BLOCK) >> (8 * g);
                else ks = *(const uint16_t *)(stage + ks_at + u * K_BLOCK) >> (8 * g);
                if (u == 0) __builtin_amdgcn_s_setprio(2);
                sacc[u] = qs.start;
#pragma unroll
                for (int st = 0; st < C::ST; ++st) {
                    sacc[u] = mfma_fp4<2>(k[st], qs.term[st][2], sacc[u], ks, qs.scale[st], st);
                    sacc[u] = mfma_fp4<1>(k[st], qs.term[st][1], sacc[u], ks, qs.scale[st], st);
                    sacc[u] = mfma_fp4<0>(k[st], qs.term[st][0], sacc[u], ks, qs.scale[st], st);
                }
            }
            __builtin_amdgcn_s_setprio(0);
            const int valid = L - (t0 + x) * C::T;                     // keys of this tile that exist
            if constexpr (!C::OWN) {
                if (x + 1 < n_pre) {
                    wait_for(min(n_pre - 2 - x, C::NS - 2));
                    convert(s1, 0, C::VBUF - vbuf, valid - C::T - wave * C::RW);
                }
            }
            uint32_t bits[C::U];
#pragma unroll
            for (int u = 0; u < C::U; ++u) {
                const int here = valid - (kg * C::U + u) * 32;
                bits[u] = here >= 32 ? 0xffffffffu : here <= 0 ? 0u : (1u << here) - 1u;
            }
            absorb<C>(sacc, qs, g, valid < C::T, bits, [&](int i, bf16x8_t (&vf)[C::CB]) __attribute__((always_inline)) {
                if constexpr (C::OWN) {
                    convert(s, i, 0, valid - wave * C::RW);
                    read16(0, 0, vf);
                } else {
                    read16(vbuf, i * 16, vf);
                }
            });
            s = s1;
        }
        __syncthreads();

        // ---- the wavefronts that share a block put their parts together; each ends up with PP pieces of its rows ----
        {
            float l_tot = half_sum(qs.l);
            f32x4_t acc[C::PP];
            const int lane = anew(tid) & 63, g = lane >> 5, ln = lane & 31;
            const auto piece = [&](int x) {
                f32x4_t v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = qs.o[x >> 2][4 * (x & 3) + e];
                return v;
            };
            if constexpr (C::KG == 1) {
#pragma unroll
                for (int x = 0; x < C::PP; ++x) acc[x] = piece(x);
            } else {
                float *ml = (float *)(lds + C::XCHG);
                auto at = [&](int o, int r, int x) { return (f32x4_t *)(lds + ((((o * (C::KG - 1) + r) * QBP + qb) * C::PP + x) * 64 + lane) * 16); };
#pragma unroll
                for (int o = 0; o < C::KG; ++o) {
                    if (o == kg) {
#pragma unroll
                        for (int x = 0; x < C::PP; ++x) acc[x] = piece(o * C::PP + x);
                    } else {
#pragma unroll
                        for (int x = 0; x < C::PP; ++x) *at(o, kg < o ? kg : kg - 1, x) = piece(o * C::PP + x);
                    }
                }
                if (g == 0) {
                    ml[(kg * QBP + qb) * 64 + ln] = qs.m_ref;
                    ml[(kg * QBP + qb) * 64 + 32 + ln] = l_tot;
                }
                __syncthreads();
                float m[C::KG], M = -INFINITY;
#pragma unroll
                for (int k = 0; k < C::KG; ++k) {
                    m[k] = ml[(k * QBP + qb) * 64 + ln];
                    M = fmaxf(M, m[k]);
                }
                const float Mf = M == -INFINITY ? 0.f : M;
                l_tot = 0.f;
#pragma unroll
                for (int k = 0; k < C::KG; ++k) l_tot = fmaf(ml[(k * QBP + qb) * 64 + 32 + ln], fast_exp2(m[k] - Mf), l_tot);
                const float own = fast_exp2(qs.m_ref - Mf);
#pragma unroll
                for (int x = 0; x < C::PP; ++x) acc[x] *= own;
#pragma unroll
                for (int r = 0; r < C::KG - 1; ++r) {
                    const float wgt = fast_exp2(ml[((r < kg ? r : r + 1) * QBP + qb) * 64 + ln] - Mf);
#pragma unroll
                    for (int x = 0; x < C::PP; ++x) acc[x] += *at(kg, r, x) * wgt;
                }
                qs.m_ref = M;
            }
            int node;
            uint16_t *const orow = p.out + row_of(ln, node);
            const bool mine = chunk * chunk_rows + qb * 32 + ln < p.rows;
            auto write_out = [&](float inv) {
                if (!mine) return;
#pragma unroll
                for (int x = 0; x < C::PP; ++x) {
                    const int y = kg * C::PP + x;
                    bf16x4_t v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = (__bf16)(acc[x][e] * inv);
                    *(bf16x4_t *)(orow + (y >> 2) * 32 + 8 * (y & 3) + 4 * g) = v;
                }
            };
            if (n == all) {
                write_out(1.f / l_tot);
            } else {
                // ---- one of several pieces: leave it in the workspace; whoever is last folds them in order ----
                if (!aligned) {
                    first_piece = (int)((done - tile) / per);
                    n_pieces = (int)((done - tile + all - 1) / per) - first_piece + 1;
                }
                if (__hip_atomic_load(p.ws_tag, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != WS_TAG) {
#pragma unroll
                    for (int x = 0; x < C::PP; ++x) acc[x] = (f32x4_t){NAN, NAN, NAN, NAN};
                    write_out(1.f);                                        // never prepared: its counters mean nothing
                } else {
                    const int ln = anew(tid) & 31, g = (anew(tid) >> 5) & 1;
                    // slot of the piece: a workgroup leaves at most two, the first of them the end of a pair that began before
                    const auto slot_of = [&](int i) { return (int64_t)(2 * (first_piece + i) + (i == 0)); };
                    const int64_t slot = slot_of(w - first_piece);
                    constexpr int AGENT = 16;                              // (sc1: past this die's L2, for the other dies)
                    constexpr int ROWS = 32 * QBP;
                    if (mine) {
                        const auto ro = __builtin_amdgcn_make_buffer_rsrc((void *)(p.part_o + slot * ROWS * D), 0, ROWS * D * 4, 0x00027000);
#pragma unroll
                        for (int x = 0; x < C::PP; ++x)
                            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(i32x4_t, acc[x]), ro, (((qb * C::CB * 4 + kg * C::PP + x) * 2 + g) * 32 + ln) * 16, 0, AGENT);
                        if (kg == 0 && g == 0) {
                            __hip_atomic_store(p.part_m + slot * ROWS + qb * 32 + ln, qs.m_ref, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                            __hip_atomic_store(p.part_l + slot * ROWS + qb * 32 + ln, l_tot, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        }
                    }
                    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                    __syncthreads();
                    unsigned long long *const s_prev = (unsigned long long *)(lds + C::LDS - 16);
                    if (tid == 0) *s_prev = __hip_atomic_fetch_add(p.ctr + (int64_t)first_piece * CTR_STRIDE, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    __syncthreads();
                    if ((int)*s_prev + 1 == n_pieces) {
                        if (tid == 0) __hip_atomic_store(p.ctr + (int64_t)first_piece * CTR_STRIDE, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        float M = -INFINITY;
                        for (int i = 0; i < n_pieces; ++i)
                            M = fmaxf(M, __hip_atomic_load(p.part_m + slot_of(i) * ROWS + qb * 32 + ln, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
                        if (M == -INFINITY) M = 0.f;
                        float den = 0.f;
#pragma unroll
                        for (int x = 0; x < C::PP; ++x) acc[x] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
                        for (int i = 0; i < n_pieces; ++i) {
                            const int64_t sl = slot_of(i);
                            const float m = __hip_atomic_load(p.part_m + sl * ROWS + qb * 32 + ln, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                            const float lp = __hip_atomic_load(p.part_l + sl * ROWS + qb * 32 + ln, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                            const auto ro = __builtin_amdgcn_make_buffer_rsrc((void *)(p.part_o + sl * ROWS * D), 0, ROWS * D * 4, 0x00027000);
                            f32x4_t v[C::PP];
#pragma unroll
                            for (int x = 0; x < C::PP; ++x)
                                v[x] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(ro, (((qb * C::CB * 4 + kg * C::PP + x) * 2 + g) * 32 + ln) * 16, 0, AGENT));
                            const float wgt = fast_exp2(m - M);
                            den = fmaf(wgt, lp, den);
#pragma unroll
                            for (int x = 0; x < C::PP; ++x) acc[x] += wgt * v[x];
                        }
                        write_out(1.f / den);
                    }
                }
            }
        }
        done += n;
        left -= n;
        tile = 0;
        if (aligned) break;
        if (++unit == p.units) {
            unit = 0;
            if (++b == p.B) break;
        }
    }
}

// ---------------------------------------------------------------------------------------------------- host
struct Fp4Plan {
    int QBP, chunks, units, workgroups, min_tiles;
    size_t bytes;                    // workspace
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
bool make_plan(int B, int H_kv, int grp, int d, int n_rows, int n, int max_prefix, Fp4Plan &pl)
{
    const int64_t rows = (int64_t)grp * n_rows;
    pl.QBP = rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
    const int64_t chunks = (rows + 32 * pl.QBP - 1) / (32 * pl.QBP), units = chunks * H_kv;
    const int T = pl.QBP == 1 ? 128 : 64;
    const int64_t tiles = (n + T - 1) / T + ((int64_t)max_prefix + T - 1) / T;
    if (rows > 0x3fffffff || units * B > 0x3fffffff || units * B * tiles > 0x3fffffff) return false;
    pl.chunks = (int)chunks;
    pl.units = (int)units;
    pl.min_tiles = pl.QBP == 1 ? 2 : 4;
    int most = 2 * compute_units();
    if (most > MAX_PIECES) most = MAX_PIECES;
    const int64_t pairs = units * B, pieces = pairs * ((tiles + pl.min_tiles - 1) / pl.min_tiles);
    pl.workgroups = (int)(pieces < most ? pieces : most);
    pl.bytes = 0;
    if (pieces > pairs || pairs > most) {
        const size_t slot_rows = (size_t)2 * pl.workgroups * 32 * pl.QBP;
        pl.bytes = WS_HEADER + WS_CTR_BYTES + 2 * align256(slot_rows * 4) + slot_rows * d * 4;
    }
    return true;
}

template <int D>
void launch(const Fp4AttnParams &p, const Fp4Plan &pl, hipStream_t st)
{
    auto kernel = pl.QBP == 1 ? tree_attn_fp4_kernel<D, 1> : pl.QBP == 2 ? tree_attn_fp4_kernel<D, 2> : tree_attn_fp4_kernel<D, 4>;
    mcsd_launch(MCSD_KERNEL_ATTN_SWEEP, kernel, dim3(pl.workgroups), dim3(256), st, p, pl.min_tiles);
}

}  // namespace

extern "C" size_t mcsd_tree_attention_fp4kv_workspace(int32_t B, int32_t H_q, int32_t H_kv, int32_t d, int32_t n_nodes,
                                                      int32_t row_begin, int32_t max_prefix)
{
    if (B < 1 || H_q < 1 || H_kv < 1 || H_q % H_kv != 0 || (d != 64 && d != 128) || n_nodes < 1 || n_nodes > MCSD_ATTN_MAX_NODES ||
        max_prefix < 0 || row_begin < 0 || row_begin >= n_nodes)
        return 0;
    size_t most = 0;                 // of any number of rows up to this one
    for (int rows = 1; rows <= n_nodes - row_begin; ++rows) {
        Fp4Plan pl;
        if (make_plan(B, H_kv, H_q / H_kv, d, rows, n_nodes, max_prefix, pl) && pl.bytes > most) most = pl.bytes;
    }
    return most;
}

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
    if (hipGetDevice(&dev) != hipSuccess || dev != mask->device) {
        (void)hipGetLastError();
        return MCSD_EINVAL;
    }
    Fp4Plan pl;
    if (!make_plan(B, H_kv, H_q / H_kv, d, n - row_begin, n, max_prefix, pl)) return MCSD_EUNSUPPORTED;
    if (pl.bytes > 0 && (!workspace || workspace_bytes < pl.bytes || ((uintptr_t)workspace & 255))) return MCSD_EWORKSPACE;

    Fp4AttnParams p = {};
    p.q = (const uint16_t *)q; p.kt = (const uint16_t *)k_tree; p.vt = (const uint16_t *)v_tree; p.out = (uint16_t *)out;
    p.cache = *cache; p.seq_base = seq_base_dev; p.lens = prefix_lens_dev; p.mask_bits = mask->bits_dev;
    p.node_stride = node_stride; p.head_stride = head_stride; p.mask_words = mask->words_per_row;
    p.B = B; p.H_q = H_q; p.H_kv = H_kv; p.grp = H_q / H_kv; p.n = n; p.row0 = row_begin; p.max_prefix = max_prefix;
    p.rows = p.grp * (n - row_begin); p.chunks = pl.chunks; p.units = pl.units;
    p.by_units = row_div_of((uint32_t)pl.units); p.by_chunks = row_div_of((uint32_t)pl.chunks); p.by_nrows = row_div_of((uint32_t)(n - row_begin));
    p.workgroups = pl.workgroups;
    p.c = softmax_scale * 1.4426950408889634f;
    if (pl.bytes > 0) {
        char *ws = (char *)workspace;
        const size_t slot_rows = (size_t)2 * pl.workgroups * 32 * pl.QBP;
        p.ws_tag = (const uint32_t *)ws;
        p.ctr = (unsigned long long *)(ws + WS_HEADER);
        ws += WS_HEADER + WS_CTR_BYTES;
        p.part_m = (float *)ws;
        ws += align256(slot_rows * 4);
        p.part_l = (float *)ws;
        ws += align256(slot_rows * 4);
        p.part_o = (float *)ws;
    }
    if (d == 128) launch<128>(p, pl, (hipStream_t)hip_stream);
    else launch<64>(p, pl, (hipStream_t)hip_stream);
    return mcsd_hip_status(hipGetLastError());
}
