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
// end to end, the tree's own keys first in each, cut into pieces: equal ones of each pair where they fit the workgroups that are
// resident at once, else whole pairs, several to a workgroup, or equal pieces of the whole.  A pair's pieces leave their unnormalised output, maximum and sum in the
// workspace, and the workgroup that is last to do so folds them.
//
// With more than 32 rows, blocks of 32 keys go through a pipeline: between the matrix instructions that make the scores of one and
// add the one before it to the output stand the exponentials of the one in the middle; all that happens rarely (a reference that is
// outgrown, the last keys of a sequence) is behind one branch per block, which is not taken.
//
// What bounds it: 120 rows on 8 x 32 heads of 16384 keys take 264 us alone, 990 TFLOP/s of the products as defined (a large bf16
// matrix product of this card: 1200), and 254 to 312 by how many calls follow each other: the clock falls to 1.85 GHz under the matrix
// unit's load (five calls 254 to 258 us each, forty 302 to 311, two hundred 270); a loop of nothing but these 14 instructions per block
// takes 160.  With all operands zero the same work takes 226.  240 rows of 4 heads on 16 x 8 key heads of 512 to 4096 keys take 59 to
// 61 us (36 GFLOP), 44 rows on 32 heads of 1024 keys 17.9 to 18.6, most of it the way to the first key (8 us) and from the last one
// through the exchange (5 us); there, outside the loops, is also what the compiler keeps in memory (160 bytes a lane with 128 rows,
// 80 with 64).  One token of 4 heads on 32 x 8 key heads of 777 to 8191 keys takes 41 to 45 us for 157 MB, 3.5 to 3.8 TB/s; while all
// workgroups are in their loops the cache streams at 5.2 to 5.7.  The smallest call takes 7.7 to 8.5 us, a chain of trips to memory:
// lengths, queries, tree rows, prefix.  (Ranges: machines.  The pairs of figures at the rules below are of one machine and day.)
#include <math.h>

#include <type_traits>

#include "fp4_format.h"
#include "wave_ops.h"

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
    RowDiv by_chunks, by_nrows;
    int32_t workgroups, single;      // of the launch: pieces that can be; compute units
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
constexpr int KEPT = 256;                            // sequences whose lengths a workgroup keeps, one per thread
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
    static constexpr int NS = OWN ? (D == 128 ? 3 : 4) : 4;            // stages; two workgroups per compute unit have 80 KB each
    static constexpr int AHEAD = OWN ? NS - 1 : NS;  // tiles requested before the first is used
    static constexpr int RING = NS * STAGE;
    static constexpr int MIN_TILES = QBP == 1 ? 2 : QBP == 2 ? 4 : 8;
    static constexpr float FOLD = QBP == 4 ? 2.f : 0.5f;
    static constexpr int PP = CB * 4 / KG;           // pieces (four columns of a row per lane) that a wavefront ends up with
    static constexpr int XCHG = (KG - 1) * QBP * 32 * D * 4;
    static constexpr int LDS = RING + NV * VBUF > XCHG + 4 * 256 + 16 ? RING + NV * VBUF : XCHG + 4 * 256 + 16;
    static_assert(LDS + KEPT * 13 <= 80 * 1024, "two workgroups per compute unit");
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

// 32 numbers as three terms of E2M3 under scales 2^-4 apart.  The first scale s has the largest magnitude in (3.75 s, 7.5 s].  E2M3
// steps are 1/8 up to 2, 1/4 up to 4, 1/2 up to 7.5, so the terms leave at most 1/4 s, then 1/8 of s / 16, then 1/16 of s / 256:
// 2^-12 / 3.75 of the largest magnitude, for every channel alike (fixed point: one far below the largest keeps fewer bits than bf16
// gave it).  The choice: of 14 matrix instructions per block of 32 keys and 128 channels, 6 are for scores; two E4M3 terms would
// hold bf16 queries exactly over 17 binades, but take the time of 8, and the softmax scale would have to be applied to every score.
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
        // The instruction writes its first results while it still reads: operands that end with it may be given the result's
        // registers (seen with the scale: wrong third terms), so they are kept alive beyond it.
        asm volatile("" : : "v"(a), "v"(b), "v"(s), "v"(term[t]));
        if (t == 2) break;
        const f32x32_t back = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(term[t], s);
        asm volatile("" : : "v"(term[t]), "v"(s), "v"(back));
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

// Weights of a pair of scores, packed for the matrix unit, and their sum (in 32 bits; a dot product of the packed ones would occupy
// the matrix unit: 3 ns each beside it, measured).  They are rounded to bf16 for the product with V, as in the attention over the other
// caches: with random values the output is then off by 0.0021 to 0.0023 of its size instead of the 0.0017 of its own rounding.  A
// second bf16 term for what the first leaves would be 8 more matrix instructions beside 14.
__device__ __forceinline__ void weigh2(const f32x16_t &s, int r, float &sum, u32x4_t *pb)
{
    const float a = fast_exp2(s[r]), b = fast_exp2(s[r + 1]);
    unsigned u = __builtin_bit_cast(unsigned, (bf16x2_t){(__bf16)a, (__bf16)b});
    sum += a;
    sum += b;
    asm volatile("" : "+v"(u), "+v"(sum));      // (stays where it is written, between two matrix instructions)
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


template <int D, int QBP, bool NT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void tree_attn_fp4_kernel(const Fp4AttnParams args)
{
    const Fp4AttnParams &p = args;
    using C = Cfg<D, QBP>;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[C::LDS];
    __shared__ int64_t s_base[KEPT];                                   // of sequences `kept` on (all of up to KEPT): here while pairs are gone through
    __shared__ int32_t s_len[KEPT];
    __shared__ unsigned char s_order[KEPT];                            // by length, longest first
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int qb = wave % QBP, kg = wave / QBP, w = blockIdx.x;
    const int tree_tiles = (p.n + C::T - 1) / C::T;
    auto tiles_of = [&](int len) { return tree_tiles + (int)(((unsigned)len + C::T - 1) / C::T); };

    // ---- this workgroup's piece of the work: `left` tiles of the whole from tile `tile` of (b, unit) on, or a split of one pair ----
    // Lengths and bases of 64 sequences from b_lanes on, one per lane (in most calls those of all: one trip to memory).
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
    fetch(0);
    const bool prepared = p.ws_tag && uniform((int)*p.ws_tag) == (int)WS_TAG;
    int total = 0, most = 0;                                           // tiles of one unit of every sequence
    int kept = 0;
    auto keep = [&](int at) __attribute__((always_inline)) {           // (every wavefront writes the same, and reads what it wrote)
        s_len[at + lane] = len_l;
        s_base[at + lane] = base_l;
    };
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        if (b0) fetch(b0);
        if (p.B <= KEPT) keep(b0);                                     // (with more of them only the ones at hand, below)
        const int t = len_l >= 0 ? tiles_of(len_l) : 0;
        total += wave_last(wave_scan(t));
        most = max(most, wave_max(t));
    }
    // One workgroup per compute unit goes through its tiles 1.4 to 1.7 times as fast as one of two, and half as many pieces are half
    // as much to exchange: two only where each has more than so many tiles (or where pieces would cross pairs otherwise).  Measured,
    // one and two, in us: 60 nodes x 4 heads on 16 x 8 key heads of 512 keys 26.0 and 34.0, of 2048 54.0 and 54.8, of 4096 89.5 and
    // 82.6; 44 nodes on 8 x 32 key heads of 1024 keys 25.7 and 28.3, of 4096 57.1 and 51.6; one token x 4 heads on 32 x 8 key heads of
    // 1024 keys 20.2 and 23.6, of 4096 45.9 and 39.8.
    constexpr int WORTH = QBP == 1 ? 8 : 24;
    // Tiles of a piece: no fewer than make its share of the exchange worth while.  Of t tiles in pieces of s, s are one after the
    // other, and so are the t / s parts that the last one folds: the sum is least at a multiple of sqrt(t).  (120 nodes on 4 key
    // heads of 16384 keys, 257 tiles: pieces of 9 take 78 us, of 16 62.5, of 32 60.5; of 4096 keys: of 8 39.6, of 16 38.5, of 32
    // 43.2.  44 nodes on the same: of 8 28.4 and 22.0, of 16 30.1 and 22.7.  One token x 4 heads on 8 key heads of 4096 keys, 33 tiles:
    // of 2 17.8, of 4 18.2, of 8 19.7.)
    const int least = max(max(C::MIN_TILES, (int)(C::FOLD * __builtin_amdgcn_sqrtf((float)most))), (most + MAX_SPLITS - 1) / MAX_SPLITS);
    int per = 0, aligned = 0;                                          // aligned > 0: pieces of at most that many tiles, none crosses a pair
    for (int all = total * p.units >= 2 * p.single * WORTH; all < 2 && !aligned; ++all) {
        const int resident = all ? p.workgroups : min(p.single, p.workgroups);
        per = max((total * p.units + resident - 1) / resident, least);
        if (p.B * p.units > resident) continue;
        if (per >= most) {
            aligned = per;
        } else if (p.B <= 64) {
            // The smallest size whose splits fit the grid, unless it is so much more than an equal piece that crossing costs less.
            // (A piece of the next pair starts from nothing: 15 to 20 us.  The batch of 16 sequences of 512 to 4096 keys under 60
            // nodes takes 61 us in pieces of 24 tiles and 71 in equal ones of 19; 32 of 777 to 8191 keys with a token each 44.5, 60.  How
            // much more is looked at: nothing 73 and 61 us, half of it 62 and 44, this 61 and 44.5, twice 62 and 45.)
            const int t = len_l >= 0 ? tiles_of(len_l) : 0;
            auto fits = [&](int size) { return wave_last(wave_scan(small_div(t + size - 1, size))) * p.units <= resident; };
            int lo = per, hi = per + per / 8 + (QBP == 1 ? 12 : 8) * (1 + all);
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
    if (aligned) per = aligned;
    // 4 times the place of the lane's sequence when they are in order of `size`, largest first (lanes without one stay where they are)
    auto place_of = [&](int size) __attribute__((always_inline)) {
        int rank = lane;
        if (total < most * p.B && lane < p.B) {                        // (not all alike)
            const unsigned key = (unsigned)size * 64 + 63 - lane;      // (fewer than 2^26 tiles)
            rank = 0;
#pragma unroll 4
            for (int o = 0; o < p.B; ++o) rank += (unsigned)__builtin_amdgcn_readlane((int)key, o) > key;
        }
        return 4 * rank;
    };
    // Or whole pairs to every workgroup, the longest first, back and forth over the workgroups, where the fullest of them (of 64 looked
    // at) has less to do than one with an equal piece, which begins and ends within pairs.  Equal pieces and whole pairs, us: 44 nodes
    // on 64 x 32 heads of 100 to 2000 keys 269 and 132; 60 nodes x 4 heads on 64 x 8 key heads of 100 to 2000 169 and 100, on 32 x 8 of
    // 100 to 4000 155 and 98; one token on 64 x 32 heads of 100 to 2000 keys 184 and 96, of 4 heads on 128 x 8 key heads of 100 to 4000
    // 124 and 76.  With more than 32 pairs to a workgroup always: one token on 256 x 80 heads of 64, of 100 to 900 keys, 630 and 417, of
    // 500 keys each 382 and 395.
    constexpr int BEGIN = 5, CROSS = QBP == 4 ? 24 : 16;               // tiles that a new pair costs, and one that is begun or ended within
    const int pairs = p.B * p.units;
    int rounds = 0;                                                    // > 0: of whole pairs
    if (__builtin_expect(!aligned && p.B <= KEPT, 0)) {
        int rank = tid;
        if (total < most * p.B && tid < p.B) {                         // (not all alike)
            const int own = s_len[tid];
            rank = 0;
#pragma unroll 8
            for (int o = 0; o < p.B; ++o) {
                const int other = s_len[o];
                rank += other > own || (other == own && o < tid);
            }
        }
        s_order[rank] = (unsigned char)tid;
        __syncthreads();
        const int n = (pairs + p.workgroups - 1) / p.workgroups, who = lane * (p.workgroups - 1) / 63;
        int load = 0;
        for (int k = 0; k < min(n, 32); ++k) {
            const int at = k * p.workgroups + (k & 1 ? p.workgroups - 1 - who : who);
            const int t = tiles_of(s_len[s_order[min(small_div(at, p.units), p.B - 1)]]);
            load += at < pairs ? t : 0;
        }
        if (n > 32 || wave_max(load) + BEGIN * n <= per + CROSS * (pairs / p.workgroups + 1)) rounds = n;
    }
    int b = -1, unit = 0, tile = 0, n_pieces = 1, first_piece = 0, left = 0, number = w;
    {
        int before = 0, t = len_l >= 0 ? tiles_of(len_l) : 0, each = aligned ? small_div(t + per - 1, per) : t, seq = lane;
        if (aligned && p.B <= 64) {
            // Pieces of different sizes, two to a compute unit: the sequences by the size of their pieces, the first half of the
            // workgroups takes them from the largest on, the second half from the smallest on (workgroups come to the compute
            // units in turn, so the longest piece shares with the shortest: 44.5 us instead of 49.2 for 32 sequences of 777 to 8191
            // keys with a token each).
            const int pieces = wave_last(wave_scan(each * p.units));
            if (__builtin_expect(pieces > p.single, 0)) {
                const int place = place_of(each > 0 ? small_div(t + each - 1, each) : 0);
                t = __builtin_amdgcn_ds_permute(place, t);
                each = __builtin_amdgcn_ds_permute(place, each);
                seq = __builtin_amdgcn_ds_permute(place, lane);
                if (w >= p.single) number = pieces - 1 - (w - p.single);
                if (w >= p.single && number < p.single) return;
            }
        }
        const int here = aligned ? number : w * per;
        if (__builtin_expect(rounds, 0)) {
            if (w >= pairs) return;
            const int l = uniform(small_div(w, p.units));
            b = uniform(s_order[l]);
            unit = w - l * p.units;
            left = tiles_of(uniform(s_len[b]));
        }
        for (int b0 = 0; b0 < p.B && b < 0; b0 += 64) {
            if (__builtin_expect(p.B > 64, 0)) {
                if (b0 != b_lanes) fetch(b0);
                t = len_l >= 0 ? tiles_of(len_l) : 0;
                each = aligned ? small_div(t + per - 1, per) : t;      // per unit: splits, or tiles
            }
            const int upto = before + wave_scan(each * p.units);
            const unsigned long long mine = __builtin_amdgcn_ballot_w64(upto > here);
            if (mine) {
                const int l = __builtin_ctzll(mine), e = __builtin_amdgcn_readlane(each, l), t_l = __builtin_amdgcn_readlane(t, l);
                const int after = here - (__builtin_amdgcn_readlane(upto, l) - e * p.units);
                b = b0 + __builtin_amdgcn_readlane(seq, l);
                unit = uniform(small_div(after, e));
                const int in = after - unit * e;
                tile = in;
                left = per;
                if (aligned) {                                         // as equal as they can be
                    const int size = t_l / e, more = t_l - size * e;
                    tile = in * size + min(in, more);
                    left = size + (in < more);
                    n_pieces = e;
                    first_piece = number - in;
                }
            }
            before = wave_last(upto);
        }
        if (b < 0) return;
    }
    if (__builtin_expect(p.B > KEPT, 0)) {
        kept = b_lanes;
        keep(0);
    }
    int round = 0;
    int done = w * per;                                                // flat: tiles before this one

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
        if (__builtin_expect(p.B > KEPT && b >= kept + 64, 0)) {
            __syncthreads();
            kept = b;
            fetch(b);
            keep(0);
        }
        const int L = uniform(s_len[b - kept]), all = tiles_of(L);
        const int64_t s_at = s_base[b - kept];
        const int64_t seq_at = (int64_t)((uint64_t)(uint32_t)uniform((int)((uint64_t)s_at >> 32)) << 32 | (uint32_t)uniform((int)s_at));
        const int n = min(left, all - tile), end = tile + n;
        const int kvh = row_div(unit, p.by_chunks), chunk = unit - kvh * p.chunks;
        const int64_t pre = seq_at + kvh * p.head_stride, tree = ((int64_t)b * p.H_kv + kvh) * p.node_stride * D;
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
        const uint32_t f_at = f_row * C::RB + f_grp * 16;
        const int f_row2 = (lane & 31) / C::GR, f_grp2 = ((lane & 31) % C::GR) ^ swz4<D>(f_row2);      // half a load: the upper lanes bring V
        const unsigned char *const f_half = (g ? vc : kc) + f_row2 * C::RB + f_grp2 * 16, *const f_sc = (g ? vsc : ksc) + sc_idx * 4;
        auto issue = [&](int x, int at) __attribute__((always_inline)) {
            const int r0 = (t0 + x) * C::T + wave * C::RW, last = L - 1 - r0;        // (may be negative: a wavefront without keys)
            unsigned char *to = stage0 + at;
            const int64_t base = (int64_t)r0 * C::RB;
            if (__builtin_expect(last >= C::RW - 1, 1)) {
                if constexpr (C::KB >= 1024) {
                    // (read by one workgroup: not kept in the caches)
#pragma unroll
                    for (int i = 0; i < C::KB / 1024; ++i) {
                        load_to_lds16<NT>(kc + base + i * 1024, f_at, to + i * 1024);
                        load_to_lds16<NT>(vc + base + i * 1024, f_at, to + C::KB + i * 1024);
                    }
                } else {
                    load_to_lds16_at(f_half + base, to);
                }
                load_to_lds4_at(f_sc + (int64_t)r0 * C::SB, to + 2 * C::KB);
                return;
            }
            if constexpr (C::KB >= 1024) {
#pragma unroll
                for (int i = 0; i < C::KB / 1024; ++i) {
                    const int64_t off = base + (int64_t)min(f_row + i * f_rows_per, last) * C::RB + f_grp * 16;
                    load_to_lds16_at(kc + off, to + i * 1024);
                    load_to_lds16_at(vc + off, to + C::KB + i * 1024);
                }
            } else {
                load_to_lds16_at(f_half + base + (int64_t)(min(f_row2, last) - f_row2) * C::RB, to);
            }
            load_to_lds4_at(f_sc + (int64_t)r0 * C::SB + (min(sc_idx * 4, (last * C::SB) & ~3) - sc_idx * 4), to + 2 * C::KB);
        };
        // 16 of this wavefront's V rows, `half` * 16 .. of its stage, of which `valid` exist: the lane's quarter of one, and into
        // the V buffer as bf16, one 16-byte chunk after the other
        struct Codes { unsigned code[D / 32], byte; };
        auto read_codes = [&](int at, int half, int valid) __attribute__((always_inline)) {
            const unsigned char *from = stage0 + at + C::KB;
            const int r = half * 16 + d_row;
            Codes c;
            if constexpr (D == 128) {
                const uint4 c4 = *(const uint4 *)(from + r * C::RB + ((d_unit ^ swz4<D>(r)) * 16));
                c.code[0] = c4.x; c.code[1] = c4.y; c.code[2] = c4.z; c.code[3] = c4.w;
            } else {
                const uint2 c2 = *(const uint2 *)(from + r * C::RB + (((d_unit >> 1) ^ swz4<D>(r)) * 16) + (d_unit & 1) * 8);
                c.code[0] = c2.x; c.code[1] = c2.y;
            }
            unsigned byte = from[C::KB + 128 + r * C::SB + (D == 128 ? d_unit : d_unit >> 1)];
            if (valid < C::RW) {                                       // (uniform) beyond the last key: zeros, whatever stands there
                byte = r < valid ? byte : 127u;
#pragma unroll
                for (int i = 0; i < D / 32; ++i) c.code[i] = r < valid ? c.code[i] : 0u;
            }
            c.byte = byte;
            return c;
        };
        auto write_codes = [&](const Codes &c, int i, int vbuf) __attribute__((always_inline)) {
            *(uint4 *)(lds + C::RING + vbuf + (wave * 16 + d_row) * 64 + (D == 128 ? d_unit : d_unit >> 1) * C::VCOLS +
                       (((D == 128 ? i : (d_unit & 1) * 2 + i) ^ vswz(d_row)) * 16)) = fp4x8_to_bf16(c.code[i], fp4_scale(c.byte));
        };
        auto convert = [&](int at, int half, int vbuf, int valid) __attribute__((always_inline)) {
            const Codes c = read_codes(at, half, valid);
#pragma unroll
            for (int i = 0; i < D / 32; ++i) write_codes(c, i, vbuf);
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

        // The queries as they are: channels 64 st + 32 g + 8 i .. +7 (also the order of the contraction with the tree's keys).
        uint4 qr[C::ST][4];
        __syncthreads();                                               // (LDS is free: the piece before may have folded in it)
        {
            int node;
            const int64_t q_row = row_of(anew(ln), node);
#pragma unroll
            for (int st = 0; st < C::ST; ++st)
#pragma unroll
                for (int i = 0; i < 4; ++i) qr[st][i] = ((const uint4 *)(p.q + q_row + st * 64 + g * 32))[i];
        }
        Block<D> qs;
#pragma unroll
        for (int cb = 0; cb < C::CB; ++cb) qs.o[cb] = (f32x16_t){0};
        qs.start = (f32x16_t){0};
        qs.m_ref = -INFINITY;
        qs.l = 0.f;

        // ---- the tree's own keys: bf16 operands from registers, values through LDS ----
        for (int t = 0; t < n_tree; ++t) {
            const int key0 = (tile + t) * C::T, lane = anew(tid) & 63, g = lane >> 5, ln = lane & 31;
            // A tile of the tree's own rows: K operands, the 16 V rows that this wavefront brings (32 where they are its own), mask bits.
            struct Tree { uint4 k[C::U][C::ST][4], v[C::OWN ? 2 : 1][D / 32]; uint64_t bits[C::U]; } tr;
            {
                int node;
                row_of(ln, node);
                const uint64_t *mrow = p.mask_bits + (int64_t)node * p.mask_words;
#pragma unroll
                for (int u = 0; u < C::U; ++u) {
                    const int k0 = key0 + (kg * C::U + u) * 32;
                    tr.bits[u] = k0 < p.n ? mrow[k0 >> 6] >> (k0 & 63) : 0;
                    const uint16_t *kr = p.kt + tree + (int64_t)min(k0 + ln, p.n - 1) * D + g * 32;
#pragma unroll
                    for (int st = 0; st < C::ST; ++st)
#pragma unroll
                        for (int i = 0; i < 4; ++i) tr.k[u][st][i] = ((const uint4 *)(kr + st * 64))[i];
                }
#pragma unroll
                for (int hf = 0; hf < (C::OWN ? 2 : 1); ++hf)
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) {                     // 16 rows of D / 8 chunks
                        const int x = i * 64 + lane, key = key0 + (C::OWN ? wave * 32 + hf * 16 : wave * 16) + x / (D / 8);
                        tr.v[hf][i] = make_uint4(0, 0, 0, 0);
                        if (key < p.n) tr.v[hf][i] = *(const uint4 *)(p.vt + tree + (int64_t)key * D + x % (D / 8) * 8);
                    }
            }
            f32x16_t sacc[C::U];
            uint32_t bits[C::U];
#pragma unroll
            for (int u = 0; u < C::U; ++u) {
                bits[u] = (uint32_t)tr.bits[u];
                sacc[u] = (f32x16_t){0};
#pragma unroll
                for (int st = 0; st < C::ST; ++st)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        sacc[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, tr.k[u][st][i]), __builtin_bit_cast(bf16x8_t, qr[st][i]), sacc[u], 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 16; ++r) sacc[u][r] = fmaf(sacc[u][r], p.c, qs.start[0]);
            }
            // values: rows beyond the tree are zeros, and so is what is no number: a weight of zero would make it NaN for rows
            // that do not see it, so those are added below where they are seen
            bool odd = false;
            auto bring = [&](int hf) {
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    const int x = i * 64 + lane, r = x / (D / 8), ch = x % (D / 8);
                    unsigned wv[4] = {tr.v[hf][i].x, tr.v[hf][i].y, tr.v[hf][i].z, tr.v[hf][i].w};
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
                    bring(i);
                    read16(0, 0, vf);
                });
            } else {
                bring(0);
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
        // ---- the queries as terms ----
        {
#pragma unroll
            for (int st = 0; st < C::ST; ++st) {
                float x[32];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const unsigned wv[4] = {qr[st][i].x, qr[st][i].y, qr[st][i].z, qr[st][i].w};
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
        // (The first tiles are requested only now: the compiler's waits for queries and tree rows would be waits for them too, and at
        // the start all workgroups' requests queue for memory together.  One token for 32 sequences of 777 to 8191 keys 44.4 us
        // instead of 45.4, 60 nodes on 16 x 8 key heads of 512 to 4096 keys 61 instead of 62.6; for calls of one to eight tiles it makes
        // no difference: 8.5 and 8.6, 12.5 and 12.4, 14.9 and 14.8, 16.6 and 16.6, 18.5 and 18.6.)
#pragma unroll
        for (int x = 0; x < C::AHEAD; ++x)
            if (x < n_pre) issue(x, x * C::STAGE);
        // ---- the prefix ----
        // (a register of their own from here on: what stands in the way before and after may be kept in memory, not in the loops)
#pragma unroll
        for (int st = 0; st < C::ST; ++st) {
#pragma unroll
            for (int t = 0; t < 3; ++t) asm volatile("" : "+v"(qs.term[st][t]));
            asm volatile("" : "+v"(qs.scale[st]), "+v"(k_at[st]));
        }
        asm volatile("" : "+v"(ks_at), "+v"(v_lo), "+v"(v_hi));
        // which keys of a tile's blocks exist
        auto exist = [&](int valid, int u) {
            const int here = valid - (kg * C::U + u) * 32;
            return here >= 32 ? 0xffffffffu : here <= 0 ? 0u : (1u << here) - 1u;
        };
        auto read_k = [&](const unsigned char *stage, int u, u32x4_t (&k)[C::ST], int &ks) __attribute__((always_inline)) {
#pragma unroll
            for (int st = 0; st < C::ST; ++st) k[st] = *(const u32x4_t *)(stage + k_at[st] + u * K_BLOCK);
            if constexpr (D == 128) ks = *(const int *)(stage + ks_at + u * K_BLOCK) >> (8 * g);
            else ks = *(const uint16_t *)(stage + ks_at + u * K_BLOCK) >> (8 * g);
        };
        // step i of S^T = K Q^T: the small terms first
        auto qk = [&](int i, f32x16_t &s, const u32x4_t (&k)[C::ST], int ks) __attribute__((always_inline)) {
            const int st = i / 3;
            if (i % 3 == 0) s = mfma_fp4<2>(k[st], qs.term[st][2], i == 0 ? qs.start : s, ks, qs.scale[st], st);
            if (i % 3 == 1) s = mfma_fp4<1>(k[st], qs.term[st][1], s, ks, qs.scale[st], st);
            if (i % 3 == 2) s = mfma_fp4<0>(k[st], qs.term[st][0], s, ks, qs.scale[st], st);
        };
        constexpr int NQK = 3 * C::ST, NPV = 2 * C::CB;
        if constexpr (C::OWN) {
            int s = 0;                                                 // stage of tile x
            for (int x = 0; x < n_pre; ++x) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // (the stage of the tile before has been read)
                if (x + C::NS - 1 < n_pre) issue(x + C::NS - 1, (s == 0 ? C::NS - 1 : s - 1) * C::STAGE);
                wait_for(min(n_pre - 1 - x, C::NS - 1));
                f32x16_t sacc[1];
                u32x4_t k[C::ST];
                int ks;
                read_k(lds + s * C::STAGE, 0, k, ks);
#pragma unroll
                for (int i = 0; i < NQK; ++i) qk(i, sacc[0], k, ks);
                const int valid = L - (t0 + x) * C::T;                 // keys of this tile that exist
                const uint32_t bits[1] = {exist(valid, 0)};
                absorb<C>(sacc, qs, g, valid < C::T, bits, [&](int i, bf16x8_t (&vf)[C::CB]) __attribute__((always_inline)) {
                    convert(s * C::STAGE, i, 0, valid - wave * C::RW);
                    read16(0, 0, vf);
                });
                s = s + 1 == C::NS ? 0 : s + 1;
            }
        } else if (n_pre > 0) {
            // Blocks of 32 keys in a pipeline: while the weights of block j are made, the matrix unit computes the scores of block
            // j + 1 and adds block j - 1 to the output, instruction by instruction in turn.
            f32x16_t S[2];
            u32x4_t P[2][2], k[C::ST];
            int ks = 0;
            float alpha = 1.f;
            unsigned pending = 0;                                      // (uniform) the output is to be scaled by alpha once block j - 1 is in
            float limit = qs.m_ref == -INFINITY ? -INFINITY : SLACK;   // what a score may be before the reference moves (none seen yet: any does)
            auto scale_o = [&]() __attribute__((always_inline)) {
#pragma unroll
                for (int cb = 0; cb < C::CB; ++cb)
#pragma unroll
                    for (int r = 0; r < 16; ++r) qs.o[cb][r] *= alpha;
                pending = 0;
            };
            // Scores of the next block, mx their maximum: its missing keys, and the reference where they outgrow it.  One branch in
            // the common case, not taken.
            auto check = [&](f32x16_t &s, float mx, int valid, int u) __attribute__((always_inline)) {
                // (the other half's keys are looked at when any lane's ask for it)
                const unsigned long long over = __builtin_amdgcn_ballot_w64(mx > limit);
                if (__builtin_expect((unsigned)over | (unsigned)(over >> 32) | pending | (unsigned)(valid - C::T) >> 31, 0)) {
                    if (pending) scale_o();
                    if (valid < C::T) {
                        const uint32_t own = exist(valid, u) >> (4 * g);
                        mx = -INFINITY;
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const uint32_t seen = (uint32_t)__builtin_amdgcn_sbfe((int)own, 8 * (r / 4) + r % 4, 1);
                            s[r] = __uint_as_float((__float_as_uint(s[r]) & seen) | (0xff800000u & ~seen));
                            mx = fmaxf(mx, s[r]);
                        }
                    }
                    mx = half_max(mx);
                    const bool none = qs.m_ref == -INFINITY, grow = mx > limit;
                    if (__builtin_amdgcn_ballot_w64(grow) != 0) {
                        const float by = grow ? mx : 0.f;
                        alpha = grow && none ? 0.f : fast_exp2(-by);
                        pending = 1;
                        if (grow) {
                            qs.m_ref = (none ? 0.f : qs.m_ref) + mx;
                            limit = SLACK;
                        }
                        qs.l *= alpha;
                        const float start = qs.m_ref == -INFINITY ? 0.f : -qs.m_ref;
#pragma unroll
                        for (int r = 0; r < 16; ++r) qs.start[r] = start;
#pragma unroll
                        for (int r = 0; r < 16; ++r) s[r] -= by;
                    }
                }
            };
            // weights of `cur` into pn; scores of the next block into nxt; pp times 32 rows of V from `vrow` on into the output;
            // CONV: this wavefront's share of a tile's V converted on the way.  Returns the largest score of nxt.  Beside the last block the scores are of whatever K
            // the registers hold, unused; before the first one pp and the V rows are zeros.
            auto slot = [&](auto conv, f32x16_t &cur, f32x16_t &nxt, const u32x4_t (&pp)[2], u32x4_t (&pn)[2], int vbuf, int vrow, int cs, int cbuf,
                            int cvalid) __attribute__((always_inline)) {
                constexpr bool CONV = decltype(conv)::value;
                asm volatile("" : "+v"(qs.start));
                bf16x8_t vf[2][C::CB];
                read16(vbuf, vrow, vf[0]);
                Codes cv;
                if (CONV) cv = read_codes(cs, 0, cvalid);
                __builtin_amdgcn_sched_barrier(0);
                float sum = 0.f, mx = -INFINITY;
#pragma unroll
                for (int i = 0; i < NQK + NPV; ++i) {
                    if (i < NQK) qk(i, nxt, k, ks);
                    else {
                        const int y = i - NQK;
                        qs.o[y % C::CB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[y / C::CB][y % C::CB], __builtin_bit_cast(bf16x8_t, pp[y / C::CB]), qs.o[y % C::CB], 0, 0, 0);
                    }
#pragma unroll
                    for (int x = 0; x < 8; ++x)                        // vector work beside it
                        if ((D == 128 ? x : x < 6 ? x / 2 : x - 3) == i) weigh2(cur, 2 * x, sum, pn);
                    if (CONV) {
#pragma unroll
                        for (int x = 0; x < D / 32; ++x)
                            if ((D == 128 ? 8 : 5) + x == i) write_codes(cv, x, cbuf);
                    }
#pragma unroll
                    for (int x = 0; x < 8; ++x)                        // (the scores are whole some matrix instructions after their last)
                        if ((D == 128 ? 10 + x / 2 : 5 + x / 4) == i) {
                            mx = fmaxf(fmaxf(mx, nxt[2 * x]), nxt[2 * x + 1]);
                            asm volatile("" : "+v"(mx));
                        }
                    if (i == NQK - 1) read16(vbuf, vrow + 16, vf[1]);
                    __builtin_amdgcn_sched_barrier(0);
                }
                asm volatile("" : "+v"(nxt));                          // (stays in this block: the compiler would move it down to its use)
                qs.l += sum;
                return mx;
            };
            auto last_pv = [&](const u32x4_t (&pp)[2], int vbuf, int vrow) __attribute__((always_inline)) {
                if (pending) scale_o();
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    bf16x8_t vf[C::CB];
                    read16(vbuf, vrow + hf * 16, vf);
#pragma unroll
                    for (int cb = 0; cb < C::CB; ++cb)
                        qs.o[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[cb], __builtin_bit_cast(bf16x8_t, pp[hf]), qs.o[cb], 0, 0, 0);
                }
            };
            constexpr std::true_type YES;
            constexpr std::false_type NO;
            const int valid0 = min(L - t0 * C::T, n_pre * C::T);       // keys of the piece (the end of the last tile may be 2^31)
            // a tile's own slot is over: its V is converted everywhere, its stage free, and tile `need` has arrived everywhere
            constexpr int NEED = 3 - C::U;                             // tile x + NEED
            // Of two workgroups on a compute unit the older one would always go first, and the other be alone at the end, at half
            // the rate: they take turns of four tiles instead (which is which makes no difference to any result).
            // (A branch that the compiler does not see: it would copy accumulators along its two ways.)
            const int late = w >= p.single ? 4 : 0;
            auto turn = [&](int x, int at) __attribute__((always_inline)) {
                asm volatile("s_setprio 0\n\ts_bitcmp0_b32 %0, 2\n\ts_cbranch_scc1 .Lturn%=\n\ts_setprio 1\n.Lturn%=:" : : "s"(x ^ late) : "scc");
                if (__builtin_expect(x + C::NS < n_pre, 1)) {
                    MCSD_WAIT_VMCNT((C::NS - 1 - NEED) * C::LPT);
                    meet();
                    issue(x + C::NS, at);
                } else {
                    if (x + NEED < n_pre) wait_for(n_pre - 1 - x - NEED);
                    meet();
                }
            };
#pragma unroll
            for (int i = 0; i < C::VBUF / 4096; ++i) *(uint4 *)(lds + C::RING + C::VBUF + i * 4096 + anew(tid) * 16) = make_uint4(0, 0, 0, 0);
            P[1][0] = P[1][1] = (u32x4_t){0, 0, 0, 0};
            wait_for(min(n_pre, C::AHEAD) - 1 - (C::U == 1 && n_pre > 1));
            meet();
            read_k(lds, 0, k, ks);
#pragma unroll
            for (int i = 0; i < NQK; ++i) qk(i, S[0], k, ks);
            if constexpr (C::U == 2) read_k(lds, 1, k, ks);
            else read_k(lds + C::STAGE, 0, k, ks);
            {
                float mx = S[0][0];
#pragma unroll
                for (int r = 1; r < 16; ++r) mx = fmaxf(mx, S[0][r]);
                check(S[0], mx, valid0, 0);
            }
            int x = 0, at = 0, vb = 0;                                 // tile, its stage's offset, its V buffer's
            const auto after = [&](int at) { return at + C::STAGE == C::RING ? 0 : at + C::STAGE; };
            if constexpr (C::U == 2) {
                while (true) {
                    const int valid = valid0 - x * C::T, next = after(at);
                    float mx = slot(YES, S[0], S[1], P[1], P[0], C::VBUF - vb, 32, at, vb, valid - wave * C::RW);
                    turn(x, at);
                    read_k(lds + next, 0, k, ks);
                    check(S[1], mx, valid, 1);
                    mx = slot(NO, S[1], S[0], P[0], P[1], vb, 0, 0, 0, 0);
                    read_k(lds + next, 1, k, ks);
                    if (__builtin_expect(++x == n_pre, 0)) break;
                    check(S[0], mx, valid - C::T, 0);
                    at = next;
                    vb = C::VBUF - vb;
                }
                last_pv(P[1], vb, 32);
            } else {
                // (two tiles per turn of the loop, the way out at its end: elsewhere the compiler copies the output at every turn.
                // After an odd number of tiles comes one without keys, and the last look at the reference finds none.)
                float mx;
                auto one = [&](f32x16_t &cur, f32x16_t &nxt, const u32x4_t (&pp)[2], u32x4_t (&pn)[2]) __attribute__((always_inline)) {
                    const int next = after(at);
                    mx = slot(YES, cur, nxt, pp, pn, C::VBUF - vb, 0, at, vb, valid0 - x * C::T - wave * C::RW);
                    turn(x, at);
                    read_k(lds + after(next), 0, k, ks);
                    at = next;
                    vb = C::VBUF - vb;
                    ++x;
                };
                while (true) {
                    one(S[0], S[1], P[1], P[0]);
                    check(S[1], mx, valid0 - x * C::T, 0);
                    one(S[1], S[0], P[0], P[1]);
                    check(S[0], mx, valid0 - x * C::T, 0);
                    if (__builtin_expect(x >= n_pre, 0)) break;
                }
                last_pv(P[1], C::VBUF - vb, 0);
            }
            __builtin_amdgcn_s_setprio(0);
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
                    first_piece = (done - tile) / per;
                    n_pieces = (done - tile + all - 1) / per - first_piece + 1;
                }
                first_piece = uniform(first_piece);
                n_pieces = uniform(n_pieces);
                if (!prepared) {
#pragma unroll
                    for (int x = 0; x < C::PP; ++x) acc[x] = (f32x4_t){NAN, NAN, NAN, NAN};
                    write_out(1.f);                                        // never prepared: its counters mean nothing
                } else {
                    const int ln = anew(tid) & 31, g = (anew(tid) >> 5) & 1;
                    // slot of the piece: a workgroup leaves at most two, the first of them the end of a pair that began before
                    const auto slot_of = [&](int i) { return (int64_t)(2 * (first_piece + i) + (i == 0)); };
                    const int64_t slot = slot_of(number - first_piece);
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
                        // NF pieces at a time, everything of them requested at once; beyond the last one loads give zero.  As many as the
                        // registers hold (64 rows: with 4 at a time 44 nodes on 32 heads of 1024 keys, five pieces, take 19.3 us, with 5
                        // 18.5, with 6, which do not fit beside the rest, 21.1).
                        constexpr int NF = C::PP >= 16 ? 2 : C::PP == 8 ? 5 : 8;
                        const auto off_of = [&](int i) { return (2 * i + (i == 0)) * ROWS; };
                        const auto rm = __builtin_amdgcn_make_buffer_rsrc((void *)(p.part_m + (int64_t)2 * first_piece * ROWS), 0, 2 * n_pieces * ROWS * 4, 0x00027000);
                        const auto rl = __builtin_amdgcn_make_buffer_rsrc((void *)(p.part_l + (int64_t)2 * first_piece * ROWS), 0, 2 * n_pieces * ROWS * 4, 0x00027000);
                        const auto ro = __builtin_amdgcn_make_buffer_rsrc((void *)(p.part_o + (int64_t)2 * first_piece * ROWS * D), 0, 2 * n_pieces * ROWS * D * 4, 0x00027000);
                        float M = -INFINITY, den = 0.f;
#pragma unroll
                        for (int x = 0; x < C::PP; ++x) acc[x] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
                        for (int i0 = 0; i0 < n_pieces; i0 += NF) {
                            float m[NF], lp[NF];
                            f32x4_t v[NF][C::PP];
#pragma unroll
                            for (int i = 0; i < NF; ++i) {
                                m[i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rm, (off_of(i0 + i) + qb * 32 + ln) * 4, 0, AGENT));
                                lp[i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rl, (off_of(i0 + i) + qb * 32 + ln) * 4, 0, AGENT));
#pragma unroll
                                for (int x = 0; x < C::PP; ++x)
                                    v[i][x] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(ro, off_of(i0 + i) * D * 4 + (((qb * C::CB * 4 + kg * C::PP + x) * 2 + g) * 32 + ln) * 16, 0, AGENT));
                            }
                            __builtin_amdgcn_sched_barrier(0);
                            float Mn = M;
#pragma unroll
                            for (int i = 0; i < NF; ++i) Mn = fmaxf(Mn, i0 + i < n_pieces ? m[i] : -INFINITY);
                            const float Mf = Mn == -INFINITY ? 0.f : Mn, a = fast_exp2(M - Mf);
                            M = Mn;
                            den *= a;
#pragma unroll
                            for (int x = 0; x < C::PP; ++x) acc[x] *= a;
#pragma unroll
                            for (int i = 0; i < NF; ++i) {
                                const float wgt = i0 + i < n_pieces ? fast_exp2(m[i] - Mf) : 0.f;
                                den = fmaf(wgt, lp[i], den);
#pragma unroll
                                for (int x = 0; x < C::PP; ++x) acc[x] += wgt * v[i][x];
                            }
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
        if (rounds) {
            if (++round == rounds) break;
            const int at = round * p.workgroups + (round & 1 ? p.workgroups - 1 - w : w);
            if (at >= pairs) break;
            const int l = uniform(small_div(at, p.units));
            b = uniform(s_order[l]);
            unit = at - l * p.units;
            left = tiles_of(uniform(s_len[b]));
            continue;
        }
        if (++unit == p.units) {
            unit = 0;
            if (++b == p.B) break;
        }
    }
}

// ---------------------------------------------------------------------------------------------------- host
struct Fp4Plan {
    int QBP, chunks, units, workgroups, single;
    size_t bytes;                    // workspace
};

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// False where the work has more tiles than the kernel's numbers hold.
bool make_plan(int B, int H_kv, int grp, int d, int n_rows, int n, int max_prefix, Fp4Plan &pl)
{
    const int64_t rows = (int64_t)grp * n_rows;
    // As few blocks of 32 rows as hold them.  One token of 4 heads on 32 x 8 key heads of 777 to 8191 keys: one block 44.5 us, two 55; 44
    // rows on 32 heads of 1024 keys: two 18.5, four 23.0, on 8 x 32 of 4096 52 and 69; 240 rows on 16 x 8 key heads of 512 to 4096
    // keys: four 61, two (twice the chunks) 72, of 2048 keys each 54.3 and 53.7; 120 rows on 8 x 32 heads of 16384 keys: four 264,
    // two 321.
    pl.QBP = rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
    const int64_t chunks = (rows + 32 * pl.QBP - 1) / (32 * pl.QBP), units = chunks * H_kv;
    const int T = pl.QBP == 1 ? 128 : 64;
    const int64_t tiles = (n + T - 1) / T + ((int64_t)max_prefix + T - 1) / T;
    if (rows > 0x3fffffff || units * B > 0x3fffffff || units * B * tiles > 0x3fffffff) return false;
    pl.chunks = (int)chunks;
    pl.units = (int)units;
    const int min_tiles = pl.QBP == 1 ? Cfg<128, 1>::MIN_TILES : pl.QBP == 2 ? Cfg<128, 2>::MIN_TILES : Cfg<128, 4>::MIN_TILES;
    pl.single = mcsd_compute_units();
    int most = 2 * pl.single;
    if (most > MAX_PIECES) most = MAX_PIECES;
    const int64_t pairs = units * B, pieces = pairs * ((tiles + min_tiles - 1) / min_tiles);
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
    // (only with 128 rows to a chunk can there be more than one)
    auto kernel = pl.QBP == 1 ? tree_attn_fp4_kernel<D, 1, true> : pl.QBP == 2 ? tree_attn_fp4_kernel<D, 2, true>
                  : pl.chunks == 1 ? tree_attn_fp4_kernel<D, 4, true> : tree_attn_fp4_kernel<D, 4, false>;
    mcsd_launch(MCSD_KERNEL_ATTN_SWEEP, kernel, dim3(pl.workgroups), dim3(256), st, p);
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
    p.by_chunks = row_div_of((uint32_t)pl.chunks); p.by_nrows = row_div_of((uint32_t)(n - row_begin));
    p.workgroups = pl.workgroups; p.single = pl.single;
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
