// From logits to the probability rows that the verification takes, and tokens drawn from them (definition in mcsd.h).
//
// A workgroup has a row and reads it once per pass, from memory the first time and from the L2 after it.  The tokens of a row are ordered
// by logit, largest first, then by index; top-k, top-p and min-p each keep a beginning of that order, and the shortest counts.  Where it
// ends is found without a sort.  For a top-k of up to half the threads: the k-th largest of the threads' own maxima is no more than the
// k-th largest logit, so the few tokens from there on are listed and ranked against each other, and the rest of the call is about the
// list.  Otherwise: two places per thread for ranges of logits, the tokens of the one place where the count or the sum reaches its goal
// listed and ranked; more of them than the list holds are cut into as many ranges again, of logit and index as one number.
//
// A weight is 2^((x - max) log2(e) / T) as a whole number of 2^-45: the sums are exact whatever their order (so atomics may add them),
// a border of top-p and a draw depend on nothing but the weights, and 2^18 of them stay below 2^64.  It is computed in binary64,
// so a border falls where 64 bits have it.  Probabilities are computed in fp32 pairs, or of a binary64 exponent.
//
// What bounds it, at 32000 logits a row: few rows, the passes and meetings of one workgroup one after the other (45 rows of bf16, top-k 50
// with top-p and min-p: 21 us; 64 rows of fp32 with top-p and four distinct draws: 39 us; 32 rows of 131077, mixed: 116 us, the vector
// instructions of the rows with a top-p alone, 7 in 10 cycles); many rows, the exponentials, made once for the sum and once for the row
// (2816 rows of bf16: 166 us for 541 MB, 3.3 TB/s; kept between the two they would need the LDS that the second workgroup has).
// Rows in LDS between the passes took 2 to 20 us longer, and so did requests two more turns ahead.
#include <math.h>

#include "mcsd_internal.h"
#include "wave_ops.h"

namespace {

typedef unsigned long long u64;

struct SampleParams {
    const void *x;
    int64_t x_batch, x_row;              // strides in elements
    int32_t W, V;
    mcsd_sampler_t s;
    float *probs;
    int64_t p_batch;
    int32_t n_draw, distinct;
    const float *u;
    int32_t *tokens;
    int64_t t_batch;
};

constexpr int MAX_DRAW = 64;
constexpr int ONE = 45;                  // a weight of 1 is 2^45
constexpr int FEW = 41;                  // distinct draws: below a sum of 2^41 the weights are made anew around the largest that is left
constexpr int MAX_SEGMENTS = MCSD_MAX_VOCAB / 512;
constexpr int HELD = 4;                  // kept tokens in the order of indices per thread

struct Ranked { u64 place, weight; };
template <int THREADS>
struct Shared {
    union {
        struct {
            u64 hist[2 * THREADS];
            Ranked list[THREADS];
        };
        uint2 roll[HELD * THREADS];      // logit and index
    };
    double table[64];                    // 2^(j / 64)
    u64 segment[MAX_SEGMENTS];           // sums of 512 tokens
    u64 wave[THREADS / 64];
    int32_t count[MAX_SEGMENTS];         // kept tokens of 512, then of all before them
    u64 above, sum, cut;
    int32_t bin, listed, kept, winner;
    int32_t drawn[MAX_DRAW];
};

__device__ __forceinline__ unsigned ordered(float x)
{
    const unsigned b = __float_as_uint(x + 0.f);                           // (-0 is 0)
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float of_ordered(unsigned k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu)); }
// Place in the order, the first has the largest.
__device__ __forceinline__ u64 place_of(float x, int i) { return (u64)ordered(x) << 18 | (unsigned)(0x3ffff - i); }

__device__ __forceinline__ int index_of(u64 place) { return 0x3ffff - (int)(place & 0x3ffff); }

// 2^(j / 64), rounded to nearest.
__device__ const double powers_of_two[64] = {
    0x1.0000000000000p+0, 0x1.02c9a3e778061p+0, 0x1.059b0d3158574p+0, 0x1.0874518759bc8p+0,
    0x1.0b5586cf9890fp+0, 0x1.0e3ec32d3d1a2p+0, 0x1.11301d0125b51p+0, 0x1.1429aaea92de0p+0,
    0x1.172b83c7d517bp+0, 0x1.1a35beb6fcb75p+0, 0x1.1d4873168b9aap+0, 0x1.2063b88628cd6p+0,
    0x1.2387a6e756238p+0, 0x1.26b4565e27cddp+0, 0x1.29e9df51fdee1p+0, 0x1.2d285a6e4030bp+0,
    0x1.306fe0a31b715p+0, 0x1.33c08b26416ffp+0, 0x1.371a7373aa9cbp+0, 0x1.3a7db34e59ff7p+0,
    0x1.3dea64c123422p+0, 0x1.4160a21f72e2ap+0, 0x1.44e086061892dp+0, 0x1.486a2b5c13cd0p+0,
    0x1.4bfdad5362a27p+0, 0x1.4f9b2769d2ca7p+0, 0x1.5342b569d4f82p+0, 0x1.56f4736b527dap+0,
    0x1.5ab07dd485429p+0, 0x1.5e76f15ad2148p+0, 0x1.6247eb03a5585p+0, 0x1.6623882552225p+0,
    0x1.6a09e667f3bcdp+0, 0x1.6dfb23c651a2fp+0, 0x1.71f75e8ec5f74p+0, 0x1.75feb564267c9p+0,
    0x1.7a11473eb0187p+0, 0x1.7e2f336cf4e62p+0, 0x1.82589994cce13p+0, 0x1.868d99b4492edp+0,
    0x1.8ace5422aa0dbp+0, 0x1.8f1ae99157736p+0, 0x1.93737b0cdc5e5p+0, 0x1.97d829fde4e50p+0,
    0x1.9c49182a3f090p+0, 0x1.a0c667b5de565p+0, 0x1.a5503b23e255dp+0, 0x1.a9e6b5579fdbfp+0,
    0x1.ae89f995ad3adp+0, 0x1.b33a2b84f15fbp+0, 0x1.b7f76f2fb5e47p+0, 0x1.bcc1e904bc1d2p+0,
    0x1.c199bdd85529cp+0, 0x1.c67f12e57d14bp+0, 0x1.cb720dcef9069p+0, 0x1.d072d4a07897cp+0,
    0x1.d5818dcfba487p+0, 0x1.da9e603db3285p+0, 0x1.dfc97337b9b5fp+0, 0x1.e502ee78b3ff6p+0,
    0x1.ea4afa2a490dap+0, 0x1.efa1bee615a27p+0, 0x1.f50765b6e4540p+0, 0x1.fa7c1819e90d8p+0
};

// 2^y for y <= 0 as 2^(k / 64) 2^r with |r| <= 1/128: the first six terms of 2^r leave 2^-54 of it, in all it is off by at most 2^-51.5.
// (A polynomial over [-1/2, 1/2] needs ten products where this one has five and a number from LDS: 32 rows of
// 131077, mixed, 135 us instead of 127, 64 rows with top-p and four distinct draws 45.5 instead of 44.1.)
__device__ __forceinline__ u64 weight_of(double y, const double *table)
{
    y = fmax(y, -60.0);                                                    // (zero, without a branch)
    const double shifted = y + 0x1.8p46, r = y - (shifted - 0x1.8p46);      // (the multiple of 1/64 next to y: without the conversions, a quarter as fast)
    const int k = (int)__builtin_bit_cast(u64, shifted);
    double p = 0x1.5d87fe78a6731p-10;
    p = fma(p, r, 0x1.3b2ab6fba4e77p-7);
    p = fma(p, r, 0x1.c6b08d704a0c0p-5);
    p = fma(p, r, 0x1.ebfbdff82c58fp-3);
    p = fma(p, r, 0x1.62e42fefa39efp-1);
    p = fma(p, r, 1.0);
    // (times 2^(k / 64 + 45), and 2^52 added: the sum's last place is 1)
    const u64 power = __builtin_bit_cast(u64, table[k & 63]) + ((u64)(unsigned)((k >> 6) + ONE) << 52);
    const double s = fma(p, __builtin_bit_cast(double, power), 0x1p52);
    return __builtin_bit_cast(u64, s) & 0xfffffffffffffull;
}

// A share in parts of 2^-64, kept within [0, 1) (NaN: 0): its product with a sum of weights is one of whole numbers.  (The sum of many
// weights has more than the 53 bits of a binary64; a product rounded to those can be hundreds of the weights' last places off.  Shares below
// 2^-40 lose their last bits here, half a last place of the product at most.)
__device__ __forceinline__ u64 parts_of(float share) { return (u64)((double)fminf(fmaxf(share, 0.f), 0x1.fffffep-1f) * 0x1p64); }

// From other lanes of the wavefront, zero where there is none (see wave_ops.h for the steps).
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 from_lane64(u64 v)
{
    return (u64)(unsigned)from_lane<CTRL, ROWS>((int)(v >> 32)) << 32 | (unsigned)from_lane<CTRL, ROWS>((int)v);
}
__device__ __forceinline__ u64 wave_scan(u64 v)                            // inclusive
{
    v += from_lane64<0x111, 0xf>(v);
    v += from_lane64<0x112, 0xf>(v);
    v += from_lane64<0x114, 0xf>(v);
    v += from_lane64<0x118, 0xf>(v);
    v += from_lane64<0x142, 0xa>(v);
    v += from_lane64<0x143, 0xc>(v);
    return v;
}
__device__ __forceinline__ u64 lane_of(u64 v, int lane)
{
    return (u64)(unsigned)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)v, lane);
}
__device__ __forceinline__ u64 wave_sum(u64 v) { return lane_of(wave_scan(v), 63); }
__device__ __forceinline__ u64 wave_largest(u64 v)
{
#define MCSD_STEP(CTRL, ROWS) { const u64 u = from_lane64<CTRL, ROWS>(v); v = u > v ? u : v; }
    MCSD_STEP(0x111, 0xf) MCSD_STEP(0x112, 0xf) MCSD_STEP(0x114, 0xf) MCSD_STEP(0x118, 0xf) MCSD_STEP(0x142, 0xa) MCSD_STEP(0x143, 0xc)
#undef MCSD_STEP
    return lane_of(v, 63);
}

// Eight logits from index i on; behind the row's end minus infinity.  (Rows begin anywhere.)
template <bool F32>
struct __attribute__((aligned(16))) Eight {
    unsigned w[F32 ? 8 : 4];
    __device__ __forceinline__ void load(const void *row, int i, int V)
    {
        struct __attribute__((packed, aligned(F32 ? 4 : 2))) Words { unsigned w[F32 ? 8 : 4]; };
        if (i + 8 <= V) {
            const Words a = *(const Words *)((const char *)row + (int64_t)i * (F32 ? 4 : 2));
#pragma unroll
            for (int k = 0; k < (F32 ? 8 : 4); ++k) w[k] = a.w[k];
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if constexpr (F32) {
                    w[k] = i + k < V ? ((const unsigned *)row)[i + k] : 0xff800000u;
                } else {
                    const unsigned v = i + k < V ? ((const uint16_t *)row)[i + k] : 0xff80u;
                    w[k / 2] = k & 1 ? w[k / 2] | v << 16 : v;
                }
            }
        }
    }
    __device__ __forceinline__ float operator[](int k) const
    {
        if constexpr (F32) return __uint_as_float(w[k]);
        else return __uint_as_float(k & 1 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16);
    }
    __device__ __forceinline__ void drop(int k)                            // minus infinity
    {
        if constexpr (F32) w[k] = 0xff800000u;
        else w[k / 2] = k & 1 ? (w[k / 2] & 0xffffu) | 0xff800000u : (w[k / 2] & 0xffff0000u) | 0xff80u;
    }
};

template <bool F32, int THREADS>
__global__ __launch_bounds__(THREADS, 4) void sample_rows_kernel(const SampleParams p)
{
    constexpr int WAVES = THREADS / 64, TURN = 8 * THREADS, BINS = 2 * THREADS, LIST = THREADS, ROLL = HELD * THREADS;
    __shared__ Shared<THREADS> sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), r = blockIdx.x, b = blockIdx.y;
    const int V = p.V, turns = (V + TURN - 1) / TURN;
    const void *row = (const char *)p.x + ((int64_t)b * p.x_batch + (int64_t)r * p.x_row) * (F32 ? 4 : 2);
    // f(turn, first index, eight logits), those from memory requested some turns ahead.  (In a loop, as every pass has its own code: of a
    // row in registers with the code of every token in it, 7 passes over 32 a thread, fetching the code took longer than all else.)
    constexpr int AHEAD = 2;
    auto each = [&](auto f) __attribute__((always_inline)) {
        Eight<F32> x[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) x[k].load(row, (k * THREADS + tid) * 8, V);
#pragma unroll 1
        for (int t = 0; t < turns; ++t) {
            const Eight<F32> now = x[0];
#pragma unroll
            for (int k = 0; k + 1 < AHEAD; ++k) x[k] = x[k + 1];
            if (t + AHEAD < turns) x[AHEAD - 1].load(row, ((t + AHEAD) * THREADS + tid) * 8, V);
            f(t, (t * THREADS + tid) * 8, now);
        }
    };
    // over the workgroup: sums, maxima; all threads get them
    auto block_sum = [&](u64 v) {
        v = wave_sum(v);
        __syncthreads();
        if (lane == 0) sh.wave[wave] = v;
        __syncthreads();
        return wave_sum(lane < WAVES ? sh.wave[lane] : 0);
    };
    auto block_max = [&](u64 v) {
        v = wave_largest(v);
        __syncthreads();
        if (lane == 0) sh.wave[wave] = v;
        __syncthreads();
        return wave_largest(lane < WAVES ? sh.wave[lane] : 0);
    };
    // sum of those before this thread, and of all
    auto block_scan = [&](u64 v, u64 &all) {
        const u64 in = wave_scan(v);
        __syncthreads();
        if (lane == 63) sh.wave[wave] = in;
        __syncthreads();
        const u64 waves = wave_scan(lane < WAVES ? sh.wave[lane] : 0);
        all = lane_of(waves, WAVES - 1);
        return in - v + (wave ? lane_of(waves, wave - 1) : 0);
    };
    float *probs = p.probs ? p.probs + (int64_t)b * p.p_batch + (int64_t)r * V : nullptr;
    int32_t *tokens = p.tokens ? p.tokens + (int64_t)b * p.t_batch + (int64_t)r * p.n_draw : nullptr;
    const float *us = p.u ? p.u + ((int64_t)b * p.W + r) * p.n_draw : nullptr;
    auto write8 = [&](int i, const float (&y)[8]) __attribute__((always_inline)) {
        struct __attribute__((packed, aligned(4))) Four { float v[4]; };
        if (i + 8 <= V) {
            *(Four *)(probs + i) = Four{{y[0], y[1], y[2], y[3]}};
            *(Four *)(probs + i + 4) = Four{{y[4], y[5], y[6], y[7]}};
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (i + k < V) probs[i + k] = y[k];
        }
    };

    if (tid < 64) sh.table[tid] = powers_of_two[tid];
    // ---- maximum (NaN where a logit is), and whether the row is a distribution
    const float T = p.s.temperature ? p.s.temperature[b] : 1.f, top_p = p.s.top_p ? p.s.top_p[b] : 1.f, min_p = p.s.min_p ? p.s.min_p[b] : 0.f;
    const int top_k = p.s.top_k ? p.s.top_k[b] : 0;
    float own_max = -INFINITY;                                             // of the thread's logits
    each([&](int, int, const Eight<F32> &x) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < 8; ++k) own_max = __builtin_elementwise_maximum(own_max, x[k]);
    });
    const bool bad = __syncthreads_or(!(own_max < INFINITY)) || !(T >= 0.f) || top_p != top_p || min_p != min_p;
    const float mx = of_ordered((unsigned)block_max(ordered(own_max)));
    if (bad || mx == -INFINITY) {                                          // no distribution: NaN, or nothing to choose from: zeros
        const float v = bad ? NAN : 0.f;
        const float y[8] = {v, v, v, v, v, v, v, v};
        if (probs)
            for (int t = 0; t < turns; ++t)
                if ((t * THREADS + tid) * 8 < V) write8((t * THREADS + tid) * 8, y);
        if (tid < p.n_draw) tokens[tid] = -1;
        return;
    }

    // ---- the cut: a token is kept if its logit is above it, or at it and its index not behind
    const double c = T > 0.f ? 1.4426950408889634074 / (double)T : 0.0, mxd = (double)mx;
    const double min_y = min_p > 0.f ? fmin(log2((double)min_p), 0.0) : -INFINITY;
    double top = mxd;                                                      // what weights are relative to
    constexpr float LOWEST = -3.402823466e38f;
    float cut_x = LOWEST;                                                  // of everything but minus infinity
    int cut_i = V;
    float below = -INFINITY;                                               // the next number below cut_x
    auto exponent = [&](float x) { return ((double)x - mxd) * c; };
    auto weight = [&](float x) { return weight_of(((double)x - top) * c, sh.table); };
    auto kept = [&](float x, int i) __attribute__((always_inline)) { return x > cut_x || (x == cut_x && i <= cut_i); };
    auto cut_at = [&](float x, int i) {
        cut_x = x;
        cut_i = i;
        below = x == 0.f ? -0x1p-149f : of_ordered(ordered(x) - 1);
    };
    // Of the eight tokens from i on those are kept whose logit exceeds the number returned: which index of a tie at the cut is kept is the
    // same for all eight, but for the eight it falls into (there it is dropped beforehand).  So every pass has one compare for a token, not
    // three (64 rows with top-p and four distinct draws 43 us, 39 so; 32 rows of 131077, mixed, 125 and 116).
    auto sift = [&](Eight<F32> &x, int i) __attribute__((always_inline)) {
        if (i <= cut_i && i + 7 > cut_i) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (i + k > cut_i && x[k] == cut_x) x.drop(k);
        }
        return i <= cut_i ? below : cut_x;
    };
    // each, sifted, but for wavefronts without a token from this logit on
    auto max8 = [](const Eight<F32> &x) { return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7]))); };
    auto each_kept = [&](auto f, float from) __attribute__((always_inline)) {
        each([&](int t, int i, const Eight<F32> &x) __attribute__((always_inline)) {
            if (__builtin_amdgcn_ballot_w64(max8(x) >= from) != 0) {
                Eight<F32> y = x;
                const float limit = sift(y, i);
                f(t, i, y, limit);
            }
        });
    };
    // The token at this place is the last that is kept; whole: all with its logit are, but for those that an earlier cut left out (a search
    // sees the kept tokens only, so it cannot tell).
    auto set_cut = [&](u64 place, bool whole) {
        const float x = of_ordered((unsigned)(place >> 18));
        cut_at(x, !whole ? index_of(place) : x == cut_x ? cut_i : V);
    };
    auto clear = [&]() {
        sh.hist[tid] = 0;
        sh.hist[tid + THREADS] = 0;
        if (tid == 0) sh.listed = 0;
        __syncthreads();
    };
    // Where the sum over the places reaches goal(sum of all): sh.bin, and sh.above up to there; above: what is before the first of them.
    u64 target = 0;
    auto choose = [&](u64 above, auto goal) {
        __syncthreads();
        const u64 h0 = sh.hist[2 * tid], h1 = sh.hist[2 * tid + 1];
        u64 all;
        const u64 before = above + block_scan(h0 + h1, all);
        target = goal(above + all);
        if (before < target && before + h0 >= target) { sh.bin = 2 * tid; sh.above = before; }
        if (before + h0 < target && before + h0 + h1 >= target) { sh.bin = 2 * tid + 1; sh.above = before + h0; }
        __syncthreads();
    };
    // The wanted ones of eight tokens behind the list: one place asked for per wavefront.
    auto append = [&](const Eight<F32> &x, int i, unsigned wanted) __attribute__((always_inline)) {
        if (__builtin_amdgcn_ballot_w64(wanted != 0) == 0) return;
        const int here = __builtin_popcount(wanted), in = ::wave_scan(here), all = ::wave_last(in);
        int n = 0;
        if (lane == 63) n = atomicAdd(&sh.listed, all);
        n = ::wave_last(n) + in - here;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (wanted >> k & 1) {
                if (n < LIST) sh.list[n].place = place_of(x[k], i + k);
                ++n;
            }
    };
    // Every thread has one of the n listed tokens: its place (0: none), its measure, and that of all tokens before it in the order.
    u64 mine = 0, own = 0, before_me = 0;
    int rank_me = 0;
    auto token_x = [&]() { return of_ordered((unsigned)(mine >> 18)); };
    auto rank = [&](int n, u64 above, auto measure) {
        mine = tid < n ? sh.list[tid].place : 0;
        own = tid < n ? measure(token_x()) : 0;
        if (tid < LIST) sh.list[tid] = Ranked{mine, own};                  // (behind the last: nothing, so that the loop below needs no end)
        __syncthreads();
        before_me = above;
        rank_me = 0;
        if (wave * 64 < n)
            for (int o = 0; o < n; o += 8) {
                Ranked r[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) r[k] = sh.list[o + k];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    rank_me += r[k].place > mine;
                    before_me += r[k].place > mine ? r[k].weight : 0;
                }
            }
    };
    // The place at which the sum of measure(logit) over the tokens from the first on reaches goal(sum of all) >= 1 becomes the cut; returns
    // the sum up to and with it.
    auto find = [&](bool by_weight, auto goal) -> u64 {
        auto measure = [&](float x) __attribute__((always_inline)) { return by_weight ? weight(x) : (u64)1; };
        const float range = 31.9f * T, scale = range < INFINITY ? (BINS - 0.5f) / range : 0.f;      // (weights are zero beyond it)
        auto bin_of = [&](float x) { return scale < INFINITY ? (int)fminf((mx - x) * scale, (float)(BINS - 1)) : 0; };
        clear();
        each_kept([&](int, int i, const Eight<F32> &x, float limit) __attribute__((always_inline)) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                u64 m = measure(x[k]);
                asm volatile("" : "+v"(m));                                // (no branch around it: 127 -> 125 us for the mixed rows of 131077)
                m = x[k] > limit ? m : 0;
                if (m) atomicAdd(&sh.hist[bin_of(x[k])], m);
                if (k % 2) __builtin_amdgcn_sched_barrier(0);              // (not all eight at once: registers)
            }
        }, cut_x);
        choose(0, goal);
        const int bin = sh.bin;
        u64 above = sh.above, lo = 0, hi = ~0ull;
        each_kept([&](int, int i, const Eight<F32> &x, float limit) __attribute__((always_inline)) {
            unsigned wanted = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) wanted |= bin_of(x[k]) == bin && x[k] > limit ? 1u << k : 0;
            append(x, i, wanted);
        }, cut_x);
        __syncthreads();
        bool parted = false;
        if (sh.listed > LIST) {
            // from here on by place: the range lo .. hi is cut until its tokens fit the list
            parted = true;
            lo = ~0ull;
            hi = 0;
            each([&](int, int i, const Eight<F32> &x) __attribute__((always_inline)) {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (bin_of(x[k]) == bin && kept(x[k], i + k)) {
                        const u64 at = place_of(x[k], i + k);
                        lo = at < lo ? at : lo;
                        hi = at > hi ? at : hi;
                    }
            });
            hi = block_max(hi);
            lo = ~block_max(~lo);
            while (sh.listed > LIST) {
                int shift = 0;
                while ((hi - lo) >> shift >= BINS) ++shift;
                __syncthreads();
                clear();
                each([&](int, int i, const Eight<F32> &x) __attribute__((always_inline)) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const u64 at = place_of(x[k], i + k);
                        if (at >= lo && at <= hi) {
                            const u64 m = measure(x[k]);
                            if (m) atomicAdd(&sh.hist[(hi - at) >> shift], m);
                        }
                    }
                });
                choose(above, [&](u64) { return target; });
                above = sh.above;
                const u64 end = hi - ((u64)sh.bin << shift), begin = end - ((1ull << shift) - 1);
                hi = end;
                lo = begin > lo && begin <= end ? begin : lo;
                each([&](int, int i, const Eight<F32> &x) __attribute__((always_inline)) {
                    unsigned wanted = 0;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const u64 at = place_of(x[k], i + k);
                        wanted |= at >= lo && at <= hi ? 1u << k : 0;
                    }
                    append(x, i, wanted);
                });
                __syncthreads();
            }
        }
        rank(sh.listed, above, measure);
        if (mine && before_me < target && before_me + own >= target) { sh.cut = mine; sh.sum = before_me + own; }
        __syncthreads();
        const u64 place = sh.cut;
        set_cut(place, !__syncthreads_or(parted || (mine && mine >> 18 == place >> 18 && mine < place)));
        return sh.sum;
    };
    auto share = [&](u64 all) {                                            // of the sum, to top-p: rounded up, 1 at least
        const u64 goal = (u64)(((unsigned __int128)parts_of(top_p) * all + ~0ull) >> 64);
        return goal ? goal : (u64)1;
    };

    // Of the n listed tokens, all from the first on down to somewhere behind what is kept: what top-k, top-p and min-p leave.
    u64 sum = 0;
    bool exact = false;                                                    // whether that is the sum of what is kept
    auto settle = [&](int n, int k) {
        rank(n, 0, weight);
        if (mine && rank_me == min(k, n) - 1) sh.sum = before_me + own;
        __syncthreads();
        const u64 goal = share(sh.sum);
        const bool in = mine && rank_me < k && (top_p >= 1.f || before_me < goal) && exponent(token_x()) >= min_y;
        const int m = __syncthreads_count(in);
        if (in && rank_me == m - 1) { sh.cut = mine; sh.sum = before_me + own; }
        __syncthreads();
        const u64 place = sh.cut;
        sum = sh.sum;
        exact = true;
        set_cut(place, !__syncthreads_or(mine && mine >> 18 == place >> 18 && mine < place));
    };
    if (T == 0.f || top_k == 1) {                                          // the largest alone
        int first = V;
        each_kept([&](int, int i, const Eight<F32> &x, float limit) __attribute__((always_inline)) {
#pragma unroll
            for (int k = 7; k >= 0; --k) first = x[k] == mx && i + k < first ? i + k : first;
        }, mx);
        first = (int)~block_max(~(u64)(unsigned)first);
        set_cut(place_of(mx, first), false);
        sum = 1ull << ONE;
        exact = true;
    } else {
        const bool some = top_k > 0 && top_k < V;
        if (some && top_k <= THREADS / 2) {
            // the threads' maxima by ranges of their own, the range in which the k-th of them is, and all tokens down to its end
            const float low = of_ordered(~(unsigned)block_max(own_max > -INFINITY ? ~ordered(own_max) : 0u));
            const float range = mx - low, scale = range > 0.f && range < INFINITY ? (BINS - 0.5f) / range : 0.f;
            auto bin_of = [&](float x) { return scale < INFINITY ? (int)fminf((mx - x) * scale, (float)(BINS - 1)) : 0; };
            clear();
            if (own_max > -INFINITY) atomicAdd(&sh.hist[bin_of(own_max)], (u64)1);
            choose(0, [&](u64 all) { return all < (u64)top_k ? all : (u64)top_k; });
            const int bin = target < (u64)top_k ? BINS : sh.bin;           // (fewer threads with tokens than top_k: all tokens)
            auto wanted = [&](float x) { return x >= cut_x && (x >= low ? bin_of(x) <= bin : bin == BINS); };
            each([&](int, int i, const Eight<F32> &x) __attribute__((always_inline)) {
                if (__builtin_amdgcn_ballot_w64(wanted(max8(x))) == 0) return;
                unsigned these = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) these |= wanted(x[k]) ? 1u << k : 0;
                append(x, i, these);
            });
            __syncthreads();
            const int n = sh.listed;
            __syncthreads();
            if (n <= LIST) settle(n, top_k);
        }
        if (!exact) {
            for (int by_weight = !some; by_weight <= (top_p < 1.f); ++by_weight)      // (one after the other: one piece of code)
                sum = find(by_weight, [&](u64 all) { return by_weight ? share(all) : all < (u64)top_k ? all : (u64)top_k; });
            exact = top_p < 1.f;
            if (min_p > 0.f) {                                             // the lowest logit that it keeps, between minus infinity and mx
                unsigned out = ordered(-INFINITY), in = ordered(mx);
                while (in - out > 1) {
                    const unsigned mid = out + (in - out) / 2;
                    if (exponent(of_ordered(mid)) >= min_y) in = mid;
                    else out = mid;
                }
                if (of_ordered(in) > cut_x) {
                    cut_at(of_ordered(in), V);
                    exact = false;
                }
            }
        }
    }

    // ---- sum of the kept weights: exactly where something is drawn, of all but the first `without` drawn tokens, and of every segment
    auto drawn_of = [&](int i, int n) {                                    // which of the eight tokens from i on are among the first n drawn
        unsigned is = 0;
        for (int d = 0; d < n; ++d) {
            const unsigned k = (unsigned)(sh.drawn[d] - i);
            is |= k < 8 ? 1u << k : 0;
        }
        return is;
    };
    auto sum_up = [&](int without) {
        u64 part = 0;
        for (int s = tid; s < turns * WAVES; s += THREADS) sh.segment[s] = 0;
        __syncthreads();
        each_kept([&](int t, int i, const Eight<F32> &x, float limit) __attribute__((always_inline)) {
            const unsigned drawn = drawn_of(i, without);
            u64 here = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                u64 m = weight(x[k]);
                asm volatile("" : "+v"(m));
                here += x[k] > limit && !(drawn >> k & 1) ? m : 0;
                if (k % 2) __builtin_amdgcn_sched_barrier(0);
            }
            const u64 s = wave_sum(here);
            if (lane == 0) sh.segment[t * WAVES + wave] = s;
            part += here;
        }, cut_x);
        return block_sum(part);
    };
    // Weights in fp32: the difference and its product with log2(e) / T in two parts each, the second of which multiplies the exponential.
    // (By way of binary64 its conversions cost most: 110 cycles of a SIMD per 64 tokens, so 60.  That way is for what fp32 does not hold.)
    const float c_hi = (float)c, c_lo = (float)(c - (double)c_hi);
    const double zero_x = mxd - 151.0 / c;                                 // (powers are zero from there down; masks are as low as -3.4e38)
    const bool beyond = !(c < 1e30) || mx > 1e37f || !(fabs(mxd) * c < 1e30) || !(zero_x > -1e38);
    float floor_x = (float)zero_x;
    if ((double)floor_x > zero_x) floor_x = of_ordered(ordered(floor_x) - 1);
    auto powers = [&](const Eight<F32> &x, float (&e)[8]) __attribute__((always_inline)) {
        if (__builtin_expect(beyond, 0)) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const double y = fmax(exponent(x[k]), -1000.0), whole = rint(y);
                e[k] = __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f((float)(y - whole)), (int)whole);
                __builtin_amdgcn_sched_barrier(0);
            }
            return;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float v = fmaxf(x[k], floor_x), d = v - mx, back = d + mx, lost = (v - back) + ((back - d) - mx);      // v - mx = d + lost
            const float y = d * c_hi, rest = fmaf(lost, c_hi, fmaf(d, c_lo, fmaf(d, c_hi, -y))), w = __builtin_amdgcn_exp2f(y);
            e[k] = fmaf(w * rest, 0.69314718f, w);
            if (k % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Nothing is cut off (and what is minus infinity has a power of zero by itself).
    const bool whole = cut_x == LOWEST && cut_i == V && !beyond;
    float inv = 0.f;
    if (exact || p.n_draw) {
        if (!exact) sum = 0;
    } else {
        double part = 0.0;
        each([&](int, int i, const Eight<F32> &x) __attribute__((always_inline)) {
            float e[8];
            powers(x, e);
            if (!whole) {
                Eight<F32> z = x;
                const float limit = sift(z, i);
#pragma unroll
                for (int k = 0; k < 8; ++k) e[k] = z[k] > limit ? e[k] : 0.f;
            }
            part += (double)(((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7])));
        });
        // (in the order of the lanes and wavefronts: the same every time)
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) part += __shfl_xor(part, o);
        __syncthreads();
        if (lane == 0) sh.wave[wave] = __builtin_bit_cast(u64, part);
        __syncthreads();
        double all = lane < WAVES ? __builtin_bit_cast(double, sh.wave[lane]) : 0.0;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) all += __shfl_xor(all, o);
        inv = (float)(1.0 / all);
    }

    // ---- what draws are made from: the kept tokens in the order of indices, HELD of them in every thread, with their weights and those of
    // all before; or, where they are too many, sums of segments of 512
    float roll_x[HELD];
    int roll_i[HELD], alive = 0;                                           // (which of them are there and not drawn: bits)
    u64 roll_w[HELD], before_roll = 0;
    bool rolled = false;
    // weights relative to `top`, their sums before every thread and of all
    auto weigh_roll = [&]() {
        u64 here = 0;
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            roll_w[k] = alive >> k & 1 ? weight(roll_x[k]) : 0;
            here += roll_w[k];
        }
        before_roll = block_scan(here, sum);
    };
    if (p.n_draw) {
        const int segments = turns * WAVES;
        for (int s = tid; s < segments; s += THREADS) sh.count[s] = 0;
        __syncthreads();
        each_kept([&](int t, int i, const Eight<F32> &x, float limit) __attribute__((always_inline)) {
            int here = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) here += x[k] > limit;
            const int all = ::wave_last(::wave_scan(here));
            if (lane == 0) sh.count[t * WAVES + wave] = all;
        }, cut_x);
        __syncthreads();
        if (wave == 0) {                                                   // eight segments a lane
            int mine8[MAX_SEGMENTS / 64], all = 0;
#pragma unroll
            for (int k = 0; k < MAX_SEGMENTS / 64; ++k) {
                const int s = lane * (MAX_SEGMENTS / 64) + k;
                mine8[k] = all;
                all += s < segments ? sh.count[s] : 0;
            }
            const int in = ::wave_scan(all);
            if (lane == 63) sh.kept = in;
#pragma unroll
            for (int k = 0; k < MAX_SEGMENTS / 64; ++k)
                if (lane * (MAX_SEGMENTS / 64) + k < segments) sh.count[lane * (MAX_SEGMENTS / 64) + k] = in - all + mine8[k];
        }
        __syncthreads();
        if (sh.kept <= ROLL) {
            rolled = true;
            each_kept([&](int t, int i, const Eight<F32> &x, float limit) __attribute__((always_inline)) {
                int here = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) here += x[k] > limit;
                int at = sh.count[t * WAVES + wave] + ::wave_scan(here) - here;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (x[k] > limit) sh.roll[at++] = make_uint2(__float_as_uint(x[k]), i + k);
            }, cut_x);
            __syncthreads();
#pragma unroll
            for (int k = 0; k < HELD; ++k) {
                const uint2 v = sh.roll[tid * HELD + k];
                roll_x[k] = __uint_as_float(v.x);
                roll_i[k] = (int)v.y;
                alive |= tid * HELD + k < sh.kept ? 1 << k : 0;
            }
            weigh_roll();
        } else {
            sum = sum_up(0);
        }
    }
    if (exact || p.n_draw) inv = (float)(0x1p45 / (double)sum);

    // ---- probabilities
    if (probs) {
        each([&](int, int i, const Eight<F32> &x) __attribute__((always_inline)) {
            float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (whole) {
                powers(x, y);
#pragma unroll
                for (int k = 0; k < 8; ++k) y[k] *= inv;
            } else if (__builtin_amdgcn_ballot_w64(max8(x) >= cut_x) != 0) {      // (the other wavefronts have zeros to write)
                Eight<F32> z = x;
                const float limit = sift(z, i);
                powers(z, y);
#pragma unroll
                for (int k = 0; k < 8; ++k) y[k] = z[k] > limit ? y[k] * inv : 0.f;
            }
            if (i < V) write8(i, y);
        });
    }
    if (!p.n_draw) return;

    // ---- draws: the first token, in the order of indices, at which the sum of the weights exceeds u times all of it
    auto goal_of = [&](float u) { return __umul64hi(parts_of(u), sum); };   // (rounded down: below the sum)
    if (rolled) {
        // the thread that has it: which of its tokens
        auto take = [&](u64 goal) {
            int who = -1;
            u64 before = before_roll;
#pragma unroll
            for (int k = 0; k < HELD; ++k) {
                if (before <= goal && before + roll_w[k] > goal) who = k;
                before += roll_w[k];
            }
            return who;
        };
        for (int d = 0; d < p.n_draw; ++d) {
            if (p.distinct && d && sum < 1ull << FEW) {                    // (the same for all threads)
                u64 best = 0;                                              // the largest that is left, and all weights relative to it
#pragma unroll
                for (int k = 0; k < HELD; ++k)
                    if (alive >> k & 1) {
                        const u64 at = place_of(roll_x[k], roll_i[k]);
                        best = at > best ? at : best;
                    }
                best = block_max(best);
                if (best == 0) {                                           // nothing is left
                    if (tid >= d && tid < p.n_draw) tokens[tid] = -1;
                    return;
                }
                top = (double)of_ordered((unsigned)(best >> 18));
                weigh_roll();
            }
            const u64 goal = goal_of(us[d]);
            const int who = take(goal);
            if (who >= 0) {
                int token = 0;
                u64 weighs = 0;
#pragma unroll
                for (int k = 0; k < HELD; ++k)
                    if (who == k) {
                        token = roll_i[k];
                        weighs = roll_w[k];
                        if (p.distinct) roll_w[k] = 0;
                    }
                tokens[d] = token;
                if (p.distinct) {
                    alive &= ~(1 << who);
                    sh.winner = tid;
                    sh.above = weighs;
                }
            }
            if (p.distinct) {
                __syncthreads();
                if (tid > sh.winner) before_roll -= sh.above;
                sum -= sh.above;
                __syncthreads();
            }
        }
        return;
    }
    const int segments = turns * WAVES;
    // by one wavefront: the token, and what it weighs
    auto draw = [&](float u, int without, u64 &weighs) {
        u64 goal = goal_of(u), here = 0;
        constexpr int PER = MAX_SEGMENTS / 64;
        const int s0 = lane * PER;
        for (int k = 0; k < PER; ++k) here += s0 + k < segments ? sh.segment[s0 + k] : 0;
        u64 in = wave_scan(here), before = in - here;
        int s = -1;
        if (before <= goal && in > goal) {
            s = s0;
            while (before + sh.segment[s] <= goal) before += sh.segment[s++];
        }
        const int from = __builtin_ctzll(__builtin_amdgcn_ballot_w64(s >= 0));
        s = __shfl(s, from);
        goal -= (u64)(unsigned)__shfl((int)(before >> 32), from) << 32 | (unsigned)__shfl((int)before, from);
        const int i = (s * 64 + lane) * 8;
        Eight<F32> x;
        x.load(row, i, V);
        const unsigned drawn = drawn_of(i, without);
        u64 w[8];
        here = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            w[k] = kept(x[k], i + k) && !(drawn >> k & 1) ? weight(x[k]) : 0;
            here += w[k];
            __builtin_amdgcn_sched_barrier(0);
        }
        in = wave_scan(here);
        before = in - here;
        int token = -1;
        weighs = 0;
        if (before <= goal && in > goal) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (token < 0 && before + w[k] > goal) {
                    token = i + k;
                    weighs = w[k];
                }
                before += w[k];
            }
        }
        const int who = __builtin_ctzll(__builtin_amdgcn_ballot_w64(token >= 0));
        weighs = (u64)(unsigned)__shfl((int)(weighs >> 32), who) << 32 | (unsigned)__shfl((int)weighs, who);
        return __shfl(token, who);
    };
    __syncthreads();
    if (!p.distinct) {
        for (int d = wave; d < p.n_draw; d += WAVES) {
            u64 weighs;
            const int token = draw(us[d], 0, weighs);
            if (lane == 0) tokens[d] = token;
        }
        return;
    }
    for (int d = 0; d < p.n_draw; ++d) {
        if (d && sum < 1ull << FEW) {                                      // (the same for all threads)
            u64 best = 0;
            each_kept([&](int, int i, const Eight<F32> &x, float limit) __attribute__((always_inline)) {
                const unsigned drawn = drawn_of(i, d);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const u64 at = place_of(x[k], i + k);
                    if (at > best && x[k] > limit && !(drawn >> k & 1)) best = at;
                }
            }, cut_x);
            best = block_max(best);
            if (best == 0) {                                               // nothing is left
                if (tid >= d && tid < p.n_draw) tokens[tid] = -1;
                return;
            }
            top = (double)of_ordered((unsigned)(best >> 18));
            sum = sum_up(d);
        }
        if (wave == 0) {
            u64 weighs;
            const int token = draw(us[d], d, weighs);
            if (lane == 0) {
                tokens[d] = token;
                sh.drawn[d] = token;
                sh.segment[token / 512] -= weighs;
                sh.sum = sum - weighs;
            }
        }
        __syncthreads();
        sum = sh.sum;
        __syncthreads();
    }
}

}  // namespace

extern "C" int mcsd_sample_rows(mcsd_dtype_t dtype, int32_t B, int32_t W, int32_t V, const void *logits, int64_t batch_stride,
                                int64_t row_stride, const mcsd_sampler_t *sampler, float *probs, int64_t probs_batch_stride,
                                mcsd_sampling_t sampling, int32_t n_draw, const float *u, int32_t *tokens, int64_t tokens_batch_stride,
                                void *hip_stream)
{
    if (!logits || !sampler || (!probs && n_draw == 0)) return MCSD_EINVAL;
    if (dtype != MCSD_F32 && dtype != MCSD_BF16) return MCSD_EINVAL;
    if (sampling != MCSD_WITH_REPLACEMENT && sampling != MCSD_WITHOUT_REPLACEMENT) return MCSD_EINVAL;
    if (B < 1 || B > 65535 || W < 1 || V < 1 || n_draw < 0 || (n_draw > 0 && (!u || !tokens))) return MCSD_EINVAL;
    if (batch_stride < 0 || row_stride < 0) return MCSD_EINVAL;
    // rows that are written must not share places
    if (probs && B > 1 && probs_batch_stride < (int64_t)W * V) return MCSD_EINVAL;
    if (n_draw > 0 && B > 1 && tokens_batch_stride < (int64_t)W * n_draw) return MCSD_EINVAL;
    const uintptr_t element = dtype == MCSD_F32 ? 3 : 1;
    if (((uintptr_t)logits & element) || (((uintptr_t)probs | (uintptr_t)u | (uintptr_t)tokens) & 3)) return MCSD_EINVAL;
    if (V > MCSD_MAX_VOCAB || n_draw > MAX_DRAW || W > MCSD_MAX_GRID_1024) return MCSD_EUNSUPPORTED;
    if (probs && (const void *)probs == logits) return MCSD_EINVAL;        // (logits are read again behind the first probabilities)

    SampleParams p = {};
    p.x = logits; p.x_batch = batch_stride; p.x_row = row_stride; p.W = W; p.V = V; p.s = *sampler;
    p.probs = probs; p.p_batch = probs_batch_stride;
    p.n_draw = n_draw; p.distinct = sampling == MCSD_WITHOUT_REPLACEMENT; p.u = u; p.tokens = n_draw ? tokens : nullptr; p.t_batch = tokens_batch_stride;
    const bool f32 = dtype == MCSD_F32;
    // Fewer rows than compute units: all of a compute unit's wavefronts that fit, on one row (512 threads took 25 / 75 / 204 us for the first
    // three above where 1024 took 22 / 50 / 157); more: two workgroups to a compute unit, one's meetings under the other's passes (188 us where 1024 threads took 255).
    const bool wide = W * (int64_t)B <= mcsd_compute_units();
    auto kernel = wide ? (f32 ? sample_rows_kernel<true, 1024> : sample_rows_kernel<false, 1024>)
                       : (f32 ? sample_rows_kernel<true, 512> : sample_rows_kernel<false, 512>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)W, B), dim3(wide ? 1024 : 512), 0, (hipStream_t)hip_stream, p);
    return mcsd_hip_status(hipGetLastError());
}
