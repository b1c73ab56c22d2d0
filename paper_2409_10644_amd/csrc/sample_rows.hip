// From logits to the probability rows that the verification takes, and tokens drawn from them (definition in mcsd.h).
//
// A workgroup of 1024 threads has a row; it stays in its registers where it fits.  The tokens of a row are ordered by logit, largest
// first, then by index; top-k, top-p and min-p each keep a beginning of that order, and the shortest counts.  Where it ends is found
// without a sort: 2048 places for ranges of logits, the tokens of the one place where the count or the sum reaches its goal listed,
// and each of them ranked against the others; more of them than the list holds are cut into 2048 ranges again, of logit and index as
// one number.
//
// A weight is 2^((x - max) log2(e) / T) as a whole number of 2^-45: the sums are exact whatever their order (so atomics may add them),
// a border of top-p and a draw depend on nothing but the weights, and 2^18 of them stay below 2^64.  It is computed in binary64,
// so a border falls where 64 bits have it.  A probability is computed in fp32, of the exponent in two parts.
#include <math.h>

#include "mcsd_internal.h"

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

constexpr int THREADS = 1024, WAVES = 16, BINS = 2048, LIST = 1024, MAX_DRAW = 64;
constexpr int ONE = 45;                  // a weight of 1 is 2^45
constexpr int FEW = 41;                  // distinct draws: below a sum of 2^41 the weights are made anew around the largest that is left
constexpr int MAX_SEGMENTS = MCSD_MAX_VOCAB / 512;

struct Shared {
    u64 hist[BINS];
    u64 list[LIST], weight[LIST];
    u64 segment[MAX_SEGMENTS];           // sums of 512 tokens
    u64 wave[WAVES], wave2[WAVES];
    u64 above, sum, cut;
    int32_t bin, listed, index, stop;
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

// 2^y for y <= 0: the polynomial is 2^f on [-1/2, 1/2] interpolated at the 11 Chebyshev points, off by at most 2^-51.5 of it.
__device__ __forceinline__ u64 weight_of(double y)
{
    if (y < -(ONE + 1.0)) return 0;
    const double n = rint(y), f = y - n;
    double p = 0x1.e6063f7217bc6p-28;
    p = fma(p, f, 0x1.b675bca4eeebbp-24);
    p = fma(p, f, 0x1.62bfd47773353p-20);
    p = fma(p, f, 0x1.ffcb54062e698p-17);
    p = fma(p, f, 0x1.430913096fd9fp-13);
    p = fma(p, f, 0x1.5d87fe9d7a584p-10);
    p = fma(p, f, 0x1.3b2ab6fba1ddap-7);
    p = fma(p, f, 0x1.c6b08d703ce49p-5);
    p = fma(p, f, 0x1.ebfbdff82c598p-3);
    p = fma(p, f, 0x1.62e42fefa3a19p-1);
    p = fma(p, f, 1.0);
    // (2^52 added: the sum's last place is 1)
    const double s = ldexp(p, (int)n + ONE) + 0x1p52;
    return __builtin_bit_cast(u64, s) & 0xfffffffffffffull;
}

__device__ __forceinline__ u64 shfl_xor64(u64 v, int o)
{
    return (u64)(unsigned)__shfl_xor((int)(v >> 32), o) << 32 | (unsigned)__shfl_xor((int)v, o);
}
__device__ __forceinline__ u64 shfl_up64(u64 v, int o)
{
    return (u64)(unsigned)__shfl_up((int)(v >> 32), o) << 32 | (unsigned)__shfl_up((int)v, o);
}
__device__ __forceinline__ u64 wave_sum(u64 v)
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v += shfl_xor64(v, o);
    return v;
}
__device__ __forceinline__ u64 wave_scan(u64 v, int lane)                // inclusive
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const u64 below = shfl_up64(v, o);
        if (lane >= o) v += below;
    }
    return v;
}

// Eight logits from index i on; behind the row's end minus infinity.  (Rows begin anywhere.)
template <bool F32>
struct Eight {
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
    // What one pass makes of them is not kept in registers for the next.
    __device__ __forceinline__ void anew()
    {
#pragma unroll
        for (int k = 0; k < (F32 ? 8 : 4); ++k) asm volatile("" : "+v"(w[k]));
    }
    __device__ __forceinline__ float operator[](int k) const
    {
        if constexpr (F32) return __uint_as_float(w[k]);
        else return __uint_as_float(k & 1 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16);
    }
};

// NIT: turns of 8192 logits that the registers hold; 0: the row is read again for every pass
template <bool F32, int NIT>
__global__ __launch_bounds__(THREADS) void sample_rows_kernel(const SampleParams p)
{
    __shared__ Shared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = blockIdx.x, b = blockIdx.y;
    const int V = p.V, turns = (V + 8191) / 8192;
    const void *row = (const char *)p.x + ((int64_t)b * p.x_batch + (int64_t)r * p.x_row) * (F32 ? 4 : 2);
    Eight<F32> kept_row[NIT > 0 ? NIT : 1];
    if constexpr (NIT > 0) {
#pragma unroll
        for (int t = 0; t < NIT; ++t) kept_row[t].load(row, (t * THREADS + tid) * 8, V);
    }
    // f(turn, first index, eight logits)
    auto each = [&](auto f) __attribute__((always_inline)) {
        if constexpr (NIT > 0) {
#pragma unroll
            for (int t = 0; t < NIT; ++t) {
                kept_row[t].anew();
                if (t < turns) f(t, (t * THREADS + tid) * 8, kept_row[t]);
            }
        } else {
            for (int t = 0; t < turns; ++t) {
                Eight<F32> x;
                x.load(row, (t * THREADS + tid) * 8, V);
                f(t, (t * THREADS + tid) * 8, x);
            }
        }
    };
    // over the workgroup: sums, maxima; all threads get them
    auto block_sum = [&](u64 v) {
        v = wave_sum(v);
        __syncthreads();
        if (lane == 0) sh.wave[wave] = v;
        __syncthreads();
        u64 s = 0;
        for (int k = 0; k < WAVES; ++k) s += sh.wave[k];
        return s;
    };
    auto block_max = [&](u64 v) {
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const u64 u = shfl_xor64(v, o);
            v = u > v ? u : v;
        }
        __syncthreads();
        if (lane == 0) sh.wave[wave] = v;
        __syncthreads();
        u64 s = 0;
        for (int k = 0; k < WAVES; ++k) s = sh.wave[k] > s ? sh.wave[k] : s;
        return s;
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

    // ---- maximum, smallest finite logit, and whether the row is one
    const float T = p.s.temperature ? p.s.temperature[b] : 1.f, top_p = p.s.top_p ? p.s.top_p[b] : 1.f, min_p = p.s.min_p ? p.s.min_p[b] : 0.f;
    const int top_k = p.s.top_k ? p.s.top_k[b] : 0;
    float mx = -INFINITY, mn = INFINITY;
    bool bad = false;
    each([&](int, int, const Eight<F32> &x) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            mx = fmaxf(mx, x[k]);
            mn = x[k] > -INFINITY ? fminf(mn, x[k]) : mn;
            bad |= !(x[k] < INFINITY);                                     // NaN or infinite
        }
    });
    bad = __syncthreads_or(bad) || !(T >= 0.f) || top_p != top_p || min_p != min_p;
    mx = of_ordered((unsigned)block_max(ordered(mx)));
    mn = of_ordered(~(unsigned)block_max(~ordered(mn)));
    if (bad || mx == -INFINITY) {                                          // no distribution: NaN, or nothing to choose from: zeros
        const float v = bad ? NAN : 0.f;
        const float y[8] = {v, v, v, v, v, v, v, v};
        if (probs)
            for (int t = 0; t < turns; ++t)
                if ((t * THREADS + tid) * 8 < V) write8((t * THREADS + tid) * 8, y);
        if (tid < p.n_draw) tokens[tid] = -1;
        return;
    }

    // ---- the cut: a token is kept if its place is not below it, and its exponent not below min_y
    const double c = T > 0.f ? 1.4426950408889634074 / (double)T : 0.0;
    double top = (double)mx;                                               // what weights are relative to
    const double min_y = min_p > 0.f ? fmin(log2((double)min_p), 0.0) : -INFINITY;
    u64 cut = place_of(-INFINITY, 0) + 1;                                  // everything but minus infinity
    // The place at which the sum of measure(logit) over the tokens from the first on reaches goal(sum of all) >= 1, which becomes the cut;
    // returns the sum up to and with it.
    auto find = [&](auto measure, auto goal) -> u64 {
        const float range = fminf(mx - mn, 31.9f * T), scale = range > 0.f && range < INFINITY ? (BINS - 0.5f) / range : 0.f;
        auto bin_of = [&](float x) { return scale > 0.f ? (int)fminf((mx - x) * scale, (float)(BINS - 1)) : 0; };
        auto clear = [&]() {
            sh.hist[tid] = 0;
            sh.hist[tid + THREADS] = 0;
            if (tid == 0) sh.listed = 0;
            __syncthreads();
        };
        // where the sum of the 2048 places reaches the goal: sh.bin, and sh.above up to there; above: what is before the first of them
        u64 target = 0;
        auto choose = [&](u64 above, bool first) {
            __syncthreads();
            const u64 h0 = sh.hist[2 * tid], h1 = sh.hist[2 * tid + 1], in = wave_scan(h0 + h1, lane);
            if (lane == 63) sh.wave2[wave] = in;
            __syncthreads();
            u64 before = above + in - (h0 + h1), all = above;
            for (int k = 0; k < WAVES; ++k) {
                all += sh.wave2[k];
                if (k < wave) before += sh.wave2[k];
            }
            if (first) target = goal(all);
            if (before < target && before + h0 >= target) { sh.bin = 2 * tid; sh.above = before; }
            if (before + h0 < target && before + h0 + h1 >= target) { sh.bin = 2 * tid + 1; sh.above = before + h0; }
            __syncthreads();
        };
        clear();
        each([&](int, int i, const Eight<F32> &x) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (place_of(x[k], i + k) >= cut) {
                    const u64 m = measure(x[k]);
                    if (m) atomicAdd(&sh.hist[bin_of(x[k])], m);
                }
        });
        choose(0, true);
        int bin = sh.bin;
        u64 above = sh.above, lo = 0, hi = ~0ull;
        each([&](int, int i, const Eight<F32> &x) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const u64 at = place_of(x[k], i + k);
                if (at >= cut && bin_of(x[k]) == bin) {
                    const int n = atomicAdd(&sh.listed, 1);
                    if (n < LIST) sh.list[n] = at;
                }
            }
        });
        __syncthreads();
        if (sh.listed > LIST) {
            // from here on by place: the range lo .. hi is cut until its tokens fit the list
            lo = ~0ull;
            hi = 0;
            each([&](int, int i, const Eight<F32> &x) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const u64 at = place_of(x[k], i + k);
                    if (at >= cut && bin_of(x[k]) == bin) {
                        lo = at < lo ? at : lo;
                        hi = at > hi ? at : hi;
                    }
                }
            });
            hi = block_max(hi);
            lo = ~block_max(~lo);
            while (sh.listed > LIST) {
                int shift = 0;
                while ((hi - lo) >> shift >= BINS) ++shift;
                __syncthreads();
                clear();
                each([&](int, int i, const Eight<F32> &x) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const u64 at = place_of(x[k], i + k);
                        if (at >= lo && at <= hi) {
                            const u64 m = measure(x[k]);
                            if (m) atomicAdd(&sh.hist[(hi - at) >> shift], m);
                        }
                    }
                });
                choose(above, false);
                above = sh.above;
                const u64 end = hi - ((u64)sh.bin << shift), begin = end - ((1ull << shift) - 1);
                hi = end;
                lo = begin > lo && begin <= end ? begin : lo;
                each([&](int, int i, const Eight<F32> &x) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const u64 at = place_of(x[k], i + k);
                        if (at >= lo && at <= hi) {
                            const int n = atomicAdd(&sh.listed, 1);
                            if (n < LIST) sh.list[n] = at;
                        }
                    }
                });
                __syncthreads();
            }
        }
        // the listed ones among themselves
        const int n = sh.listed;
        u64 mine = 0, own = 0;
        if (tid < n) {
            mine = sh.list[tid];
            own = measure(of_ordered((unsigned)(mine >> 18)));
            sh.weight[tid] = own;
        }
        __syncthreads();
        if (tid < n) {
            u64 before = above;
            for (int k = 0; k < n; ++k) before += sh.list[k] > mine ? sh.weight[k] : 0;
            if (before < target && before + own >= target) { sh.cut = mine; sh.sum = before + own; }
        }
        __syncthreads();
        cut = sh.cut;
        return sh.sum;
    };
    auto weight = [&](float x) { return weight_of(((double)x - top) * c); };
    if (T == 0.f || top_k == 1) {                                          // the largest alone
        int first = V;
        each([&](int, int i, const Eight<F32> &x) {
#pragma unroll
            for (int k = 7; k >= 0; --k) first = x[k] == mx && i + k < first ? i + k : first;
        });
        cut = place_of(mx, (int)~block_max(~(u64)(unsigned)first));
    } else {
        if (top_k > 0 && top_k < V)
            find([](float) { return (u64)1; }, [&](u64 all) { return all < (u64)top_k ? all : (u64)top_k; });
        if (top_p < 1.f)
            find([&](float x) { return weight(x); },
                 [&](u64 all) { const double g = ceil((double)top_p * (double)all); return g < 1.0 ? (u64)1 : (u64)g; });
    }
    auto exponent = [&](float x) { return ((double)x - (double)mx) * c; };
    auto kept = [&](float x, int i) { return place_of(x, i) >= cut && exponent(x) >= min_y; };
    auto drawn_before = [&](int i, int n) {
        bool is = false;
        for (int k = 0; k < n; ++k) is |= sh.drawn[k] == i;
        return is;
    };

    // ---- sum, probabilities
    // (all but the first `without` drawn tokens; also of every segment, where there is something to draw)
    auto sum_up = [&](int without) {
        u64 part = 0;
        each([&](int t, int i, const Eight<F32> &x) {
            u64 here = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (kept(x[k], i + k) && !drawn_before(i + k, without)) here += weight(x[k]);
            if (p.n_draw) {
                const u64 s = wave_sum(here);
                if (lane == 0) sh.segment[t * WAVES + wave] = s;
            }
            part += here;
        });
        return block_sum(part);
    };
    u64 sum = sum_up(0);
    if (probs) {
        const float inv = (float)(0x1p45 / (double)sum);
        each([&](int, int i, const Eight<F32> &x) {
            float y[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const double e = fmax(exponent(x[k]), -200.0);             // (nothing in fp32 either way; masks are as low as -3.4e38)
                const float hi = (float)e, lo = (float)(e - (double)hi);
                y[k] = kept(x[k], i + k) ? __builtin_amdgcn_exp2f(hi) * inv * fmaf(lo, 0.69314718f, 1.f) : 0.f;
            }
            if (i < V) write8(i, y);
        });
    }

    // ---- draws: the first token, in the order of indices, at which the sum of the weights exceeds u times all of it
    const int segments = turns * WAVES;
    // by one wavefront: the token, and what it weighs
    auto draw = [&](float u, int without, u64 &weighs) {
        u = fminf(fmaxf(u, 0.f), 0x1.fffffep-1f);
        u64 goal = (u64)((double)u * (double)sum);
        goal = goal < sum ? goal : sum - 1;
        u64 own = 0;
        constexpr int PER = MAX_SEGMENTS / 64;
        const int s0 = lane * PER;
        for (int k = 0; k < PER; ++k) own += s0 + k < segments ? sh.segment[s0 + k] : 0;
        u64 in = wave_scan(own, lane), before = in - own;
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
        u64 w[8];
        own = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            w[k] = kept(x[k], i + k) && !drawn_before(i + k, without) ? weight(x[k]) : 0;
            own += w[k];
        }
        in = wave_scan(own, lane);
        before = in - own;
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
    if (!p.n_draw) return;
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
            // the largest that is left, and all weights relative to it
            u64 best = 0;
            each([&](int, int i, const Eight<F32> &x) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const u64 at = place_of(x[k], i + k);
                    if (at > best && kept(x[k], i + k) && !drawn_before(i + k, d)) best = at;
                }
            });
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

    SampleParams p = {};
    p.x = logits; p.x_batch = batch_stride; p.x_row = row_stride; p.W = W; p.V = V; p.s = *sampler;
    p.probs = probs; p.p_batch = probs_batch_stride;
    p.n_draw = n_draw; p.distinct = sampling == MCSD_WITHOUT_REPLACEMENT; p.u = u; p.tokens = n_draw ? tokens : nullptr; p.t_batch = tokens_batch_stride;
    const bool f32 = dtype == MCSD_F32;
    auto kernel = f32 ? (V <= 8192 ? sample_rows_kernel<true, 1> : V <= 32768 ? sample_rows_kernel<true, 4> : sample_rows_kernel<true, 0>)
                      : (V <= 8192 ? sample_rows_kernel<false, 1> : V <= 32768 ? sample_rows_kernel<false, 4> : V <= 65536 ? sample_rows_kernel<false, 8> : sample_rows_kernel<false, 0>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)W, B), dim3(THREADS), 0, (hipStream_t)hip_stream, p);
    return mcsd_hip_status(hipGetLastError());
}
