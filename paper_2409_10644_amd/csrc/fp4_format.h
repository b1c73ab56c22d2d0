// The 4-bit cache format on gfx950 (see the format in mcsd.h): 32 channels share an E8M0 scale byte, codes are E2M1.
#pragma once
#include "mcsd_internal.h"

// Lanes that exchange within their group of four: quad permutations 1,0,3,2 and 2,3,0,1.
template <int CTRL>
__device__ __forceinline__ unsigned dpp_move(unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }
constexpr int DPP_XOR1 = 0xB1, DPP_XOR2 = 0x4E, DPP_HALF_MIRROR = 0x141;

// Eight numbers of a lane, 32 of its quad (a group): codes of the lane's eight, and the group's scale byte.
// The maximum is taken over magnitudes as integers, which orders infinities and NaN above every number.
__device__ __forceinline__ unsigned fp4_quantise8(const float (&x)[8], unsigned &byte)
{
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
    m = max(m, dpp_move<DPP_XOR1>(m));
    m = max(m, dpp_move<DPP_XOR2>(m));
    // half a step of one fraction bit added, then the exponent field: a carry is the step to the next power of two
    const int e = max((int)((m + 0x200000u) >> 23) - 2, 1);
    const float scale = __uint_as_float((unsigned)e << 23);
    unsigned codes = 0;                                        // (rounds to nearest, ties to the even code, saturates at 6)
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], scale, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], scale, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], scale, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], scale, 3);
    const bool number = m < 0x7f800000u;
    byte = number ? (unsigned)e : 255u;
    return number ? codes : 0u;
}

// The scale operand of the conversions below: they take its exponent field alone, as E8M0 (0: 2^-127, 255: NaN).
__device__ __forceinline__ float fp4_scale(unsigned byte) { return __uint_as_float(byte << 23); }

// 8 codes of one group -> 8 bf16 (two per dword), exact.
__device__ __forceinline__ uint4 fp4x8_to_bf16(unsigned codes, float scale)
{
    return make_uint4(__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                      __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                      __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                      __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3)));
}

// Division by a number the host knows: floor(a / d) = a * mul >> (31 + shift) for 0 <= a < 2^31 with shift = ceil(log2 d),
// mul = ceil(2^(31 + shift) / d).
struct RowDiv { uint32_t mul, shift; };
static inline RowDiv row_div_of(uint32_t d)
{
    RowDiv f = {0, 0};
    while ((1ull << f.shift) < d) ++f.shift;
    f.mul = (uint32_t)(((1ull << (31 + f.shift)) + d - 1) / d);
    return f;
}
__device__ __forceinline__ int row_div(int a, RowDiv f) { return (int)(((uint64_t)(uint32_t)a * f.mul) >> (31 + f.shift)); }

static inline bool fp4_cache_ok(const mcsd_fp4_cache_t *c)
{
    if (!c || !c->k_codes || !c->k_scales || !c->v_codes || !c->v_scales) return false;
    return !(((uintptr_t)c->k_codes | (uintptr_t)c->v_codes) & 15) && !(((uintptr_t)c->k_scales | (uintptr_t)c->v_scales) & 3);
}
