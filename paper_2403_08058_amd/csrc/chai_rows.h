// Cached rows of 128 elements in registers: storage types, how the lanes of a wave share rows, widening, cross-lane sums.
#pragma once

#include "chai_internal.h"

namespace chai {

namespace {

constexpr int kUnroll = 8;        // 16-byte loads per lane in one batch

// storage types of the caches: CHAI_F32, CHAI_BF16, and 8-bit E4M3 codes with per-row scales
constexpr int DT_F32 = CHAI_F32, DT_BF16 = CHAI_BF16, DT_E4M3 = 2;
template <int DT>
struct Elem {
    static constexpr int BYTES = DT == DT_F32 ? 4 : (DT == DT_BF16 ? 2 : 1);
    static constexpr int EPL = 16 / BYTES;                 // elements per lane per load (16 bytes)
};

template <int DT>
struct Tile {
    static constexpr int EPL = Elem<DT>::EPL;
    static constexpr int LPR = kHeadDim / EPL;             // lanes per row: 32 (fp32) / 16 (bf16) / 8 (codes)
    static constexpr int RPW = 64 / LPR;                   // rows per wave load: 2 / 4 / 8
    static constexpr int BATCH = RPW * kUnroll;            // rows per wave batch: 16 / 32 / 64
    static constexpr int ROW_BYTES = kHeadDim * Elem<DT>::BYTES;
};

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ void unpack(const u32x4 &raw, float (&f)[8])
{
    // bf16 pairs: the low half-word is the even element; a bf16 is the top half of an fp32
    f[0] = __uint_as_float(raw.x << 16); f[1] = __uint_as_float(raw.x & 0xffff0000u);
    f[2] = __uint_as_float(raw.y << 16); f[3] = __uint_as_float(raw.y & 0xffff0000u);
    f[4] = __uint_as_float(raw.z << 16); f[5] = __uint_as_float(raw.z & 0xffff0000u);
    f[6] = __uint_as_float(raw.w << 16); f[7] = __uint_as_float(raw.w & 0xffff0000u);
}

// sixteen E4M3 codes: the hardware conversion widens two bytes of a word at a time (exact)
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void unpack(const u32x4 &raw, float (&f)[16])
{
    const unsigned int w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false);
        const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
        f[4 * i + 0] = lo.x; f[4 * i + 1] = lo.y; f[4 * i + 2] = hi.x; f[4 * i + 3] = hi.y;
    }
}

__device__ __forceinline__ void unpack(const u32x4 &raw, float (&f)[4])
{
    f[0] = __uint_as_float(raw.x); f[1] = __uint_as_float(raw.y);
    f[2] = __uint_as_float(raw.z); f[3] = __uint_as_float(raw.w);
}

// The caches are read exactly once per call: non-temporal loads keep them from displacing the small,
// re-read score and statistics buffers in L2 (and measure ~10% faster than plain loads on a pure stream).
__device__ __forceinline__ u32x4 stream16(const char *p)
{
    return __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
}

// x + (x of the lane selected by a DPP control) -- cross-lane adds inside a 16-lane DPP row
template <int CTRL>
__device__ __forceinline__ float dpp_add(float x)
{
    int y = __builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, false);
    return x + __int_as_float(y);
}

// Sum over the lanes that share a row; every one of them ends up with the total.
template <int DT>
__device__ __forceinline__ float row_sum(float x)
{
    x = dpp_add<0xB1>(x);    // quad_perm [1,0,3,2]: lane ^ 1
    x = dpp_add<0x4E>(x);    // quad_perm [2,3,0,1]: lane ^ 2
    x = dpp_add<0x141>(x);   // row_half_mirror: other quad of the same 8 lanes (rows of 8-bit codes end here)
    if (DT != DT_E4M3) x = dpp_add<0x140>(x);   // row_mirror: other half of the same 16 lanes
    if (DT == DT_F32) x += __shfl_xor(x, 16);   // fp32 rows span 32 lanes
    return x;
}

__device__ __forceinline__ float wave_max(float x)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
    return x;
}

__device__ __forceinline__ float wave_sum(float x)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
    return x;
}

// E4M3 codes of four values of at most 448 (the clamp leaves no NaN): the hardware's conversion (nearest, ties to even, subnormals
// kept), two at a time.  It gives the code that integer arithmetic on the bits gave for all 2 277 507 074 fp32 numbers of that size.
// Those, some fifteen instructions each, were what the kernel waited for.
__device__ __forceinline__ unsigned int e4m3_codes(float a, float b, float c, float d)
{
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (unsigned int)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}

// max over the sixteen lanes of a DPP row, in every one of them
template <int CTRL>
__device__ __forceinline__ float dpp_max(float x)
{
    return fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, false)));
}

// Sixteen lanes quantise one row, eight elements each (x): returns the eight codes of this lane (two words) and the
// row's scale.  All sixteen lanes of the group must call it together.
struct Piece {
    float x[8];
};
template <bool BF16>
__device__ __forceinline__ Piece load_piece(const char *row, int piece)
{
    Piece p;
    if (BF16) {
        const uint4 raw = *reinterpret_cast<const uint4 *>(row + piece * 16);
        const unsigned int w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p.x[2 * i] = __uint_as_float(w[i] << 16);
            p.x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    } else {
        const float4 lo = *reinterpret_cast<const float4 *>(row + piece * 32);
        const float4 hi = *reinterpret_cast<const float4 *>(row + piece * 32 + 16);
        p.x[0] = lo.x; p.x[1] = lo.y; p.x[2] = lo.z; p.x[3] = lo.w;
        p.x[4] = hi.x; p.x[5] = hi.y; p.x[6] = hi.z; p.x[7] = hi.w;
    }
    return p;
}
// the largest magnitude of the row
__device__ __forceinline__ float largest_of(const Piece &p)
{
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(p.x[i]));
    amax = dpp_max<0xB1>(amax);                      // quad_perm [1,0,3,2], [2,3,0,1], row_half_mirror, row_mirror
    amax = dpp_max<0x4E>(amax);
    amax = dpp_max<0x141>(amax);
    return dpp_max<0x140>(amax);
}
// the codes of a piece; inv = 448 / the largest magnitude
__device__ __forceinline__ uint2 codes_of(const Piece &p, float inv)
{
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = fminf(fmaxf(p.x[i] * inv, -448.0f), 448.0f);
    return make_uint2(e4m3_codes(y[0], y[1], y[2], y[3]), e4m3_codes(y[4], y[5], y[6], y[7]));
}
__device__ __forceinline__ uint2 quantize_piece(const Piece &p, float &scale)
{
    const float amax = largest_of(p);
    if (amax == 0.f) {
        scale = 0.f;
        return make_uint2(0u, 0u);
    }
    scale = amax / 448.0f;
    return codes_of(p, 448.0f / amax);
}

}  // namespace

}  // namespace chai
