// What the kernels of both translation units share: element types and conversions, wavefront reductions, the two-term form of activations.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace msd {

typedef uint16_t bf16_t;  // raw bf16 bit pattern
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------------------------------
// element conversion

__device__ __forceinline__ float bf2f(bf16_t b) { return __uint_as_float(((uint32_t)b) << 16); }

// round-to-nearest-even float -> bf16, the hardware's conversion (one instruction for two values; the same bits as adding the rounding
// term by hand for every finite value and infinity, six instructions each)
typedef __bf16 hbf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t f2bf2(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, hbf16x2)); }
__device__ __forceinline__ bf16_t f2bf(float f) { return __builtin_bit_cast(bf16_t, (__bf16)f); }

template <typename T> struct El;
template <> struct El<float> {
    static __device__ __forceinline__ float ld(float v) { return v; }
    static __device__ __forceinline__ float st(float v) { return v; }
};
template <> struct El<bf16_t> {
    static __device__ __forceinline__ float ld(bf16_t v) { return bf2f(v); }
    static __device__ __forceinline__ bf16_t st(float v) { return f2bf(v); }
};

// ------------------------------------------------------------------------------------------
// wavefront (64 lanes) reductions

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}

// Reductions in the vector unit's own lane moves (DPP): four shifts inside rows of 16 lanes, then the row totals handed on.  A step is
// one dependent move and one operation, about a tenth of the LDS permute that __shfl_xor is; used where such chains are on the
// critical path (accept and sampling kernels).  Every lane gets the inclusive scan; the total is lane 63's.
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_move(float old, float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(old), __float_as_int(v), CTRL, ROWS, 0xf, false));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_move(double v) {          // lanes without a source get 0
    constexpr bool ALL = ROWS == 0xf;                           // (rows left out keep the 0 that the destination is filled with first)
    const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, ROWS, 0xf, ALL);
    const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, ROWS, 0xf, ALL);
    return __hiloint2double(hi, lo);
}
__device__ __forceinline__ float dpp_max(float v) {
    // row_shr:1, 2, 4, 8, row_bcast:15 into rows 1 and 3, row_bcast:31 into rows 2 and 3; a lane without a source keeps its value.  (A DPP
    // operand is read two wait states after it was written.)
    asm("s_nop 1\n\tv_max_f32_dpp %0, %0, %0 row_shr:1 row_mask:0xf bank_mask:0xf\n\t"
        "s_nop 1\n\tv_max_f32_dpp %0, %0, %0 row_shr:2 row_mask:0xf bank_mask:0xf\n\t"
        "s_nop 1\n\tv_max_f32_dpp %0, %0, %0 row_shr:4 row_mask:0xf bank_mask:0xf\n\t"
        "s_nop 1\n\tv_max_f32_dpp %0, %0, %0 row_shr:8 row_mask:0xf bank_mask:0xf\n\t"
        "s_nop 1\n\tv_max_f32_dpp %0, %0, %0 row_bcast:15 row_mask:0xa bank_mask:0xf\n\t"
        "s_nop 1\n\tv_max_f32_dpp %0, %0, %0 row_bcast:31 row_mask:0xc bank_mask:0xf" : "+v"(v));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ double dpp_scan(double v) {
    v += dpp_move<0x111, 0xf>(v);
    v += dpp_move<0x112, 0xf>(v);
    v += dpp_move<0x114, 0xf>(v);
    v += dpp_move<0x118, 0xf>(v);
    v += dpp_move<0x142, 0xa>(v);
    v += dpp_move<0x143, 0xc>(v);
    return v;
}
__device__ __forceinline__ double dpp_sum(double v) {
    v = dpp_scan(v);
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), 63), __builtin_amdgcn_readlane(__double2loint(v), 63));
}

// ------------------------------------------------------------------------------------------
// Activations handed to the bf16 GEMM are stored as two bf16 terms, x = hi + lo with hi = bf16(x),
// lo = bf16(x - hi): array hi[n] at `base`, array lo[n] right behind it (n = elements of the whole
// block).  The producer pays the conversion once; every GEMM workgroup then copies 16-byte pieces.
__device__ __forceinline__ void store_split4(float* base, size_t n, size_t at, const float4& v) {
    bf16_t* hi = reinterpret_cast<bf16_t*>(base) + at;
    bf16_t* lo = hi + n;
    const uint32_t h01 = f2bf2(v.x, v.y), h23 = f2bf2(v.z, v.w);
    *reinterpret_cast<uint2*>(hi) = make_uint2(h01, h23);
    *reinterpret_cast<uint2*>(lo) = make_uint2(
        f2bf2(v.x - __uint_as_float(h01 << 16), v.y - __uint_as_float(h01 & 0xffff0000u)),
        f2bf2(v.z - __uint_as_float(h23 << 16), v.w - __uint_as_float(h23 & 0xffff0000u)));
}
// The interleaved form of the same two terms, read by the many-row GEMM (gemm_tiles.h): per row and 32-wide chunk one 128-byte
// line, the 32 hi terms, then the 32 lo terms.  at: element index in a row-major block whose rows are a multiple of 32 long.
__device__ __forceinline__ size_t il_index(size_t at) { return 2 * at - (at & 31); }
// split = 1: two arrays, n = elements of the whole block; split = 2: interleaved
__device__ __forceinline__ void store_terms4(float* base, int split, size_t n, size_t at, const float4& v) {
    if (split == 2) store_split4(base, 32, il_index(at), v);
    else store_split4(base, n, at, v);
}
__device__ __forceinline__ void store_split1(float* base, size_t n, size_t at, float v) {
    bf16_t* hi = reinterpret_cast<bf16_t*>(base) + at;
    const bf16_t h = f2bf(v);
    hi[0] = h;
    hi[n] = f2bf(v - bf2f(h));
}
// the two-term form of a pair: hi = bf16(x), lo = bf16(x - hi)
__device__ __forceinline__ void split_pair(float a, float b, uint32_t& hi, uint32_t& lo) {
    hi = f2bf2(a, b);
    lo = f2bf2(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xffff0000u));
}

}  // namespace msd
