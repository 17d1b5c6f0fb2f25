// Device helpers of the microscaling formats: block scales, packing of channels
// into MXFP4 and MXFP8 codes, decoding, and the scaled matrix instructions.
//
// The conversions are gfx950's (v_cvt_scalef32_*).  Checked against the formats'
// definition on every bf16 number, on each border between two codes and on its
// neighbours in fp32, at five scales: rounding to nearest even is exact, E2M1
// saturates; E4M3 gives the NaN pattern from 464 on, and both keep the sign of a
// zero, so those two are mended after the conversion.  Only the exponent field of
// the scale operand counts, 0 for 2^-127 and 255 for NaN.
#pragma once

#include "common.hpp"
#include "polestar_mx.h"

namespace ps {

constexpr int kMxBlock = 32;                     // channels per scale

inline bool mx_fmt_ok(int fmt) { return fmt == POLESTAR_MXFP4 || fmt == POLESTAR_MXFP8; }
inline bool aligned_to(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

typedef int intx8 __attribute__((ext_vector_type(8)));
typedef int intx2 __attribute__((ext_vector_type(2)));
typedef short shortx2 __attribute__((ext_vector_type(2)));

template <int FMT> struct Mx;
template <> struct Mx<POLESTAR_MXFP4> {
    static constexpr int kBits = 4, kEmax = 2, kMant = 1, kEmin = 0;
    static constexpr int kMfma = 4;              // the matrix instructions' number of the format
};
template <> struct Mx<POLESTAR_MXFP8> {
    static constexpr int kBits = 8, kEmax = 8, kMant = 3, kEmin = -6;
    static constexpr int kMfma = 0;
};

constexpr uint32_t kMxNanScale = 255;

// Scale byte of a block from the bits of its largest magnitude (fp32, sign off):
// exponent field - emax is floor(log2 amax) - emax + 127, and a subnormal's field
// of 0 ends at the lower clamp like every exponent below it.
template <int FMT>
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t amax) {
    if (amax >= 0x7f800000u) return kMxNanScale;
    return static_cast<uint32_t>(max(static_cast<int>(amax >> 23) - Mx<FMT>::kEmax, 0));
}

// 2^(byte - 127) as the conversions take it.
__device__ __forceinline__ float mx_scale(uint32_t byte) {
    return __uint_as_float(byte == 0 ? 0x00400000u : byte << 23);
}

// Eight channels divided by sc, rounded: a dword of MXFP4 codes.
__device__ __forceinline__ uint32_t mx_pack_fp4(const float* v, float sc) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], sc, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], sc, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], sc, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], sc, 3);
    // a magnitude plus 7 reaches the sign's bit exactly where it is not 0
    return w & (0x77777777u | ((w & 0x77777777u) + 0x77777777u));
}

// Four channels divided by sc, rounded: a dword of MXFP8 codes.
__device__ __forceinline__ uint32_t mx_pack_fp8(const float* v, float sc) {
    shortx2 p = {0, 0};
    p = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(p, v[0], v[1], sc, false);
    p = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(p, v[2], v[3], sc, true);
    uint32_t w = __builtin_bit_cast(uint32_t, p);
    const uint32_t mag = w & 0x7f7f7f7fu;
    w -= ((mag + 0x01010101u) & 0x80808080u) >> 7;          // NaN pattern 0x7f: saturate to 0x7e
    return w & (0x7f7f7f7fu | (mag + 0x7f7f7f7fu));
}

// Eight channels of a block with this scale byte as codes (one dword or two).
template <int FMT>
__device__ __forceinline__ void mx_store8(uint8_t* dst, const float* v, uint32_t byte) {
    const float sc = mx_scale(byte);
    if constexpr (FMT == POLESTAR_MXFP4) {
        const uint32_t w = mx_pack_fp4(v, sc);
        *reinterpret_cast<uint32_t*>(dst) = byte == kMxNanScale ? 0u : w;
    } else {
        uint2 w = make_uint2(mx_pack_fp8(v, sc), mx_pack_fp8(v + 4, sc));
        if (byte == kMxNanScale) w = make_uint2(0u, 0u);
        *reinterpret_cast<uint2*>(dst) = w;
    }
}

// Eight consecutive channels as fp32.
template <bool BF16>
__device__ __forceinline__ void ld8(const char* p, float* v) {
    if constexpr (BF16) {
        Elem<true>::unpack(ld16(p), v);
    } else {
        Elem<false>::unpack(ld16(p), v);
        Elem<false>::unpack(ld16(p + 16), v + 4);
    }
}

// The block's scale byte where four neighbouring lanes hold its 32 channels.
template <int FMT>
__device__ __forceinline__ uint32_t mx_block_byte(const float* v) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 1)));
    m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 2)));
    return mx_scale_byte<FMT>(m);
}

// Eight MXFP4 codes (a dword) of a block as bf16, exact but for magnitudes below
// bf16's subnormals, in the order of the channels.
__device__ __forceinline__ uint4 mx_fp4_bf16(uint32_t w, float sc) {
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 0)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 1)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 2)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 3)));
}
// Eight MXFP8 codes (two dwords) as bf16.
__device__ __forceinline__ uint4 mx_fp8_bf16(uint32_t a, uint32_t b, float sc) {
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, sc, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, sc, true)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, sc, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, sc, true)));
}

}  // namespace ps
