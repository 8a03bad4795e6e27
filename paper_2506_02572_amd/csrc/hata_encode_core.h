// Operands and results of the key encoders on the matrix cores (hata_encode.hip, hata_pages.hip).
#pragma once
#include "hata_device.h"

namespace hata {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
#define HATA_MFMA_PITCH 136   // LDS row pitch in bf16 elements (272 B: rows shift by 4 banks)

// Bit 8 (i / 4) + i % 4: acc[i] >= 0, the complement of the sign bit (a sum of exact products that starts from +0 is
// never -0; the NaN that the matrix cores make of a NaN or of infinities that cancel has its sign bit set, whatever the
// input's was, so such a bit is 0 as in a comparison).  One instruction a value and four to part the groups of four; with two a value, shift and
// insertion, 131072 keys of eight heads took encode_dma_kernel 135.4 us instead of 132.1 (r = 256), 70.8 instead of 68.1 (128).
__device__ __forceinline__ uint32_t sign_bits(const f32x16_t& acc) {
    uint32_t neg = 0;
#pragma unroll
    for (int i = 15; i >= 0; --i) neg = __builtin_amdgcn_alignbit(neg, __float_as_uint(acc[i]), 31);  // 2 neg + sign
    neg = (neg | neg << 8) & 0x00ff00ffu;
    return ~(neg | neg << 4) & 0x0f0f0f0fu;
}

// fp32 weight pair -> the three bf16 planes (hi, mid, lo) whose sum is the weight exactly; two weights per dword
__device__ __forceinline__ void split_weight_pair(float w0, float w1, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
    uint32_t ph[2], pm[2], pl[2];
    const float wv2[2] = {w0, w1};
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const float wv = wv2[q];
        ph[q] = f32_to_bf16(wv);
        const float r1 = wv - __uint_as_float(ph[q] << 16);
        pm[q] = f32_to_bf16(r1);
        const float r2 = r1 - __uint_as_float(pm[q] << 16);
        pl[q] = f32_to_bf16(r2);
    }
    hi = ph[0] | (ph[1] << 16);
    mid = pm[0] | (pm[1] << 16);
    lo = pl[0] | (pl[1] << 16);
}

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8_t;

// eight bf16 values (one 16-byte operand fragment) -> fp16
__device__ __forceinline__ f16x8_t bf16x8_to_f16(const uint4 v) {
    const uint32_t x[4] = {v.x, v.y, v.z, v.w};
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        o[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(bf16_lo(x[i]), bf16_hi(x[i])));
    return __builtin_bit_cast(f16x8_t, make_uint4(o[0], o[1], o[2], o[3]));
}

// 16 bytes that nobody reads again
__device__ __forceinline__ uint4 load_once(const uint16_t* p) {
    typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
    return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p)));
}

}  // namespace hata
