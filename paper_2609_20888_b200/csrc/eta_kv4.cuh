// The 4-bit cache format: where its bytes are, and what they stand for.
//
// A block of b tokens of one KV head is one run of bytes: K codes [b][d / 2], K scales [b][d / 16], V codes, V scales.  A code is an
// e2m1 value, a scale an e4m3 one: their product has at most six significant bits and lies between 2^-10 and 2688, so it is an
// exact fp16 number, and the product of two such operands is exact in the fp32 accumulators of the tensor cores.
#pragma once

#include "eta_common.cuh"

namespace eta {

constexpr int KV4_GROUP = 16;          // channels that share a scale

// Byte offsets inside a block, and its size
struct Kv4Block {
    int k_scales, v_codes, v_scales, bytes;
    __host__ __device__ constexpr Kv4Block(int b, int d)
        : k_scales(b * d / 2), v_codes(b * d / 2 + b * d / KV4_GROUP), v_scales(b * d + b * d / KV4_GROUP),
          bytes(b * d + 2 * (b * d / KV4_GROUP)) {}
};

// -> ETA_OK, or what is wrong with the description of a pool of such blocks
int validate_kv4(const eta_cache_desc* d, const eta_kv4_desc* kv4, const void* pool, bool paged);

#ifdef __CUDACC__

// Eight codes as four fp16 pairs, byte by byte (channel 2 j low, 2 j + 1 high).  The bytes are named in place: a conversion then takes its
// byte itself and costs two cycles of a scheduler, where cutting the byte out first costs four more.
__device__ __forceinline__ void e2m1x8_to_f16x2(uint32_t w, uint32_t (&h)[4]) {
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}
// two fp32 -> a byte of codes, `lo` in the low half: nearest, ties to even, saturating
__device__ __forceinline__ uint32_t f32x2_to_e2m1x2(float lo, float hi) {
    uint32_t r;
    asm("{\n\t.reg .b8 c;\n\tcvt.rn.satfinite.e2m1x2.f32 c, %2, %1;\n\tcvt.u32.u8 %0, c;\n\t}" : "=r"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float f16_lo(uint32_t p) { return __low2float(*reinterpret_cast<const __half2*>(&p)); }
__device__ __forceinline__ float f16_hi(uint32_t p) { return __high2float(*reinterpret_cast<const __half2*>(&p)); }
// the larger of two numbers; a NaN if either is one
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// fp16 pairs held as words
__device__ __forceinline__ uint32_t hmul2_u(uint32_t a, uint32_t b) {
    const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t hfma2_u(uint32_t a, uint32_t b, uint32_t c) {
    const __half2 r = __hfma2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b), *reinterpret_cast<const __half2*>(&c));
    return *reinterpret_cast<const uint32_t*>(&r);
}

#endif  // __CUDACC__
}  // namespace eta
