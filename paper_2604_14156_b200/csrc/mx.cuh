// Blocks of 32 elements under a shared power of two (the OCP microscaling layouts mxfp4 and mxfp8): what the quantiser, the norm and the FFN
// on such operands (mx_quant.cu, mx_norm.cu, mx_ffn.cu) share.
//
// A block with largest magnitude amax has the scale 2^e, e the smallest integer >= -127 with amax <= M 2^e, M the
// largest finite element (e2m1: 6 = 1.5 2^2, e4m3: 448 = 1.75 2^8), stored as the byte e + 127.  No element saturates, so an element is off by
// half a step of its own type at most.  All of it is integer work on amax's bits: with exponent field E and
// fraction F the byte is E - 2 + (F > .5) for e2m1 and E - 8 + (F > .75) for e4m3, never below 0.  A block that holds a NaN or
// an infinity gets the byte 255, which stands for NaN.
#pragma once

#include "cs_internal.cuh"

namespace cs {

constexpr int kMxBlock = 32;
constexpr int kMxTileBytes = 512;   // scales of 128 rows x 4 blocks: byte [row % 32][row / 32][block % 4]

// The scale byte of a block whose largest magnitude has these bits (sign bit clear).
template <bool E4M3> __host__ __device__ __forceinline__ uint32_t mx_scale_byte(uint32_t amax) {
    const int E = (int)(amax >> 23), F = (int)(amax & 0x7fffff);
    if (E == 255) return 255;
    const int c = E4M3 ? E - 8 + (F > 0x600000) : E - 2 + (F > 0x400000);
    return c > 0 ? (uint32_t)c : 0u;
}
// 2^-e of a scale byte below 254.  (255, a block of NaN: 0 here, so that its codes are zeros of either sign.)
__device__ __forceinline__ float mx_inverse(uint32_t byte) { return byte == 255 ? 0.f : __uint_as_float((254 - byte) << 23); }
// 2^e of any scale byte.
__device__ __forceinline__ float mx_scale(uint32_t byte) {
    return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7fffffffu : byte << 23);
}
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Eight floats as e2m1 codes, the first in the lowest four bits.
__device__ __forceinline__ uint32_t pack_e2m1(const float (&v)[8]) {
    uint32_t r;
    asm("{\n.reg .b8 a, b, c, d;\n"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n"
        "mov.b32 %0, {a, b, c, d};\n}"
        : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
// Four floats as e4m3 bytes, the first in the lowest.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
    uint32_t r;
    asm("{\n.reg .b16 lo, hi;\n"
        "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n"
        "cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n"
        "mov.b32 %0, {lo, hi};\n}" : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
    return r;
}

// silu(gate) up = gate up / (1 + 2^t), t = -gate log2 e, by the bare approximate exponential (2^-22) and reciprocal (2^-23).  t in one f32 is off by up to
// 2^-19 at 2^6, and the exponential by as much of itself, so 2^t is corrected by what t lost: with the roundings of the sum and the two products
// less than 2^-20 of the result, against the 2^-4 of the rounding that follows.  Clamped where 2^t is below 2^-128, or above 2^126, whose reciprocal counts
// as 0 (gates below -87.3): so that nothing overflows in between.  A NaN comes back through the last product.
__device__ __forceinline__ float swiglu(float gate, float up) {
    const float x = fminf(fmaxf(-gate, -89.f), 88.f), t = 1.44269502f * x;
    const float lost = fmaf(x, 1.92596299e-8f, fmaf(x, 1.44269502f, -t));
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(t));
    e = fmaf(e * 0.693147181f, lost, e);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    return gate * r * up;
}
// max(m, |v|), NaN where either is.
__device__ __forceinline__ float max_abs(float m, float v) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(m), "f"(fabsf(v)));
    return r;
}

// mx_norm.cu
cs_status prepare_mx_norm();
cs_status launch_mx_norm(cs_plan *plan, const void *x, int x_dtype, const void *delta, int delta_dtype, const float *gamma, int B,
                         void *x_out, float *n_out, uint8_t *q, uint8_t *s, cudaStream_t st);
// mx_ffn.cu: support [B, k], or with `shared` [k]
cs_status prepare_mx_ffn(cs_plan *plan);
constexpr int kMxDoneOffset = 32;                    // mx_done: the next item in a line of its own, then a count for each token tile, then one of pairs
inline size_t mx_done_bytes(const cs_plan *plan) { return (kMxDoneOffset + ((size_t)plan->cfg.max_tokens + 255) / 256 + 1) * sizeof(unsigned); }
size_t mx_wide_partial_bytes(const cs_plan *plan);   // mx_wide.cu's scratch for parts of an output
cs_status launch_mx_ffn(cs_plan *plan, const cs_mx_layer *L, const uint8_t *q, const uint8_t *s, const int32_t *support, bool shared,
                        int B, void *out, cudaStream_t st);

}  // namespace cs
