// 4-bit values of a cache: sixteen channels of a token and head share an 8-bit scale s (e4m3: 4 bits of exponent, 3 of fraction); a value is s times a code (e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6
// and their negatives), so it has at most six significant bits and is exact in fp16 (2^-10 to 2688) and bf16 (contract: specdec.h).
#pragma once
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/specdec.h"

namespace sd {

constexpr int FP4_BLOCK = 16, FP4_MIN_PAGE = 16;          // channels of a scale; tokens of a page: copies of a page's codes and scales are whole 16-byte pieces

// Eight codes (channel 2 i in the low half of byte i) as four pairs of fp16.
__device__ __forceinline__ void fp4_unpack8(uint32_t w, uint32_t* o) {
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}" : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3]) : "r"(w));
}
// The codes nearest to four, eight numbers, ties to the even one, beyond 6 that of 6.  (By sixteen bits: with nvcc 12.9.86 four bytes of codes joined in one move came out as zeros in some kernels.)
__device__ __forceinline__ uint32_t fp4_pack4(float x, float y, float z, float w) {
    uint16_t o;
    asm("{\n\t.reg .b8 a, b;\n\tcvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\tmov.b16 %0, {a, b};\n\t}" : "=h"(o) : "f"(x), "f"(y), "f"(z), "f"(w));
    return o;
}
__device__ __forceinline__ uint32_t fp4_pack8(const float* x) { return fp4_pack4(x[0], x[1], x[2], x[3]) | fp4_pack4(x[4], x[5], x[6], x[7]) << 16; }
// Two scales (low byte first) as fp16; the scale nearest to a number >= 0, at most 448.
__device__ __forceinline__ uint32_t fp4_scales2(uint32_t two) {
    uint32_t o;
    asm("{\n\t.reg .b16 t;\n\tcvt.u16.u32 t, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, t;\n\t}" : "=r"(o) : "r"(two));
    return o;
}
__device__ __forceinline__ uint32_t fp4_scale_of(float x) {
    uint16_t o;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(o) : "f"(0.f), "f"(x));
    return o & 0xff;
}
__device__ __forceinline__ uint32_t h2_mul(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// What keeps this from being a cache in 4 bits (nullptr: nothing).
inline const char* fp4_why_not(const specdec_packed_cache* f) {
    if (!f) return "a pointer is NULL";
    const specdec_cache* c = &f->codes;
    if (!c->d_kv || !f->d_scales || !c->d_table || !c->d_length || !c->d_status) return "a pointer is NULL";
    if (c->dtype != SPECDEC_DTYPE_FP4) return "the codes' dtype is not SPECDEC_DTYPE_FP4";
    if (c->n_layers < 1 || c->n_heads < 1 || c->n_pages < 1 || c->n_seqs < 1 || c->max_pages < 1) return "a size is below 1";
    if (c->head_dim != 64 && c->head_dim != 128) return "head_dim is neither 64 nor 128";
    if (c->page_tokens < FP4_MIN_PAGE || (c->page_tokens & (c->page_tokens - 1))) return "page_tokens is not a power of two of at least 16";
    if ((long long)c->max_pages * c->page_tokens > 0x7fffffffLL - 65536) return "a sequence could pass 2^31 tokens";
    if (((uintptr_t)c->d_kv | (uintptr_t)f->d_scales) & 15) return "d_kv or d_scales is not 16-byte aligned";
    if ((uintptr_t)f->d_unit & 3) return "d_unit is not aligned to its type";
    const long long st[8] = {c->n_layers > 1 ? c->stride_layer : 0, c->stride_side, c->n_pages > 1 ? c->stride_page : 0, c->n_heads > 1 ? c->stride_head : 0,
                             c->n_layers > 1 ? f->scale_stride_layer : 0, f->scale_stride_side, c->n_pages > 1 ? f->scale_stride_page : 0, c->n_heads > 1 ? f->scale_stride_head : 0};
    for (long long s : st) if (s < 0 || s % 16) return "a stride is negative or not a multiple of 16 bytes";
    return nullptr;
}

}  // namespace sd
