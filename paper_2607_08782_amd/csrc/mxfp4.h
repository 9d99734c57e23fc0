// MXFP4 blocks (E2M1 elements, one E8M0 scale per 32) inside kernels: encoding of a
// block that four lanes hold between them, eight values each.
#pragma once

#include "common.h"

namespace moe {

constexpr int MX_BLOCK = 32;

__host__ __device__ constexpr int64_t mx_cols(int64_t cols) { return (cols + 127) / 128 * 128; }

// E2M1 codes of eight values whose magnitudes are below 8, the first in the low bits:
// round to nearest, ties to even, 6 at most (v_cvt_scalef32_pk_fp4_f32).
__device__ __forceinline__ uint32_t e2m1x8(const float* v) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], 1.0f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], 1.0f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], 1.0f, 3);
    return w;
}

// Scale byte of a block from the bits of its largest magnitude (above every finite
// value's where it holds an infinity or a NaN: byte 255).
__device__ __forceinline__ uint32_t mx_byte(uint32_t most) {
    const int e = (int)(most >> 23);
    return e == 255 ? 255u : (uint32_t)max(e - 2, 0);
}

// 2^(127 - b): takes a block's values below 8.  Zero for b = 255, whose codes are zero
// (an infinity or NaN times it still gives NaN, which mx_encode8 drops).
__device__ __forceinline__ float mx_factor(uint32_t b) {
    return b == 255u ? 0.f : __uint_as_float((254u - b) << 23);
}

// 2^(b - 127), NaN for 255
__device__ __forceinline__ float mx_scale(uint32_t b) {
    return b == 255u ? __uint_as_float(0x7fc00000u) : b == 0u ? __uint_as_float(1u << 22)
                                                              : __uint_as_float(b << 23);
}

__device__ __forceinline__ uint32_t magnitude8(const float* v) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    return m;
}

// Codes of eight values v of a block whose largest magnitude has the bits `most`.
__device__ __forceinline__ uint32_t mx_encode8(float* v, uint32_t most, uint32_t& byte) {
    byte = mx_byte(most);
    const float s = mx_factor(byte);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= s;
    const uint32_t w = e2m1x8(v);
    return byte == 255u ? 0u : w;
}

// The largest of a value over the lane's quad (every lane of it active).
__device__ __forceinline__ uint32_t quad_max(uint32_t m) {
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 0xf, 0xf, false));
    return max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4e, 0xf, 0xf, false));
}

[[nodiscard]]
int launch_quantize_mxfp4(const void* x, int dtype, int64_t rows, int cols, uint8_t* codes,
                          uint8_t* scales, hipStream_t s);
[[nodiscard]]
int launch_dequantize_mxfp4(const uint8_t* codes, const uint8_t* scales, int64_t rows, int cols,
                            int dtype, void* y, hipStream_t s);
// step-major codes [P / 128][rows][64] and scale words [P / 128][rows] (moe_mxfp4_lay_out), of
// a row-major MXFP4 matrix or straight from the quantization of bf16 rows (cols % 8 == 0,
// 16-byte aligned)
[[nodiscard]]
int launch_mxfp4_lay_out(const uint8_t* codes, const uint8_t* scales, int64_t rows, int cols,
                         uint8_t* steps, uint32_t* words, hipStream_t s);
[[nodiscard]]
int launch_quantize_mxfp4_steps(const bf16_t* x, int64_t rows, int cols, uint8_t* codes,
                                uint32_t* words, hipStream_t s);

// Grouped FFN of MXFP4 experts (ffn_mxfp4.hip): n_groups groups in all, the first `lead` of
// lead_rows rows each; `rows`: rows of all groups at most.
size_t grouped_ffn_mxfp4_ws_bytes(int64_t T, int64_t rows, int d, int f);
[[nodiscard]]
int launch_grouped_ffn_mxfp4(const void* x, int64_t T, const int32_t* row_token,
                             const int32_t* offsets, int n_groups, int lead, int lead_rows,
                             const uint8_t* const* w13, const uint32_t* const* s13,
                             const uint8_t* const* w2, const uint32_t* const* s2, int d, int f,
                             int64_t rows, void* y, void* ws, hipStream_t s);

}  // namespace moe
