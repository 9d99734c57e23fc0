// Rows in 8-bit integers with a scale each: the scale and the codes of a row, as kernels that
// hold a row's values make them.
#pragma once

#include "common.h"

namespace moe {

// Bytes of a row: its columns padded with zeros to whole steps of the products.
__host__ __device__ constexpr int64_t int8_cols(int64_t cols) { return (cols + 127) / 128 * 128; }

// Longest sum of products: 2^17 of them, at most 127 x 127 each, stay below 2^31.
constexpr int INT8_MAX_K = 1 << 17;

// Elements as loaded in one chunk of V.
template <typename Elem, int V>
struct Piece;
template <>
struct Piece<bf16_t, 8> {
    uint4 u;
    __device__ __forceinline__ void load(const bf16_t* p) { u = *(const uint4*)p; }
    __device__ __forceinline__ void values(float (&v)[8]) const {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void set(const float (&v)[8]) {
        u = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                       pack_bf16x2(v[6], v[7]));
    }
    __device__ __forceinline__ void store(bf16_t* p) const { *(uint4*)p = u; }
};
template <>
struct Piece<float, 4> {
    float4 u;
    __device__ __forceinline__ void load(const float* p) { u = *(const float4*)p; }
    __device__ __forceinline__ void values(float (&v)[4]) const {
        v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
    }
    __device__ __forceinline__ void set(const float (&v)[4]) { u = make_float4(v[0], v[1], v[2], v[3]); }
    __device__ __forceinline__ void store(float* p) const { *(float4*)p = u; }
};
template <>
struct Piece<bf16_t, 1> {
    bf16_t u;
    __device__ __forceinline__ void load(const bf16_t* p) { u = *p; }
    __device__ __forceinline__ void values(float (&v)[1]) const { v[0] = bf16_to_f32(u); }
    __device__ __forceinline__ void set(const float (&v)[1]) { u = f32_to_bf16(v[0]); }
    __device__ __forceinline__ void store(bf16_t* p) const { *p = u; }
};
template <>
struct Piece<float, 1> {
    float u;
    __device__ __forceinline__ void load(const float* p) { u = *p; }
    __device__ __forceinline__ void values(float (&v)[1]) const { v[0] = u; }
    __device__ __forceinline__ void set(const float (&v)[1]) { u = v[0]; }
    __device__ __forceinline__ void store(float* p) const { *p = u; }
};

// Bits of the largest magnitude of V values: above every finite value's for an infinity or NaN.
template <int V>
__device__ __forceinline__ uint32_t magnitude(const float (&v)[V]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    return m;
}

// A row's scale: max |x| / 127 (the fp32 division), 2^-126 at least, so that no code's
// quotient overflows, and NaN for a row that is not finite, whose codes are zero.
struct Int8Scale {
    float s, y;                                          // the scale, 1 / scale rounded
    bool finite, fast;                                   // fast: quotients by y lose no bits

    __device__ __forceinline__ explicit Int8Scale(uint32_t most) {
        finite = most < 0x7f800000u;
        s = finite ? fmaxf(__fdiv_rn(__uint_as_float(most), 127.0f), 0x1p-126f)
                   : __uint_as_float(0x7fc00000u);
        y = __fdiv_rn(1.0f, s);
        fast = s > 0x1p-60f && s < 0x1p60f;
    }

    // Codes of up to four values, the first in the low byte.  The quotient is RN(v / s): y is
    // 1 / s correctly rounded, and a residual step by fma on v y gives the correctly rounded
    // quotient (Markstein's theorem) when that is within an ulp, which a first such step makes
    // sure of; of values with eight significant bits (NARROW) the first step already gives it.
    // Adding 3 2^22 rounds it to a whole number, ties to even, whose low byte is the code.
    template <bool NARROW, int N>
    __device__ __forceinline__ uint32_t codes(const float* v) const {
        if (!finite) return 0;
        uint32_t b[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float q;
            if (fast) {
                q = v[i] * y;
                q = fmaf(fmaf(-q, s, v[i]), y, q);
                if (!NARROW) q = fmaf(fmaf(-q, s, v[i]), y, q);
            } else {
                q = __fdiv_rn(v[i], s);
            }
            b[i] = __float_as_uint(q + 12582912.0f);
        }
        if constexpr (N == 1) return b[0] & 0xffu;
        else {
            const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u);
            const uint32_t hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000c0cu);
            return lo | hi;
        }
    }

    // Codes of a chunk, stored.
    template <bool NARROW, int V>
    __device__ __forceinline__ void store(const float (&v)[V], int8_t* p) const {
        if constexpr (V == 8)
            *(uint2*)p = make_uint2(codes<NARROW, 4>(v), codes<NARROW, 4>(v + 4));
        else if constexpr (V == 4)
            *(uint32_t*)p = codes<NARROW, 4>(v);
        else
            *p = (int8_t)codes<NARROW, 1>(v);
    }
};

// A value over the wave's lanes: the sum, the same order in each, and the largest.
template <typename F>
__device__ __forceinline__ F lanes_sum(F v) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
    return v;
}

__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
    return v;
}

[[nodiscard]]
int launch_quantize_int8(const void* x, int dtype, int64_t rows, int cols, int8_t* q, float* scales,
                         hipStream_t s);
[[nodiscard]]
int launch_dequantize_int8(const int8_t* q, const float* scales, int64_t rows, int cols, int dtype,
                           void* y, hipStream_t s);

size_t grouped_ffn_int8_ws_bytes(int64_t rows, int d, int f, int n_groups);
// n_groups groups in all, the first `lead` of lead_rows rows each; rows: of all groups at most
[[nodiscard]]
int launch_grouped_ffn_int8(const int8_t* xq, const float* x_scale, int64_t T,
                            const int32_t* row_token, const int32_t* offsets, int n_groups, int lead,
                            int lead_rows, const int8_t* const* w13, const float* const* s13,
                            const int8_t* const* w2, const float* const* s2, int d, int f,
                            int64_t rows, void* y, void* ws, hipStream_t s);

[[nodiscard]]
int launch_rmsnorm(const void* x, const void* residual, int dtype, const void* weight, float eps,
                   int64_t T, int d, void* h, void* y, float* rstd, int8_t* q, float* scales,
                   hipStream_t s);
size_t rmsnorm_backward_ws_bytes(int dtype, int64_t T, int d);
[[nodiscard]]
int launch_rmsnorm_backward(const void* dy, const void* h, int dtype, const void* weight,
                            const float* rstd, const void* dh_add, int64_t T, int d, void* dh,
                            float* dw, void* ws, hipStream_t s);

size_t balance_loss_ws_bytes(int64_t T, int E);
[[nodiscard]]
int launch_balance_loss(const float* logits, const int32_t* idx, const uint8_t* mask, int64_t T, int E,
                        int k, int32_t* counts, float* prob_sum, int32_t* n_tokens, float* loss,
                        void* ws, hipStream_t s);
[[nodiscard]]
int launch_balance_loss_backward(const float* logits, const uint8_t* mask, const int32_t* counts,
                                 const int32_t* n_tokens, int64_t T, int E, int k, float scale,
                                 float* dlogits, hipStream_t s);

int64_t grad_chunks(const int64_t* sizes, int n);
[[nodiscard]]
int launch_grad_norm(const void* const* grads, const int64_t* sizes, const int* dtypes, int n,
                     float* norm, void* ws, hipStream_t s);
[[nodiscard]]
int launch_clip_grads(const void* const* grads, const int64_t* sizes, const int* dtypes, int n,
                      const float* norm, float max_norm, void* const* out, hipStream_t s);

}  // namespace moe
