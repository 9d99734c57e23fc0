// A matrix to MXFP4 and back (the format of moe.h): for every block of 32 columns the
// scale 2^(b - 127), b = max(exponent of the largest |x| - 2, 0), and E2M1 codes of
// x 2^(127 - b).
//
// Bound by the memory rate: 2 or 4 bytes a value on one side, 17/32 on the other.  A
// thread takes eight columns (16 or 32 bytes in, 4 out), so a block is a quad of lanes
// and its largest magnitude two DPP moves; MX_UNROLL such pieces per thread are loaded
// before the first is used.  Codes and scales are dense over the padded rows: piece i
// is always code word i and quad i / 4 scale byte i / 4, and only the matrix itself
// needs a piece's row and column (not even that where rows need no padding).
#include "mxfp4.h"

#include <algorithm>

namespace moe {
namespace {

constexpr int MX_THREADS = 256;
constexpr int MX_UNROLL = 4;
constexpr int MX_PIECES = MX_THREADS * MX_UNROLL;        // per workgroup

template <typename T>
struct Elem;
template <>
struct Elem<bf16_t> {
    static __device__ __forceinline__ void load8(const bf16_t* p, float* v) {
        const uint4 u = *(const uint4*)p;
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ float load(const bf16_t* p) { return bf16_to_f32(*p); }
    static __device__ __forceinline__ void store8(bf16_t* p, const float* v) {
        *(uint4*)p = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    }
    static __device__ __forceinline__ void store(bf16_t* p, float v) { *p = f32_to_bf16(v); }
};
template <>
struct Elem<float> {
    static __device__ __forceinline__ void load8(const float* p, float* v) {
        const float4 a = ((const float4*)p)[0], b = ((const float4*)p)[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
    static __device__ __forceinline__ float load(const float* p) { return *p; }
    static __device__ __forceinline__ void store8(float* p, const float* v) {
        ((float4*)p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        ((float4*)p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
    static __device__ __forceinline__ void store(float* p, float v) { *p = v; }
};

// How a matrix's pieces are reached: rows of a multiple of 128 columns, one after the
// other; of a multiple of 8, with vectors; any other width (or address), by element.
enum Form { DENSE, PADDED, ELEMENTS };

// Row and first column of the workgroup's pieces, from one division per workgroup and a
// 32-bit one per piece.
struct Place {
    int64_t row0;
    uint32_t first, per_row;
    __device__ __forceinline__ Place(int64_t base, int cols) {
        per_row = (uint32_t)(mx_cols(cols) / 8);
        row0 = base / per_row;
        first = (uint32_t)(base - row0 * per_row);
    }
    __device__ __forceinline__ int64_t at(int j, int cols, int& col) const {
        const uint32_t o = first + (uint32_t)j, r = o / per_row;
        col = (int)(o - r * per_row) * 8;
        return (row0 + r) * cols + col;
    }
};

template <typename T, Form F>
__global__ __launch_bounds__(MX_THREADS) void quantize_mxfp4_kernel(const T* __restrict__ x, int64_t first,
                                                                    int64_t pieces, int cols,
                                                                    uint32_t* __restrict__ codes,
                                                                    uint8_t* __restrict__ scales) {
    const int64_t base = (first + blockIdx.x) * MX_PIECES;
    const Place place(base, cols);
    float v[MX_UNROLL][8];
#pragma unroll
    for (int u = 0; u < MX_UNROLL; ++u) {
        const int j = u * MX_THREADS + threadIdx.x;
        // a piece past the last, or wholly in the padding, is zeros (quads stay whole:
        // their blocks' pieces end together)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[u][i] = 0.f;
        if (base + j >= pieces) continue;
        if (F == DENSE) {
            Elem<T>::load8(x + (base + j) * 8, v[u]);
            continue;
        }
        int col;
        const int64_t at = place.at(j, cols, col);
        if (F == PADDED) {
            if (col < cols) Elem<T>::load8(x + at, v[u]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (col + i < cols) v[u][i] = Elem<T>::load(x + at + i);
        }
    }
#pragma unroll
    for (int u = 0; u < MX_UNROLL; ++u) {
        const int64_t i = base + u * MX_THREADS + threadIdx.x;
        uint32_t byte;
        const uint32_t most = quad_max(magnitude8(v[u]));
        const uint32_t w = mx_encode8(v[u], most, byte);
        if (i < pieces) {
            codes[i] = w;
            if ((threadIdx.x & 3) == 0) scales[i >> 2] = (uint8_t)byte;
        }
    }
}

// Token rows, step-major: a row per workgroup (and 2048 columns of it), so that no piece
// needs a division, and a short batch is spread over the chip.
__global__ __launch_bounds__(MX_THREADS) void quantize_steps_kernel(const bf16_t* __restrict__ x,
                                                                    int64_t first, int64_t rows, int cols,
                                                                    uint32_t* __restrict__ codes,
                                                                    uint8_t* __restrict__ scales) {
    const int64_t row = first + blockIdx.x;
    const int piece = blockIdx.y * MX_THREADS + threadIdx.x;
    if (piece >= (int)(mx_cols(cols) / 8)) return;       // whole quads
    float v[8] = {};
    if (piece * 8 < cols) Elem<bf16_t>::load8(x + row * cols + piece * 8, v);
    uint32_t byte;
    const uint32_t most = quad_max(magnitude8(v));
    const uint32_t w = mx_encode8(v, most, byte);
    const int64_t at = (piece >> 4) * rows + row;
    codes[at * 16 + (piece & 15)] = w;
    if ((threadIdx.x & 3) == 0) scales[at * 4 + ((piece >> 2) & 3)] = (uint8_t)byte;
}

template <typename T, Form F>
__global__ __launch_bounds__(MX_THREADS) void dequantize_mxfp4_kernel(
    const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t first,
    int64_t pieces, int cols, T* __restrict__ y) {
    const int64_t base = (first + blockIdx.x) * MX_PIECES;
    const Place place(base, cols);
    uint32_t w[MX_UNROLL], byte[MX_UNROLL];
#pragma unroll
    for (int u = 0; u < MX_UNROLL; ++u) {
        const int64_t i = base + u * MX_THREADS + threadIdx.x;
        w[u] = i < pieces ? codes[i] : 0u;
        byte[u] = i < pieces ? scales[i >> 2] : 0u;
    }
#pragma unroll
    for (int u = 0; u < MX_UNROLL; ++u) {
        const int j = u * MX_THREADS + threadIdx.x;
        if (base + j >= pieces) continue;
        const float s = mx_scale(byte[u]);
        float v[8];
        const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], 1.0f, 0);
        const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], 1.0f, 1);
        const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], 1.0f, 2);
        const auto e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], 1.0f, 3);
        v[0] = a[0] * s; v[1] = a[1] * s; v[2] = b[0] * s; v[3] = b[1] * s;
        v[4] = c[0] * s; v[5] = c[1] * s; v[6] = e[0] * s; v[7] = e[1] * s;
        if (F == DENSE) {
            Elem<T>::store8(y + (base + j) * 8, v);
            continue;
        }
        int col;
        const int64_t at = place.at(j, cols, col);
        if (F == PADDED) {
            if (col < cols) Elem<T>::store8(y + at, v);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (col + i < cols) Elem<T>::store(y + at + i, v[i]);
        }
    }
}

// [rows][steps] -> [steps][rows], of 64-byte code pieces and of scale words: blocks of 32
// rows x 8 steps, so that reads are 512 contiguous bytes and writes 2 KB.
constexpr int LAY_ROWS = 32, LAY_STEPS = 8, LAY_THREADS = 256;

__global__ __launch_bounds__(LAY_THREADS) void lay_out_kernel(const uint4* __restrict__ codes,
                                                      const uint32_t* __restrict__ scales,
                                                      int64_t first, int64_t rows, int n,
                                                      uint4* __restrict__ steps,
                                                      uint32_t* __restrict__ words) {
    __shared__ uint4 piece[LAY_ROWS][LAY_STEPS * 4 + 1];
    __shared__ uint32_t word[LAY_ROWS][LAY_STEPS + 1];
    const int64_t r0 = (first + blockIdx.x) * LAY_ROWS;
    const int tid = threadIdx.x;
    for (int s0 = blockIdx.y * LAY_STEPS; s0 < n; s0 += gridDim.y * LAY_STEPS) {
        for (int i = tid; i < LAY_ROWS * LAY_STEPS * 4; i += LAY_THREADS) {
            const int r = i / (LAY_STEPS * 4), c = i % (LAY_STEPS * 4);
            if (r0 + r < rows && s0 + c / 4 < n) piece[r][c] = codes[(r0 + r) * n * 4 + s0 * 4 + c];
        }
        {
            const int r = tid / LAY_STEPS, c = tid % LAY_STEPS;
            if (r0 + r < rows && s0 + c < n) word[r][c] = scales[(r0 + r) * n + s0 + c];
        }
        __syncthreads();
        for (int i = tid; i < LAY_ROWS * LAY_STEPS * 4; i += LAY_THREADS) {
            const int c = i / (LAY_ROWS * 4), r = i % (LAY_ROWS * 4) / 4, q = i % 4;
            if (r0 + r < rows && s0 + c < n)
                steps[((int64_t)(s0 + c) * rows + r0 + r) * 4 + q] = piece[r][c * 4 + q];
        }
        {
            const int c = tid / LAY_ROWS, r = tid % LAY_ROWS;
            if (r0 + r < rows && s0 + c < n) words[(int64_t)(s0 + c) * rows + r0 + r] = word[r][c];
        }
        __syncthreads();
    }
}

Form form_of(const void* p, int cols) {
    if (cols % 8 || ((uintptr_t)p & 15u)) return ELEMENTS;
    return cols % 128 ? PADDED : DENSE;
}

template <typename T>
int quantize(const T* x, int64_t rows, int cols, uint8_t* codes, uint8_t* scales, hipStream_t s) {
    const int64_t pieces = rows * (mx_cols(cols) / 8);
    const Form form = form_of(x, cols);
    return launch_groups(ceil_div(pieces, MX_PIECES), MX_THREADS, [&](int64_t first, unsigned groups) {
#define MOE_MXQ(F)                                                                             \
    hipLaunchKernelGGL((quantize_mxfp4_kernel<T, F>), dim3(groups), dim3(MX_THREADS), 0, s, x, \
                       first, pieces, cols, (uint32_t*)codes, scales)
        switch (form) {
            case DENSE: MOE_MXQ(DENSE); break;
            case PADDED: MOE_MXQ(PADDED); break;
            default: MOE_MXQ(ELEMENTS); break;
        }
#undef MOE_MXQ
    });
}

template <typename T>
int dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int cols, T* y,
               hipStream_t s) {
    const int64_t pieces = rows * (mx_cols(cols) / 8);
    const Form form = form_of(y, cols);
    return launch_groups(ceil_div(pieces, MX_PIECES), MX_THREADS, [&](int64_t first, unsigned groups) {
#define MOE_MXD(F)                                                                          \
    hipLaunchKernelGGL((dequantize_mxfp4_kernel<T, F>), dim3(groups), dim3(MX_THREADS), 0,  \
                       s, (const uint32_t*)codes, scales, first, pieces, cols, y)
        switch (form) {
            case DENSE: MOE_MXD(DENSE); break;
            case PADDED: MOE_MXD(PADDED); break;
            default: MOE_MXD(ELEMENTS); break;
        }
#undef MOE_MXD
    });
}

}  // namespace

int launch_quantize_mxfp4(const void* x, int dtype, int64_t rows, int cols, uint8_t* codes,
                          uint8_t* scales, hipStream_t s) {
    if (rows == 0) return MOE_OK;
    return dtype == MOE_BF16 ? quantize((const bf16_t*)x, rows, cols, codes, scales, s)
                             : quantize((const float*)x, rows, cols, codes, scales, s);
}

int launch_quantize_mxfp4_steps(const bf16_t* x, int64_t rows, int cols, uint8_t* codes,
                                uint32_t* words, hipStream_t s) {
    if (rows == 0) return MOE_OK;
    const unsigned along = (unsigned)ceil_div(mx_cols(cols) / 8, MX_THREADS);
    return launch_groups(rows, MX_THREADS, [&](int64_t first, unsigned groups) {
        hipLaunchKernelGGL(quantize_steps_kernel, dim3(groups, along), dim3(MX_THREADS), 0, s, x, first, rows,
                           cols, (uint32_t*)codes, (uint8_t*)words);
    });
}

int launch_mxfp4_lay_out(const uint8_t* codes, const uint8_t* scales, int64_t rows, int cols,
                         uint8_t* steps, uint32_t* words, hipStream_t s) {
    if (rows == 0) return MOE_OK;
    const int n = (int)(mx_cols(cols) / 128);
    const unsigned along = (unsigned)std::min(ceil_div(n, LAY_STEPS), (int64_t)65535);
    return launch_groups(ceil_div(rows, LAY_ROWS), LAY_THREADS, [&](int64_t first, unsigned groups) {
        hipLaunchKernelGGL(lay_out_kernel, dim3(groups, along), dim3(LAY_THREADS), 0, s, (const uint4*)codes,
                           (const uint32_t*)scales, first, rows, n, (uint4*)steps, words);
    });
}

int launch_dequantize_mxfp4(const uint8_t* codes, const uint8_t* scales, int64_t rows, int cols,
                            int dtype, void* y, hipStream_t s) {
    if (rows == 0) return MOE_OK;
    return dtype == MOE_BF16 ? dequantize(codes, scales, rows, cols, (bf16_t*)y, s)
                             : dequantize(codes, scales, rows, cols, (float*)y, s);
}

}  // namespace moe
