// Matrices in 8-bit integers with a scale for each row (moe_quantize_int8,
// moe_dequantize_int8): a token's activations, an output channel's weights.
#include "int8.h"

namespace moe {
namespace {

constexpr int THREADS = 256;

// A row by W waves: the maximum, then the codes.  A thread owns the chunks i, i + 64 W, ...; the
// first CH of them stay in registers in between, later ones are read again.  Bound by the memory rate: 16384
// rows of 2048 bf16, 101 MB, in 17.5 us, of fp32, 168 MB, in 31; of few rows by its launch (64 of 4096: 3.6).
template <typename Elem, int V, int CH, int W>
__global__ __launch_bounds__(THREADS) void quantize_int8_kernel(const Elem* __restrict__ x, int64_t rows,
                                                                int cols, int8_t* __restrict__ q,
                                                                float* __restrict__ scales) {
    __shared__ uint32_t red[THREADS / 64];
    constexpr int NT = 64 * W, PER = THREADS / NT;       // threads of a row, rows of a workgroup
    constexpr bool NARROW = sizeof(Elem) == 2;
    const int tid = threadIdx.x % NT;
    const int chunks = cols / V, P = (int)int8_cols(cols);
    for (int64_t r = (int64_t)blockIdx.x * PER + threadIdx.x / NT; r < rows; r += (int64_t)gridDim.x * PER) {
        const Elem* xr = x + r * cols;
        Piece<Elem, V> held[CH];
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < CH; ++i)
            held[i].load(xr + (int64_t)(tid + i * NT < chunks ? tid + i * NT : 0) * V);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            float v[V];
            held[i].values(v);
            most = max(most, magnitude(v));
        }
        for (int c = tid + CH * NT; c < chunks; c += NT) {
            Piece<Elem, V> p;
            float v[V];
            p.load(xr + (int64_t)c * V);
            p.values(v);
            most = max(most, magnitude(v));
        }
        most = lanes_max(most);
        if (W > 1) {
            if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = most;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < W; ++w) most = max(most, red[w]);
            __syncthreads();
        }
        const Int8Scale scale(most);
        if (tid == 0) scales[r] = scale.s;
        int8_t* qr = q + r * P;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = tid + i * NT;
            float v[V];
            held[i].values(v);
            if (c < chunks) scale.template store<NARROW>(v, qr + (int64_t)c * V);
        }
        for (int c = tid + CH * NT; c < chunks; c += NT) {
            Piece<Elem, V> p;
            float v[V];
            p.load(xr + (int64_t)c * V);
            p.values(v);
            scale.template store<NARROW>(v, qr + (int64_t)c * V);
        }
        for (int c = cols + tid; c < P; c += NT) qr[c] = 0;
    }
}

template <typename Elem, int V>
int quantize(const Elem* x, int64_t rows, int cols, int8_t* q, float* scales, hipStream_t s) {
    const int chunks = cols / V;
    const bool wave = chunks <= 64 * 4 && rows >= 1024;
    const int64_t groups = wave ? ceil_div(rows, THREADS / 64) : rows;
    const dim3 grid((unsigned)(groups < 65536 ? groups : 65536));
#define MOE_Q8(CH, W)                                                                               \
    hipLaunchKernelGGL((quantize_int8_kernel<Elem, V, CH, W>), grid, dim3(THREADS), 0, s, x, rows, cols, q, \
                       scales)
    if (wave) {
        if (chunks <= 64) MOE_Q8(1, 1);
        else if (chunks <= 128) MOE_Q8(2, 1);
        else MOE_Q8(4, 1);
    } else {
        if (chunks <= 256) MOE_Q8(1, 4);
        else if (chunks <= 512) MOE_Q8(2, 4);
        else if (chunks <= 1024) MOE_Q8(4, 4);
        else MOE_Q8(8, 4);
    }
#undef MOE_Q8
    return launch_status();
}

// V elements a thread.  Bound by the memory rate (16384 rows of 2048 to bf16: 100 MB in 16 us).
template <typename Elem, int V>
__global__ __launch_bounds__(THREADS) void dequantize_int8_kernel(const int8_t* __restrict__ q,
                                                                  const float* __restrict__ scales,
                                                                  int64_t rows, int cols, int64_t first,
                                                                  Elem* __restrict__ y) {
    const int chunks = cols / V;
    const int64_t i = (first + blockIdx.x) * THREADS + threadIdx.x;
    const int64_t r = i / chunks;
    const int c = (int)(i - r * chunks) * V;
    if (r >= rows) return;
    const float s = scales[r];
    const int8_t* p = q + r * int8_cols(cols) + c;
    float v[V];
    if constexpr (V == 1) {
        v[0] = (float)p[0] * s;
    } else {
        uint32_t w[V / 4];
#pragma unroll
        for (int j = 0; j < V / 4; ++j) w[j] = ((const uint32_t*)p)[j];
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = (float)(int8_t)(w[j / 4] >> (8 * (j % 4))) * s;
    }
    Piece<Elem, V> out;
    out.set(v);
    out.store(y + r * cols + c);
}

template <typename Elem, int V>
int dequantize(const int8_t* q, const float* scales, int64_t rows, int cols, Elem* y, hipStream_t s) {
    return launch_groups(ceil_div(rows * (cols / V), THREADS), THREADS, [&](int64_t first, unsigned n) {
        hipLaunchKernelGGL((dequantize_int8_kernel<Elem, V>), dim3(n), dim3(THREADS), 0, s, q, scales, rows,
                           cols, first, y);
    });
}

bool aligned(const void* p) { return ((uintptr_t)p & 15u) == 0; }

}  // namespace

int launch_quantize_int8(const void* x, int dtype, int64_t rows, int cols, int8_t* q, float* scales,
                         hipStream_t s) {
    if (rows == 0) return MOE_OK;
    if (dtype == MOE_BF16)
        return cols % 8 == 0 && aligned(x) ? quantize<bf16_t, 8>((const bf16_t*)x, rows, cols, q, scales, s)
                                           : quantize<bf16_t, 1>((const bf16_t*)x, rows, cols, q, scales, s);
    return cols % 4 == 0 && aligned(x) ? quantize<float, 4>((const float*)x, rows, cols, q, scales, s)
                                       : quantize<float, 1>((const float*)x, rows, cols, q, scales, s);
}

int launch_dequantize_int8(const int8_t* q, const float* scales, int64_t rows, int cols, int dtype,
                           void* y, hipStream_t s) {
    if (rows == 0) return MOE_OK;
    if (dtype == MOE_BF16)
        return cols % 8 == 0 && aligned(y) ? dequantize<bf16_t, 8>(q, scales, rows, cols, (bf16_t*)y, s)
                                           : dequantize<bf16_t, 1>(q, scales, rows, cols, (bf16_t*)y, s);
    return cols % 4 == 0 && aligned(y) ? dequantize<float, 4>(q, scales, rows, cols, (float*)y, s)
                                       : dequantize<float, 1>(q, scales, rows, cols, (float*)y, s);
}

}  // namespace moe
