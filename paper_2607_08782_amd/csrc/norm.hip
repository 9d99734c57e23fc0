// The root-mean-square norm in front of a layer, with the residual's addition and the normed
// rows in 8 bits, and its gradient.
//
//   h = x + residual (as stored),  rstd = 1 / sqrt(mean_i h_i^2 + eps),  y_i = h_i rstd w_i
//
// Both are bound by the memory rate: a row's values are read once, stay in registers over the
// row's reductions, and every output is written from there.  16384 rows of 2048 bf16 with a residual,
// h and codes: 302 MB in 62 us, 4.9 TB/s (a copy of that size: 5.4).  A few rows: 5 us, a launch and
// a row's loads, two reductions and stores in turn.
#include <algorithm>

#include "int8.h"

namespace moe {
namespace {

constexpr int THREADS = 256;

// A row by W waves: by one, with no barrier, where a wave holds it and the rows fill the chip, else by
// a workgroup.  A thread owns the chunks i, i + 64 W, ... of V elements; the first CH stay
// in registers, later ones are read again for each of the three passes (sum of squares,
// largest |y|, outputs).  Pointers may be the same (h over x or residual, y over either).
template <typename Elem, int V, int CH, int W>
__global__ __launch_bounds__(THREADS) void rmsnorm_kernel(const Elem* x, const Elem* residual,
                                                          const Elem* weight, float eps, int64_t T, int d,
                                                          Elem* h, Elem* y, float* rstd, int8_t* q,
                                                          float* scales) {
    __shared__ double sums[THREADS / 64];
    __shared__ uint32_t most[THREADS / 64];
    constexpr int NT = 64 * W, PER = THREADS / NT;
    constexpr bool NARROW = sizeof(Elem) == 2;
    const int tid = threadIdx.x % NT, wave = threadIdx.x >> 6;
    const int chunks = d / V, P = (int)int8_cols(d);
    Piece<Elem, V> w[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) w[i].load(weight + (int64_t)(tid + i * NT < chunks ? tid + i * NT : 0) * V);
    for (int64_t t = (int64_t)blockIdx.x * PER + threadIdx.x / NT; t < T; t += (int64_t)gridDim.x * PER) {
        const int64_t row = t * d;
        Piece<Elem, V> held[CH];
        // (64 bits: no row's sum of squares passes their range)
        double sum = 0.0;
        auto add = [&](Piece<Elem, V>& a, const Piece<Elem, V>& b) {
            float u[V], v[V];
            a.values(u);
            b.values(v);
#pragma unroll
            for (int j = 0; j < V; ++j) u[j] += v[j];
            a.set(u);
        };
        auto square = [&](const Piece<Elem, V>& a) {
            float v[V];
            a.values(v);
#pragma unroll
            for (int j = 0; j < V; ++j) sum = fma((double)v[j], (double)v[j], sum);
        };
        Piece<Elem, V> extra[CH];
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = tid + i * NT < chunks ? tid + i * NT : 0;
            held[i].load(x + row + (int64_t)c * V);
            if (residual != nullptr) extra[i].load(residual + row + (int64_t)c * V);
        }
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = tid + i * NT;
            if (residual != nullptr) add(held[i], extra[i]);
            if (c >= chunks) continue;
            if (residual != nullptr) held[i].store(h + row + (int64_t)c * V);
            square(held[i]);
        }
        for (int c = tid + CH * NT; c < chunks; c += NT) {
            Piece<Elem, V> a, b;
            a.load(x + row + (int64_t)c * V);
            if (residual != nullptr) {
                b.load(residual + row + (int64_t)c * V);
                add(a, b);
                a.store(h + row + (int64_t)c * V);
            }
            square(a);
        }
        sum = lanes_sum(sum);
        if (W > 1) {
            if ((threadIdx.x & 63) == 0) sums[wave] = sum;
            __syncthreads();
            sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
        }
        const float r = (float)(1.0 / sqrt(sum / d + (double)eps));
        if (rstd != nullptr && tid == 0) rstd[t] = r;
        // y of a chunk, rounded as it is stored
        const Elem* stored = residual != nullptr ? h : x;
        auto normed = [&](const Piece<Elem, V>& a, const Piece<Elem, V>& b) {
            float u[V], v[V];
            a.values(u);
            b.values(v);
#pragma unroll
            for (int j = 0; j < V; ++j) u[j] = u[j] * r * v[j];
            Piece<Elem, V> out;
            out.set(u);
            return out;
        };
        auto again = [&](int c) {
            Piece<Elem, V> a, b;
            a.load(stored + row + (int64_t)c * V);
            b.load(weight + (int64_t)c * V);
            return normed(a, b);
        };
#pragma unroll
        for (int i = 0; i < CH; ++i) held[i] = normed(held[i], w[i]);
        uint32_t top = 0;
        if (q != nullptr) {
            float v[V];
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                held[i].values(v);
                if (tid + i * NT < chunks) top = max(top, magnitude(v));
            }
            for (int c = tid + CH * NT; c < chunks; c += NT) {
                again(c).values(v);
                top = max(top, magnitude(v));
            }
            top = lanes_max(top);
        }
        if (W > 1) {
            if ((threadIdx.x & 63) == 0) most[wave] = top;
            __syncthreads();                             // and the sums above are read
            top = max(max(most[0], most[1]), max(most[2], most[3]));
        }
        const Int8Scale scale(top);
        auto put = [&](const Piece<Elem, V>& a, int c) {
            if (q != nullptr) {
                float v[V];
                a.values(v);
                scale.template store<NARROW>(v, q + t * P + (int64_t)c * V);
            }
            if (y != nullptr) a.store(y + row + (int64_t)c * V);
        };
#pragma unroll
        for (int i = 0; i < CH; ++i)
            if (tid + i * NT < chunks) put(held[i], tid + i * NT);
        for (int c = tid + CH * NT; c < chunks; c += NT) put(again(c), c);
        if (q != nullptr) {
            if (tid == 0) scales[t] = scale.s;
            for (int c = d + tid; c < P; c += NT) q[t * P + c] = 0;
        }
    }
}

template <typename Elem, int V>
int rmsnorm(const Elem* x, const Elem* residual, const Elem* weight, float eps, int64_t T, int d, Elem* h,
            Elem* y, float* rstd, int8_t* q, float* scales, hipStream_t s) {
    const int chunks = d / V;
    const bool wave = chunks <= 64 * 4 && T >= 1024;
    const int64_t groups = wave ? ceil_div(T, THREADS / 64) : T;
    const dim3 grid((unsigned)(groups < 65536 ? groups : 65536));
#define MOE_RN(CH, W)                                                                                 \
    hipLaunchKernelGGL((rmsnorm_kernel<Elem, V, CH, W>), grid, dim3(THREADS), 0, s, x, residual, weight, \
                       eps, T, d, h, y, rstd, q, scales)
    if (wave) {
        if (chunks <= 64) MOE_RN(1, 1);
        else if (chunks <= 128) MOE_RN(2, 1);
        else MOE_RN(4, 1);
    } else {
        if (chunks <= 256) MOE_RN(1, 4);
        else if (chunks <= 512) MOE_RN(2, 4);
        else MOE_RN(4, 4);
    }
#undef MOE_RN
    return launch_status();
}

// ---------------------------------------------------------------------------
// The gradient.  With g = dy w and n = h rstd,
//
//   dh = rstd (g - n mean_i(g_i n_i)) + dh_add,     dw = sum_t dy n
//
// A workgroup takes the rows of one of `parts` ranges, in order; W waves share a row, a thread
// its CH chunks of columns in every row, so dw's sums stay in its registers until the range's
// end.  The ranges' sums meet in sum_ranges_kernel, in order.  8192 rows of 2048 bf16 with dh_add: 134 MB
// in 29 us, 4.6 TB/s, and 4 for the sums (512 ranges: the rows' loads need two workgroups a CU to be
// hidden; the next row's loads ahead of a row's sums were no faster).

// dh of rows whose chunks a thread holds, and the range's part of dw (nullable: not wanted).
template <typename Elem, int V, int CH, int W>
__global__ __launch_bounds__(THREADS) void rmsnorm_backward_kernel(
    const Elem* __restrict__ dy, const Elem* __restrict__ h, const Elem* __restrict__ weight,
    const float* __restrict__ rstd, const Elem* dh_add, int64_t T, int d, int64_t per, Elem* dh,
    float* __restrict__ parts) {
    __shared__ float sums[2][THREADS / 64];
    constexpr int NT = 64 * W, PER = THREADS / NT;
    const int tid = threadIdx.x % NT, wave = threadIdx.x >> 6;
    const int chunks = d / V;
    const int64_t begin = blockIdx.x * per, end = min(begin + per, T);
    float acc[CH][V];
    Piece<Elem, V> w[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        w[i].load(weight + (int64_t)(tid + i * NT < chunks ? tid + i * NT : 0) * V);
#pragma unroll
        for (int j = 0; j < V; ++j) acc[i][j] = 0.f;
    }
    int turn = 0;
    for (int64_t t = begin + threadIdx.x / NT; t < end; t += PER, turn ^= 1) {
        Piece<Elem, V> up[CH], at[CH], add[CH];
        const float r = rstd[t];
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int64_t c = t * d + (int64_t)(tid + i * NT < chunks ? tid + i * NT : 0) * V;
            up[i].load(dy + c);
            at[i].load(h + c);
            if (dh_add != nullptr) add[i].load(dh_add + c);
        }
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            if (tid + i * NT >= chunks) continue;
            float u[V], n[V], v[V];
            up[i].values(u);
            at[i].values(n);
            w[i].values(v);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                n[j] *= r;
                dot = fmaf(u[j] * v[j], n[j], dot);
                acc[i][j] = fmaf(u[j], n[j], acc[i][j]);
            }
        }
        if (dh == nullptr) continue;
        dot = lanes_sum(dot);
        if (W > 1) {                                     // (the other half: the row before's)
            if ((threadIdx.x & 63) == 0) sums[turn][wave] = dot;
            __syncthreads();
            dot = (sums[turn][0] + sums[turn][1]) + (sums[turn][2] + sums[turn][3]);
        }
        const float mean = dot / (float)d;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = tid + i * NT;
            if (c >= chunks) continue;
            float u[V], n[V], v[V];
            up[i].values(u);
            at[i].values(n);
            w[i].values(v);
#pragma unroll
            for (int j = 0; j < V; ++j) u[j] = r * fmaf(-n[j] * r, mean, u[j] * v[j]);
            if (dh_add != nullptr) {
                add[i].values(v);
#pragma unroll
                for (int j = 0; j < V; ++j) u[j] += v[j];
            }
            Piece<Elem, V> out;
            out.set(u);
            out.store(dh + t * d + (int64_t)c * V);
        }
    }
    if (parts == nullptr) return;
    // a workgroup's rows in turn: one part for each of its PER row streams
    float* part = parts + ((int64_t)blockIdx.x * PER + threadIdx.x / NT) * d;
#pragma unroll
    for (int i = 0; i < CH; ++i)
        if (tid + i * NT < chunks)
#pragma unroll
            for (int j = 0; j < V; ++j) part[(tid + i * NT) * V + j] = acc[i][j];
}

// Rows of any length (past 4096 columns in fp32, 8192 in bf16, 1024 where a pointer is not 16-byte aligned):
// dh by a workgroup each, which reads them twice, element by element (8192 rows of 5120 fp32 with dh_add,
// 671 MB: 187 us, the parts of dw 73, little over half the rate of the rows above) ...
template <typename Elem>
__global__ __launch_bounds__(THREADS) void rmsnorm_backward_rows_kernel(
    const Elem* __restrict__ dy, const Elem* __restrict__ h, const Elem* __restrict__ weight,
    const float* __restrict__ rstd, const Elem* dh_add, int64_t T, int d, Elem* dh) {
    __shared__ float sums[THREADS / 64];
    for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
        const float r = rstd[t];
        auto at = [&](const Elem* p, int64_t i) {
            Piece<Elem, 1> e;
            float v[1];
            e.load(p + i);
            e.values(v);
            return v[0];
        };
        float dot = 0.f;
        for (int c = threadIdx.x; c < d; c += THREADS)
            dot = fmaf(at(dy, t * d + c) * at(weight, c), at(h, t * d + c) * r, dot);
        dot = lanes_sum(dot);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = dot;
        __syncthreads();
        const float mean = ((sums[0] + sums[1]) + (sums[2] + sums[3])) / (float)d;
        for (int c = threadIdx.x; c < d; c += THREADS) {
            float v[1] = {r * fmaf(-at(h, t * d + c) * r, mean, at(dy, t * d + c) * at(weight, c))};
            if (dh_add != nullptr) v[0] += at(dh_add, t * d + c);
            Piece<Elem, 1> out;
            out.set(v);
            out.store(dh + t * d + c);
        }
    }
}

// ... and a range's part of dw, a column a thread.
template <typename Elem>
__global__ __launch_bounds__(THREADS) void rmsnorm_backward_columns_kernel(
    const Elem* __restrict__ dy, const Elem* __restrict__ h, const float* __restrict__ rstd, int64_t T,
    int d, int64_t per, int columns, float* __restrict__ parts) {
    const int64_t range = blockIdx.x / columns;
    const int c = (int)(blockIdx.x % columns) * THREADS + threadIdx.x;
    if (c >= d) return;
    float sum = 0.f;
    for (int64_t t = range * per; t < min(range * per + per, T); ++t) {
        Piece<Elem, 1> a, b;
        float u[1], n[1];
        a.load(dy + t * d + c);
        b.load(h + t * d + c);
        a.values(u);
        b.values(n);
        sum = fmaf(u[0], n[0] * rstd[t], sum);
    }
    parts[range * d + c] = sum;
}

// dw[c] = the sum of the ranges' parts in 64 bits, by slices of them that are joined in a fixed order;
// eight of a slice's parts in flight (2048 columns of 512 parts, one after the other by 16 slices: 9.4 us;
// so 4; 16 columns a workgroup even).  In 32 bits dw was off by 1.5e-7 for 8192 rows, so by 8e-8.
constexpr int JOIN = 1024, COLS = 32, SLICES = JOIN / COLS;

__global__ __launch_bounds__(JOIN) void sum_ranges_kernel(const float* __restrict__ parts, int64_t n, int d,
                                                          float* __restrict__ dw) {
    __shared__ double s[JOIN / 64][COLS];
    constexpr int AHEAD = 8;
    const int slice = threadIdx.x / COLS, col = threadIdx.x % COLS;
    const int64_t c = (int64_t)blockIdx.x * COLS + col;
    double v = 0.0;
    if (c < d)
        for (int64_t q0 = slice; q0 < n; q0 += SLICES * AHEAD) {
            float a[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) a[i] = q0 + i * SLICES < n ? parts[(q0 + i * SLICES) * d + c] : 0.f;
            // (without this the compiler converts, and waits, under each load's condition)
            asm volatile("" : "+v"(a[0]), "+v"(a[1]), "+v"(a[2]), "+v"(a[3]), "+v"(a[4]), "+v"(a[5]), "+v"(a[6]), "+v"(a[7]));
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) v += (double)a[i];
        }
    // slices side by side in a wave, then the waves'
#pragma unroll
    for (int o = COLS; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
    if ((threadIdx.x & 63) < COLS) s[threadIdx.x >> 6][col] = v;
    __syncthreads();
    if (slice > 0 || c >= d) return;
    double sum[2] = {0.0, 0.0};
#pragma unroll
    for (int q = 0; q < JOIN / 64; ++q) sum[q % 2] += s[q][col];
    dw[c] = (float)(sum[0] + sum[1]);
}

// Ranges of the rows, and of each how many: as many as fill the chip, several rows each.
struct Ranges {
    int64_t n, per;
    explicit Ranges(int64_t T) {
        per = std::max<int64_t>(ceil_div(T, 512), 4);
        n = std::max<int64_t>(ceil_div(T, per), 1);
    }
};

constexpr int BACK_CH = 4;

template <typename Elem, int V>
int rmsnorm_backward(const Elem* dy, const Elem* h, const Elem* weight, const float* rstd,
                     const Elem* dh_add, int64_t T, int d, Elem* dh, float* dw, float* parts,
                     hipStream_t s) {
    const Ranges ranges(T);
    const int chunks = d / V;
    int64_t n = ranges.n;
    int st = MOE_OK;
    if (T == 0) {
        n = 0;                                           // dw is zero
    } else if (chunks <= THREADS * BACK_CH) {
        const dim3 grid((unsigned)ranges.n);
#define MOE_RB(CH, W)                                                                              \
    hipLaunchKernelGGL((rmsnorm_backward_kernel<Elem, V, CH, W>), grid, dim3(THREADS), 0, s, dy, h,   \
                       weight, rstd, dh_add, T, d, ranges.per, dh, dw ? parts : nullptr)
        if (chunks <= 64) {
            MOE_RB(1, 1);
            n *= 4;
        } else if (chunks <= 128) {
            MOE_RB(2, 1);
            n *= 4;
        } else if (chunks <= 256) {
            MOE_RB(1, 4);
        } else if (chunks <= 512) {
            MOE_RB(2, 4);
        } else {
            MOE_RB(4, 4);
        }
#undef MOE_RB
        st = launch_status();
    } else {
        if (dh != nullptr) {
            hipLaunchKernelGGL(rmsnorm_backward_rows_kernel<Elem>, dim3((unsigned)std::min<int64_t>(T, 65536)),
                               dim3(THREADS), 0, s, dy, h, weight, rstd, dh_add, T, d, dh);
            st = launch_status();
        }
        if (st == MOE_OK && dw != nullptr) {
            const int columns = (int)ceil_div(d, THREADS);
            // (512 ranges of 2^14 blocks of columns at most: one grid)
            hipLaunchKernelGGL(rmsnorm_backward_columns_kernel<Elem>, dim3((unsigned)(ranges.n * columns)),
                               dim3(THREADS), 0, s, dy, h, rstd, T, d, ranges.per, columns, parts);
            st = launch_status();
        }
    }
    if (st != MOE_OK || dw == nullptr) return st;
    hipLaunchKernelGGL(sum_ranges_kernel, dim3((unsigned)ceil_div(d, COLS)), dim3(JOIN), 0, s, parts, n, d, dw);
    return launch_status();
}

bool aligned(const void* p) { return ((uintptr_t)p & 15u) == 0; }

}  // namespace

int launch_rmsnorm(const void* x, const void* residual, int dtype, const void* weight, float eps,
                   int64_t T, int d, void* h, void* y, float* rstd, int8_t* q, float* scales,
                   hipStream_t s) {
    if (T == 0) return MOE_OK;
    const bool whole = aligned(x) && aligned(residual) && aligned(weight) && aligned(h) && aligned(y);
#define MOE_RN(E, V)                                                                                  \
    rmsnorm<E, V>((const E*)x, (const E*)residual, (const E*)weight, eps, T, d, (E*)h, (E*)y, rstd, q, \
                  scales, s)
    if (dtype == MOE_BF16) return whole && d % 8 == 0 ? MOE_RN(bf16_t, 8) : MOE_RN(bf16_t, 1);
    return whole && d % 4 == 0 ? MOE_RN(float, 4) : MOE_RN(float, 1);
#undef MOE_RN
}

size_t rmsnorm_backward_ws_bytes(int, int64_t T, int d) {
    return (size_t)(Ranges(T).n * 4 * d * 4) + 256;
}

int launch_rmsnorm_backward(const void* dy, const void* h, int dtype, const void* weight,
                            const float* rstd, const void* dh_add, int64_t T, int d, void* dh,
                            float* dw, void* ws, hipStream_t s) {
    if ((!dh && !dw) || (T == 0 && !dw)) return MOE_OK;
    const bool whole = aligned(dy) && aligned(h) && aligned(weight) && aligned(dh_add) && aligned(dh);
#define MOE_RB(E, V)                                                                                   \
    rmsnorm_backward<E, V>((const E*)dy, (const E*)h, (const E*)weight, rstd, (const E*)dh_add, T, d,     \
                           (E*)dh, dw, (float*)ws, s)
    if (dtype == MOE_BF16) return whole && d % 8 == 0 ? MOE_RB(bf16_t, 8) : MOE_RB(bf16_t, 1);
    return whole && d % 4 == 0 ? MOE_RB(float, 4) : MOE_RB(float, 1);
#undef MOE_RB
}

}  // namespace moe
