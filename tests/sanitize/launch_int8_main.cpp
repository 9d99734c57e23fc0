// Driver of the launch checks of the 8-bit experts, the norm, the balance loss and the clipping (test
// infrastructure, no GPU), as launch_main.cpp is of the other calls: the executable defines the HIP
// calls that the library makes, so they take the place of the runtime's, and nothing is launched.
// Every entry point is called along each branch of its dispatch, and at the largest sizes that it
// accepts; with all launches succeeding it must return MOE_OK, and with any one of them failing
// MOE_ERR_DEVICE.  A launch larger than a grid holds fails, as in the runtime.  Prints "launch errors:
// OK" when every status is the expected one.
#include <dlfcn.h>
#include <stdint.h>
#include <stdio.h>

#include <functional>
#include <vector>

#include "moe.h"

static int launches, fail_at = -1, last_error;

struct Dim3 {
    uint32_t x, y, z;
};
static Dim3 grid_, block_;

extern "C" {
// the launch shape between a <<< >>> and its kernel's host stub
int __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t, void*) {
    grid_ = grid;
    block_ = block;
    return 0;
}
int __hipPopCallConfiguration(Dim3* grid, Dim3* block, size_t* lds, void** stream) {
    *grid = grid_;
    *block = block_;
    *lds = 0;
    *stream = nullptr;
    return 0;
}
int hipLaunchKernel(const void*, Dim3 grid, Dim3 block, void**, size_t, void*) {
    const bool holds = grid.x && grid.y && grid.z && block.x && (uint64_t)grid.x * block.x < 1ull << 32 &&
                       grid.y <= 65535 && grid.z <= 65535;
    if (!holds || launches++ == fail_at) return last_error = holds ? 719 : 9;
    return 0;
}
int hipGetLastError() {
    const int e = last_error;
    last_error = 0;
    return e;
}
int hipGetDevice(int* d) {
    *d = 0;
    return 0;
}
int hipDeviceGetAttribute(int* v, int, int) {
    *v = 256;
    return 0;
}
int hipFuncSetAttribute(const void*, int, int) { return 0; }
int hipGetSymbolAddress(void** p, const void*) {
    *p = (void*)0x100000;
    return 0;
}
}

int main(int argc, char** argv) {
    void* lib = dlopen(argc > 1 ? argv[1] : "", RTLD_NOW);
    if (!lib) {
        fprintf(stderr, "%s\n", dlerror());
        return 1;
    }
#define FN(name) auto name##_ = (decltype(&name))dlsym(lib, #name)
    FN(moe_quantize_int8);
    FN(moe_dequantize_int8);
    FN(moe_grouped_ffn_int8);
    FN(moe_rmsnorm);
    FN(moe_rmsnorm_backward);
    FN(moe_balance_loss);
    FN(moe_balance_loss_backward);
    FN(moe_grad_norm);
    FN(moe_clip_grads);
    FN(moe_route_topk_backward_aux);
#undef FN
    void* F = (void*)0x1000;                 // handed to kernels only, and none runs
    void* O = (void*)0x1002;                 // aligned for bf16 alone
    float* f = (float*)F;
    int32_t* i32 = (int32_t*)F;
    int8_t* i8 = (int8_t*)F;
    void* W = (void*)0x100000;
    const size_t big = (size_t)1 << 50;
    const int8_t* codes[MOE_MAX_GROUPS];
    const float* scales[MOE_MAX_GROUPS];
    for (auto& p : codes) p = i8;
    for (auto& p : scales) p = f;

    int failures = 0, calls = 0, runs = 0;
    auto check = [&](const char* what, long a, long b, long c, const std::function<int()>& call) {
        launches = last_error = 0;
        fail_at = -1;
        int st = call();
        const int n = launches;
        ++calls;
        if (st != MOE_OK || n == 0) {
            fprintf(stderr, "%s %ld %ld %ld: status %d after %d launches\n", what, a, b, c, st, n);
            ++failures;
        }
        // (of many launches alike the first ones and the last)
        for (int i = 0; i < n; ++i, ++runs) {
            if (i == 8 && n > 9) i = n - 1;
            launches = last_error = 0;
            fail_at = i;
            st = call();
            if (st != MOE_ERR_DEVICE) {
                fprintf(stderr, "%s %ld %ld %ld: launch %d of %d failed, status %d\n", what, a, b, c, i, n, st);
                ++failures;
            }
        }
    };

    for (int64_t rows : {(int64_t)1, (int64_t)777, (int64_t)30000, (int64_t)1 << 29})
        for (int cols : {1, 100, 1000, 4096, 20000})
            for (int dtype : {MOE_F32, MOE_BF16}) {
                check("quantize_int8", rows, cols, dtype,
                      [&] { return moe_quantize_int8_(F, dtype, rows, cols, i8, f, nullptr); });
                check("dequantize_int8", rows, cols, dtype,
                      [&] { return moe_dequantize_int8_(i8, f, rows, cols, dtype, F, nullptr); });
            }
    // strips that quantize, strips of both widths and in slices, tiles of both sizes and in slices
    for (int64_t T : {1, 2, 9, 16, 33, 64, 65, 600, 5000})
        for (int n : {1, 8, 64})
            for (int d : {64, 2048, 4096})
                for (int ff : {96, 1408, 4100, 14336})
                    for (int shared : {0, 2})
                        check("grouped_ffn_int8", T, n, d, [&] {
                            return moe_grouped_ffn_int8_(i8, f, T, i32, i32, n, shared, codes, scales, codes, scales, d,
                                                         ff, 2 * T, F, W, big, nullptr);
                        });
    check("grouped_ffn_int8 rows", 1 << 24, 8, 8, [&] {
        return moe_grouped_ffn_int8_(i8, f, 1 << 23, i32, i32, 8, 0, codes, scales, codes, scales, 8, 8, 0x7fffffff,
                                     F, W, big, nullptr);
    });
    check("grouped_ffn_int8 widths", 1, 1 << 17, 1 << 13, [&] {
        return moe_grouped_ffn_int8_(i8, f, 1, i32, i32, 128, 0, codes, scales, codes, scales, 1 << 13, (1 << 17) - 8,
                                     128, F, W, big, nullptr);
    });
    for (int64_t T : {(int64_t)1, (int64_t)300, (int64_t)9000, (int64_t)0x7fffffff})
        for (int d : {7, 64, 512, 2048, 4096, 40000, (1 << 22) - 1})
            for (int dtype : {MOE_F32, MOE_BF16})
                for (void* x : {F, dtype == MOE_BF16 ? O : F}) {
                    check("rmsnorm", T, d, dtype, [&] {
                        return moe_rmsnorm_(x, F, dtype, F, 1e-6f, T, d, (void*)0x2000, (void*)0x3000, f, i8, f,
                                            nullptr);
                    });
                    for (int want = 1; want < 4; ++want)
                        check("rmsnorm_backward", T, d, want, [&] {
                            return moe_rmsnorm_backward_(x, F, dtype, F, f, F, T, d, want & 1 ? F : nullptr,
                                                         want & 2 ? f : nullptr, W, big, nullptr);
                        });
                }
    check("rmsnorm_backward of no rows", 0, 64, 0, [&] {
        return moe_rmsnorm_backward_(nullptr, nullptr, MOE_BF16, nullptr, nullptr, nullptr, 0, 64, nullptr, f, W, big,
                                     nullptr);
    });
    for (int64_t T : {(int64_t)0, (int64_t)1, (int64_t)100, (int64_t)777, (int64_t)90000, (int64_t)0x7fffffff})
        for (int E : {1, 8, 9, 16, 30, 60, 128, 250})
            for (float* at : {f, (float*)0x1004}) {
                check("balance_loss", T, E, 1, [&] {
                    return moe_balance_loss_(at, i32, nullptr, T, E, 1, i32, f, i32, f, W, big, nullptr);
                });
                if (T > 0)
                    check("balance_loss_backward", T, E, 1, [&] {
                        return moe_balance_loss_backward_(at, nullptr, i32, i32, T, E, 1, 1.0f, f, nullptr);
                    });
            }
    for (int n : {1, 96, 97, 300})
        for (int64_t size : {(int64_t)1, (int64_t)100000, (int64_t)1 << 38}) {
            std::vector<const void*> in(n, F);
            std::vector<void*> out(n, F);
            std::vector<int64_t> sizes(n, size);
            std::vector<int> types(n);
            for (int i = 0; i < n; ++i) types[i] = i % 2;
            check("grad_norm", n, size, 0, [&] {
                return moe_grad_norm_(in.data(), sizes.data(), types.data(), n, f, W, big, nullptr);
            });
            check("clip_grads", n, size, 0, [&] {
                return moe_clip_grads_(in.data(), sizes.data(), types.data(), n, f, 1.0f, out.data(), nullptr);
            });
        }
    for (int64_t T : {1, 100, 777})
        for (int E : {8, 60, 250})
            for (int dtype : {MOE_F32, MOE_BF16})
                for (int flags : {0, MOE_RENORM})
                    for (int want = 1; want < 16; ++want)
                        check("route_topk_backward_aux", T, E, want, [&] {
                            return moe_route_topk_backward_aux_(f, f, i32, f, f, F, F, dtype, T, 64, E, 6, flags,
                                                                want & 1 ? f : nullptr, want & 2 ? F : nullptr,
                                                                want & 4 ? f : nullptr, want & 8 ? f : nullptr, W,
                                                                big, nullptr);
                        });
    if (failures) return 1;
    printf("launch errors: OK (%d calls, %d failed launches)\n", calls, runs);
    return 0;
}
