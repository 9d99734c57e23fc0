// Driver of the launch-error checks of the 4-bit experts and the gradients (test
// infrastructure, no GPU), as launch_main.cpp is of the other calls: the executable defines
// the HIP calls that the library makes, so they take the place of the runtime's, and
// nothing is launched.  Every entry point is called along each branch of its dispatch;
// with all launches succeeding it must return MOE_OK, and with any one of them failing
// MOE_ERR_DEVICE.  As in the runtime, a launch's error stays until hipGetLastError reads
// and clears it.  Prints "launch errors: OK" when every status is the expected one.
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
    const bool empty = grid.x == 0 || grid.y == 0 || grid.z == 0 || block.x == 0;
    if (empty || launches++ == fail_at) return last_error = empty ? 9 : 719;
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
    FN(moe_quantize_mxfp4);
    FN(moe_dequantize_mxfp4);
    FN(moe_mxfp4_lay_out);
    FN(moe_grouped_ffn_mxfp4);
    FN(moe_combine_backward);
    FN(moe_permute_backward);
    FN(moe_route_topk_backward);
#undef FN
    void* F = (void*)0x1000;                 // handed to kernels only, and none runs
    float* f = (float*)F;
    int32_t* i32 = (int32_t*)F;
    uint8_t* u8 = (uint8_t*)F;
    uint32_t* u32 = (uint32_t*)F;
    void* W = (void*)0x100000;
    const size_t big = (size_t)1 << 40;
    const uint8_t* codes[MOE_MAX_GROUPS];
    const uint32_t* scales[MOE_MAX_GROUPS];
    for (auto& p : codes) p = u8;
    for (auto& p : scales) p = u32;

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
        for (int i = 0; i < n; ++i, ++runs) {
            launches = last_error = 0;
            fail_at = i;
            st = call();
            if (st != MOE_ERR_DEVICE) {
                fprintf(stderr, "%s %ld %ld %ld: launch %d of %d failed, status %d\n", what, a, b,
                        c, i, n, st);
                ++failures;
            }
        }
    };

    for (int64_t rows : {1, 777, 30000})
        for (int cols : {1, 100, 1000, 4096})
            for (int dtype : {MOE_F32, MOE_BF16}) {
                check("quantize_mxfp4", rows, cols, dtype, [&] {
                    return moe_quantize_mxfp4_(F, dtype, rows, cols, u8, u8, nullptr);
                });
                check("dequantize_mxfp4", rows, cols, dtype, [&] {
                    return moe_dequantize_mxfp4_(u8, u8, rows, cols, dtype, F, nullptr);
                });
                check("mxfp4_lay_out", rows, cols, dtype, [&] {
                    return moe_mxfp4_lay_out_(u8, u8, rows, cols, u8, u32, nullptr);
                });
            }
    // strips that quantize and strips that do not, wide and narrow; both tile sizes
    for (int64_t T : {1, 9, 16, 33, 128, 129, 600, 5000})
        for (int n : {1, 8, 64})
            for (int d : {64, 2048, 4096})
                for (int ff : {96, 1408, 14336})
                    for (int shared : {0, 2})
                        check("grouped_ffn_mxfp4", T, n, d, [&] {
                            return moe_grouped_ffn_mxfp4_(F, T, i32, i32, n, shared, codes, scales, codes,
                                                          scales, d, ff, 2 * T, F, W, big, nullptr);
                        });
    for (int64_t T : {1, 300, 9000})
        for (int d : {7, 64, 512, 2048, 40000})
            for (int k : {1, 3, 8, 16})
                for (int dtype : {MOE_F32, MOE_BF16})
                    for (float* dgate : {f, (float*)nullptr}) {
                        check("combine_backward", T, d, k, [&] {
                            return moe_combine_backward_(F, F, dtype, i32, f, T, d, k, F, dgate, nullptr);
                        });
                        check("permute_backward", T, d, k, [&] {
                            return moe_permute_backward_(F, dtype, i32, dgate, T, d, k, F, nullptr);
                        });
                    }
    for (int64_t T : {1, 100, 777, 9000})
        for (int E : {8, 30, 60, 128, 250})
            for (int d : {64, 2048})
                for (int dtype : {MOE_F32, MOE_BF16})
                    for (int flags : {0, MOE_RENORM})
                        for (int want = 1; want < 16; ++want)
                            check("route_topk_backward", T, E, want, [&] {
                                return moe_route_topk_backward_(
                                    f, f, i32, f, F, F, dtype, T, d, E, 6, flags, want & 1 ? f : nullptr,
                                    want & 2 ? F : nullptr, want & 4 ? f : nullptr,
                                    want & 8 ? f : nullptr, W, big, nullptr);
                            });
    if (failures) return 1;
    printf("launch errors: OK (%d calls, %d failed launches)\n", calls, runs);
    return 0;
}
