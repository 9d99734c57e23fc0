// Driver of the launch-size checks (test infrastructure, no GPU): as in launch_main.cpp the
// executable defines the HIP calls that the library makes, and nothing is launched.  The entry
// points of one group are called at the largest sizes that they accept; every launch must
// keep to what a HIP grid holds: fewer than 2^32 work-items and, past the first dimension, at
// most 65535 workgroups.  As in the runtime a launch past that is an error.  Prints "launch
// sizes: OK" when every call returns MOE_OK.
#include <dlfcn.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <functional>

#include "moe.h"

struct Dim3 {
    uint32_t x, y, z;
};
static Dim3 grid_, block_;
static int launches, last_error;

extern "C" {
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
int hipLaunchKernel(const void*, Dim3 g, Dim3 b, void**, size_t, void*) {
    ++launches;
    const bool holds = g.x && g.y && g.z && (uint64_t)g.x * b.x < 1ull << 32 &&
                       (uint64_t)g.y * b.y < 1ull << 32 && g.y <= 65535 && g.z <= 65535;
    return holds ? 0 : (last_error = 9);
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
    if (argc < 3) return 2;
    void* lib = dlopen(argv[1], RTLD_NOW);
    if (!lib) {
        fprintf(stderr, "%s\n", dlerror());
        return 1;
    }
    const char* group = argv[2];
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
    const size_t big = (size_t)1 << 62;
    const uint8_t* codes[MOE_MAX_GROUPS];
    const uint32_t* scales[MOE_MAX_GROUPS];
    for (auto& p : codes) p = u8;
    for (auto& p : scales) p = u32;

    int failures = 0, calls = 0;
    auto check = [&](const char* what, int64_t a, int64_t b, int64_t c, const std::function<int()>& call) {
        launches = last_error = 0;
        const int st = call();
        ++calls;
        if (st != MOE_OK || launches == 0) {
            fprintf(stderr, "%s %lld %lld %lld: status %d after %d launches\n", what, (long long)a,
                    (long long)b, (long long)c, st, launches);
            ++failures;
        }
    };
    const int64_t most = 0x7fffffff;
    if (!strcmp(group, "mxfp4")) {
        for (int cols : {1, 8, 128, 1000, (1 << 28) - 1})
            for (int dtype : {MOE_F32, MOE_BF16}) {
                const int64_t rows = most * 8192 / MOE_MXFP4_COLS(cols);
                check("quantize_mxfp4", rows, cols, dtype, [&] {
                    return moe_quantize_mxfp4_(F, dtype, rows, cols, u8, u8, nullptr);
                });
                check("dequantize_mxfp4", rows, cols, dtype, [&] {
                    return moe_dequantize_mxfp4_(u8, u8, rows, cols, dtype, F, nullptr);
                });
                check("mxfp4_lay_out", most * 32, cols, 0, [&] {
                    return moe_mxfp4_lay_out_(u8, u8, most * 32, cols, u8, u32, nullptr);
                });
            }
        for (int64_t T : {(int64_t)1 << 24, ((int64_t)1 << 25) - 1})
            for (int d : {8, (1 << 21) - 8})
                for (int ff : {1, 32, (1 << 21) - 1})
                    for (const int32_t* rows : {(const int32_t*)i32, (const int32_t*)nullptr})
                        for (int64_t cap : {(int64_t)1, T})
                            for (int n : {1, MOE_MAX_GROUPS})
                                check("grouped_ffn_mxfp4", T, d, ff, [&] {
                                    return moe_grouped_ffn_mxfp4_(F, T, rows, i32, n, 0, codes, scales, codes, scales,
                                                                  d, ff, cap, F, W, big, nullptr);
                                });
        for (int n : {1, MOE_MAX_GROUPS})
            for (int64_t cap : {16, 128})
                check("grouped_ffn_mxfp4 strips", n, cap, 0, [&] {
                    return moe_grouped_ffn_mxfp4_(F, 128, i32, i32, n, 0, codes, scales, codes, scales, (1 << 21) - 8,
                                                  (1 << 21) - 1, cap, F, W, big, nullptr);
                });
    } else if (!strcmp(group, "gradients")) {
        for (int64_t T : {(int64_t)1 << 24, most})
            for (int d : {1, 8, 513, 2048, 2049, 8192})
                for (int dtype : {MOE_F32, MOE_BF16})
                    check("combine_backward", T, d, dtype, [&] {
                        return moe_combine_backward_(F, F, dtype, i32, f, T, d, 2, F, f, nullptr);
                    });
        // T and d together as far as one call takes them
        struct {
            int64_t T;
            int d;
        } sizes[] = {{most, 64}, {128 * 32767, (1 << 22) - 8}, {1, (1 << 22) - 8}, {1, (1 << 22) - 1}};
        for (auto s : sizes)
            for (int E : {1, 250, 256})
                for (int dtype : {MOE_F32, MOE_BF16})
                    for (int flags : {0, MOE_RENORM})
                        if (dtype == MOE_F32 || s.d % 8 == 0)
                            check("route_topk_backward", s.T, s.d, E, [&] {
                                return moe_route_topk_backward_(f, f, i32, f, F, F, dtype, s.T, s.d, E, 1, flags, f, F,
                                                                f, f, W, big, nullptr);
                            });
    } else if (!strcmp(group, "packaging")) {
        for (int64_t T : {(int64_t)1 << 26, most})
            for (int d : {1, 8, 512, 2049, 4096})
                for (int dtype : {MOE_F32, MOE_BF16})
                    check("permute_backward", T, d, dtype, [&] {
                        return moe_permute_backward_(F, dtype, i32, F, T, d, 2, F, nullptr);
                    });
    } else {
        return 2;
    }
    if (failures) return 1;
    printf("launch sizes: OK (%d calls)\n", calls);
    return 0;
}
