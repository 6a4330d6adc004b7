// Which kernel a product goes to (test infrastructure): the library's own launch code with a stand-in for the HIP runtime that
// notes launches instead of making them.  Reads lines "tokens k n bf16" and prints "kernel workgroups tiles" for each, after a line "have
// kernel" for every product kernel that is built.  Pointers are plain addresses, never dereferenced.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstdio>
#include <map>
#include <string>

#include "leapquant.h"
#include "lq_internal.hpp"

namespace {
std::map<const void *, std::string> &names() {
    static std::map<const void *, std::string> n;
    return n;
}
struct Launch {
    dim3 grid, block;
    size_t lds;
    hipStream_t stream;
} launch;
}  // namespace

extern "C" {
void **__hipRegisterFatBinary(const void *) {
    static void *module;
    return &module;
}
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *name, unsigned, void *, void *, void *, void *, int *) { names()[host] = name; }
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream) {
    launch = {grid, block, lds, stream};
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *stream) {
    *grid = launch.grid;
    *block = launch.block;
    *lds = launch.lds;
    *stream = launch.stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *host, dim3 grid, dim3, void **args, size_t, hipStream_t) {
    const std::string &name = names()[host];
    const unsigned groups = grid.x * grid.y;
    // (the tiled kernel's arguments: ..., its tiles of tokens and of channels)
    const bool tiled = name.find("product_kernel") != std::string::npos;
    std::printf("%s %u %u\n", name.c_str(), groups, tiled ? (unsigned)(*(int *)args[1] * *(int *)args[2]) : groups);
    return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
}

int main() {
    for (const auto &n : names()) std::printf("have %s\n", n.second.c_str());
    long long tokens;
    int k, n, bf16;
    while (std::scanf("%lld %d %d %d", &tokens, &k, &n, &bf16) == 4) {
        lq_matmul m = {};
        m.tokens = tokens;
        m.n = n;
        m.k = k;
        m.out_dtype = bf16 ? LQ_TOKEN_BF16 : LQ_TOKEN_F32;
        m.x_stride = m.w_stride = k;
        m.x_scale_stride = (k + 127) / 128;
        m.out_stride = (n + 7) / 8 * 8;
        m.x = m.w = m.out = (void *)0x10000;
        m.x_scale = m.w_scale = (const float *)0x10000;
        if (lq::launch_matmul(m, nullptr) != hipSuccess) return 1;
    }
    return 0;
}
