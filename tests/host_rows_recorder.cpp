// The operators on rows (gv_rows_api.cpp and the host side of their kernels' files) without a GPU: the HIP calls that they make
// are defined here and keep what was launched, so that a test can look at it.  Pointers that the calls are given are never read.
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <map>
#include <string>
#include <vector>

#include "gv_host.hpp"
#include "gv_rows.hpp"
#include "gvhot.h"

namespace {

struct Launch {
    std::string kernel;
    uint64_t blocks, threads;
    gv::DenseArgs product;  // of the kernels of a layer's products
};
std::vector<Launch> launches;
std::map<const void *, std::string> &names() {
    static std::map<const void *, std::string> all;
    return all;
}
char text[512];

}  // namespace

int gv::fail_call(int code, const char *fmt, ...) noexcept {
    va_list args;
    va_start(args, fmt);
    vsnprintf(text, sizeof text, fmt, args);
    va_end(args);
    return code;
}

extern "C" {

const char *gv_last_error(const gv_ctx *) { return text; }

void **__hipRegisterFatBinary(const void *) {
    static void *handle;
    return &handle;
}
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *device, int, void *, void *, void *, void *, int *) { names()[host] = device; }
hipError_t __hipPopCallConfiguration(dim3 *, dim3 *, size_t *, hipStream_t *) { return hipErrorUnknown; }
const char *hipGetErrorString(hipError_t) { return "an error"; }
hipError_t hipGetLastError() { return hipSuccess; }

hipError_t hipLaunchKernel(const void *kernel, dim3 blocks, dim3 threads, void **args, size_t, hipStream_t) {
    Launch l{names()[kernel], (uint64_t)blocks.x * blocks.y * blocks.z, threads.x, {}};
    if (l.kernel.find("k_product") != std::string::npos || l.kernel.find("k_join_product") != std::string::npos)
        memcpy(&l.product, args[0], sizeof l.product);
    launches.push_back(l);
    return hipSuccess;
}

// what the tests ask
void recorded_clear() { launches.clear(); }
uint64_t recorded_count() { return launches.size(); }
const char *recorded_kernel(uint64_t i) { return launches[i].kernel.c_str(); }
uint64_t recorded_blocks(uint64_t i) { return launches[i].blocks; }
uint64_t recorded_threads(uint64_t i) { return launches[i].threads; }
// of a product: its rows, its first row in bytes from address 0, and whether it leaves parts to be joined
uint64_t recorded_rows(uint64_t i) { return launches[i].product.rows; }
uint64_t recorded_out(uint64_t i) { return (uint64_t)launches[i].product.out; }
int recorded_cut(uint64_t i) { return launches[i].product.partial != nullptr; }

}  // extern "C"
