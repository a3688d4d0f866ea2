// A HIP runtime that records the launches of the 8-bit rows' kernels instead of
// making them: linked with the host half of csrc/q8_kernels.hip, so that what
// each launch is handed is checked without a GPU.  Allocations of the host code
// fail on request.
#include <cstdint>
#include <cstdlib>
#include <map>
#include <new>
#include <string>
#include <vector>

#include <hip/hip_runtime_api.h>

#include "q8_kernels.h"

namespace {

long allocations_left = -1;   // before one fails (negative: none does)

std::map<const void *, std::string> names;

// A launch: its rows, and where the first of them lies in the arrays; list is a
// weight gradient's number of slices.
struct Launch {
    int64_t rows, in, scales, out, list;
};
std::vector<Launch> launches;

struct Call {
    dim3 grid, block;
    size_t lds;
    hipStream_t stream;
} pending;

// Places of the arguments in a kernel's list: input, scales, output, row list
// (-1: none), slices.
struct Kernel {
    const char *name;
    int in, scales, out, list, slices;
};
constexpr Kernel kernels[] = {
    {"k_quantize_rows", 2, 8, 6, 4, 0},   {"k_dequantize_rows", 2, 4, 7, 5, 0},
    {"k_dequantize_flat", 3, 5, 8, 6, 0}, {"k_q8_fewI", 3, 5, 10, -1, 0},
    {"k_q8_gemm", 4, 6, 11, -1, 0},       {"k_q8_stream", 3, 5, 10, -1, 0},
    {"k_q8_gradI", 7, 9, 14, -1, 4},
};

}  // namespace

void *operator new(size_t n)
{
    if (allocations_left >= 0 && allocations_left-- == 0)
        throw std::bad_alloc();
    if (void *p = std::malloc(n ? n : 1))
        return p;
    throw std::bad_alloc();
}
void operator delete(void *p) noexcept { std::free(p); }
void operator delete(void *p, size_t) noexcept { std::free(p); }

extern "C" {

void fail_allocation(long after) { allocations_left = after; }

extern const char __hip_fatbin[8];
const char __hip_fatbin[8] = {};
void **__hipRegisterFatBinary(const void *) { return nullptr; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *name, unsigned, void *,
                           void *, void *, void *, int *)
{
    names[host] = name;
}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream)
{
    pending = {grid, block, lds, stream};
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *stream)
{
    *grid = pending.grid, *block = pending.block, *lds = pending.lds, *stream = pending.stream;
    return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipLaunchKernel(const void *f, dim3 grid, dim3 block, void **args, size_t, hipStream_t)
{
    // (a grid's threads are counted in 32 bits, its other sides in 16)
    if (!grid.x || (uint64_t)grid.x * block.x > UINT32_MAX || grid.y > 65535 || block.x > 1024)
        return hipErrorInvalidConfiguration;
    for (const Kernel &k : kernels)
        if (names[f].find(k.name) != std::string::npos) {
            auto at = [&](int i) { return *(const int64_t *)args[i]; };
            launches.push_back({*(const int32_t *)args[0], at(k.in), at(k.scales), at(k.out),
                                k.slices     ? *(const int32_t *)args[k.slices]
                                : k.list < 0 ? 0
                                             : (int64_t)((const digest::RowList *)args[k.list])->p});
            return hipSuccess;
        }
    if (names[f].find("k_q8_grad_few") != std::string::npos ||
        names[f].find("k_q8_grad_sum") != std::string::npos)
        return hipSuccess;
    return hipErrorInvalidDeviceFunction;
}

// The launches since the last call, five numbers each; how many there were.
int recorded_launches(int64_t *out, int most)
{
    const int n = (int)launches.size();
    for (int i = 0; i < n && i < most; ++i) {
        const Launch &l = launches[i];
        const int64_t v[5] = {l.rows, l.in, l.scales, l.out, l.list};
        for (int j = 0; j < 5; ++j)
            out[5 * i + j] = v[j];
    }
    launches.clear();
    return n;
}

}  // extern "C"
