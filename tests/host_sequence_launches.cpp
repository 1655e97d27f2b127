// What the calls of include/sig_sequence.h launch, on the CPU: libsig's host code over a HIP runtime of its own, which writes launches
// down instead of running them.  Built and driven by tests/test_host_sequence_launches.py.
// A call is a line of words and numbers, NUMBERS as the entry point takes them:
//   norm|norm_backward ROWS WIDTH TYPE      rotary B T HEADS DIM TURNED TYPE      forward|backward B T HEADS SHARED KEY_DIM VALUE_DIM TYPE
// the answer "STATUS MOST_BYTES kernel,grid.x,grid.y,grid.z,block.x ..." with the most bytes of device memory that it asked for at once.
#include <unistd.h>

#include <algorithm>
#include <cstdint>
#include <cstdlib>
#include <iostream>
#include <map>
#include <sstream>
#include <string>
#include <vector>

#include <hip/hip_runtime_api.h>

#include "sig_sequence.h"

struct Launched { std::string kernel; dim3 grid, block; };
static std::vector<Launched> launched;
static size_t most_asked = 0;
static std::map<const void *, std::string> &kernels()
{
    static std::map<const void *, std::string> names;
    return names;
}
static thread_local dim3 pushed_grid, pushed_block;
static char storage[1 << 16];

extern "C" {
void **__hipRegisterFatBinary(const void *) { static void *handle; return &handle; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *name, unsigned, void *, void *, dim3 *, dim3 *, int *) { kernels()[host] = name; }
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t)
{
    pushed_grid = grid;
    pushed_block = block;
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *stream)
{
    *grid = pushed_grid;
    *block = pushed_block;
    *lds = 0;
    *stream = nullptr;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *host, dim3 grid, dim3 block, void **, size_t, hipStream_t)
{
    launched.push_back({kernels()[host], grid, block});
    return hipSuccess;
}
hipError_t hipGetDevice(int *device) { *device = 0; return hipSuccess; }
hipError_t hipDeviceGetAttribute(int *value, hipDeviceAttribute_t, int) { *value = 256; return hipSuccess; }
hipError_t hipGetSymbolAddress(void **address, const void *) { *address = storage; return hipSuccess; }
hipError_t hipFuncGetAttributes(hipFuncAttributes *attributes, const void *) { *attributes = hipFuncAttributes{}; return hipErrorInvalidValue; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *status) { *status = hipStreamCaptureStatusNone; return hipSuccess; }
hipError_t hipMalloc(void **p, size_t bytes)
{
    most_asked = std::max(most_asked, bytes);
    *p = std::malloc(64);   // (nothing is launched, so nothing writes to it)
    return hipSuccess;
}
hipError_t hipFree(void *p) { std::free(p); return hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
}

int main()
{
    alarm(60);
    static float room[64];   // every pointer of a call: nothing is read or written
    float *p = room;
    for (std::string line; std::getline(std::cin, line);) {
        std::istringstream words(line);
        std::string what;
        words >> what;
        std::vector<int64_t> n;
        for (int64_t value; words >> value;) n.push_back(value);
        sig_ctx *ctx = nullptr;
        if (sig_create(&ctx) != SIG_OK) return 1;
        launched.clear();
        most_asked = 0;
        int rc = -1;
        if (what == "norm") {
            rc = sig_layer_norm(ctx, p, n[1], n[0], n[1], (int)n[2], p, p, SIG_F32, 1e-5, p, p, nullptr);
        } else if (what == "norm_backward") {
            rc = sig_layer_norm_backward(ctx, p, n[1], n[0], n[1], (int)n[2], p, SIG_F32, p, p, n[1], p, p, p, nullptr);
        } else if (what == "rotary") {
            const int64_t places[2] = {0, 1};
            rc = sig_rotary(ctx, p, nullptr, p, nullptr, (int)n[5], n[0], n[1], n[2], n[3], n[4], p, SIG_POSITION_I64, places, (const double *)p, 0, 1.0, 0, nullptr);
        } else {
            sig_attention_t s = {n[0], n[1], (int32_t)n[2], (int32_t)n[3], (int32_t)n[4], (int32_t)n[5], (int32_t)n[6], 1.0f, {}, {}, {}};
            rc = what == "forward" ? sig_linear_attention(ctx, &s, p, p, p, p, p, nullptr, p, p, nullptr)
                                   : sig_linear_attention_backward(ctx, &s, p, p, p, p, p, nullptr, p, p, p, p, p, p, nullptr);
        }
        std::cout << rc << ' ' << most_asked;
        for (const Launched &l : launched) std::cout << ' ' << l.kernel << ',' << l.grid.x << ',' << l.grid.y << ',' << l.grid.z << ',' << l.block.x;
        std::cout << std::endl;
        sig_destroy(ctx);
    }
    return 0;
}
