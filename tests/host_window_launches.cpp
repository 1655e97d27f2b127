// What the calls of window attention and the paged cache (include/sig_sequence.h) launch, on the CPU: libsig's host code over a HIP runtime of its own, which
// writes launches down instead of running them.  Built and driven by tests/test_host_window_launches.py.
// A call is a line of words and numbers:
//   forward|backward B T HEADS SHARED KEY_DIM VALUE_DIM TYPE WINDOW SINKS
//   append B T HEADS CACHE_HEADS KEY_DIM VALUE_DIM TYPE CACHE_TYPE PAGE_TOKENS TURNED
//   attend B T HEADS CACHE_HEADS KEY_DIM VALUE_DIM TYPE CACHE_TYPE PAGE_TOKENS TABLE_PAGES WINDOW SINKS
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
        const int64_t *lengths = (const int64_t *)p;
        if (what == "forward" || what == "backward") {
            const sig_window_t s = {n[0], n[1], (int32_t)n[2], (int32_t)n[3], (int32_t)n[4], (int32_t)n[5], (int32_t)n[6], 1.0f, n[7], n[8], {}, {}, {}};
            rc = what == "forward" ? sig_window_attention(ctx, &s, p, p, p, lengths, p, p, p, nullptr)
                                   : sig_window_attention_backward(ctx, &s, p, p, p, lengths, p, p, p, p, p, p, p, nullptr);
        } else {
            const bool attend = what == "attend";
            sig_cache_t c = {};
            c.pages = 16;
            c.page_tokens = n[8];
            c.heads = (int32_t)n[3];
            c.key_dim = (int32_t)n[4];
            c.value_dim = (int32_t)n[5];
            c.type = (int32_t)n[7];
            c.keys = c.values = p;
            c.key_scales = c.value_scales = p;
            c.table = (const int32_t *)p;
            c.table_pages = attend ? n[9] : 1;
            if (attend) {
                const sig_queries_t s = {n[0], n[1], (int32_t)n[2], (int32_t)n[6], 1.0f, n[10], n[11], {}};
                rc = sig_cache_attention(ctx, &c, &s, p, lengths, lengths, p, nullptr);
            } else {
                sig_append_t s = {};
                s.B = n[0];
                s.T = n[1];
                s.heads = (int32_t)n[2];
                s.type = (int32_t)n[6];
                s.frequencies = (const double *)p;
                s.turned = n[9];
                s.scale = 1.0;
                rc = sig_cache_append(ctx, &c, &s, p, p, p, lengths, lengths, p, nullptr);
            }
        }
        std::cout << rc << ' ' << most_asked;
        for (const Launched &l : launched) std::cout << ' ' << l.kernel << ',' << l.grid.x << ',' << l.grid.y << ',' << l.grid.z << ',' << l.block.x;
        std::cout << std::endl;
        sig_destroy(ctx);
    }
    return 0;
}
