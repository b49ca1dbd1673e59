// Two host threads raise a kernel's shared-memory limit to different sizes for the first time, in the one order in
// which an unlocked record would end above the limit: both have seen that nothing is recorded; the larger size is
// set, then the smaller one; the smaller is recorded, then the larger.  The two runtime calls are stand-ins, so no device
// is needed.  Prints the limit and the record's effect; exits 0 if a size that needs no further call fits the limit.
#include <chrono>
#include <cstdarg>
#include <cstdio>
#include <thread>

#include <cuda_runtime.h>

static cudaError_t get_device(int *dev);
static cudaError_t set_attribute(void (*)(int), cudaFuncAttribute, int value);
#define cudaGetDevice get_device
#define cudaFuncSetAttribute set_attribute
#include "gs_attn.cuh"

namespace gs {
void set_error(const char *, ...) {}
gs_status cuda_fail(cudaError_t, const char *) { return GS_ERR_CUDA; }
}  // namespace gs

static constexpr int SMALL = 60 * 1024, LARGE = 100 * 1024;
static std::atomic<int> limit{0}, calls{0};
static std::atomic<bool> large_set{false}, small_done{false};

static void wait_for(const std::atomic<bool> &flag)        // at most 300 ms
{
    for (int i = 0; i < 300 && !flag; ++i) std::this_thread::sleep_for(std::chrono::milliseconds(1));
}

static cudaError_t get_device(int *dev)
{
    *dev = 0;
    return cudaSuccess;
}
static cudaError_t set_attribute(void (*)(int), cudaFuncAttribute, int value)
{
    ++calls;
    if (value == LARGE) {
        limit = value;
        large_set = true;
        wait_for(small_done);
    } else if (value == SMALL) {
        wait_for(large_set);
        limit = value;
    } else {
        limit = value;
    }
    return cudaSuccess;
}

static void kernel(int) {}

int main()
{
    static gs::SharedRecord record;
    std::thread a([] {
        gs::allow_shared(&kernel, SMALL, record);
        small_done = true;
    });
    std::thread b([] { gs::allow_shared(&kernel, LARGE, record); });
    a.join();
    b.join();
    const int before = calls;
    const gs_status s = gs::allow_shared(&kernel, LARGE - 1024, record);
    std::printf("limit %d, calls %d then %d, status %d\n", limit.load(), before, calls.load(), (int)s);
    return s == GS_OK && limit >= LARGE - 1024 ? 0 : 1;
}
