// allow_smem of csrc/esp_moe_launch.cuh against a fake cudaFuncSetAttribute (no GPU): whatever a call needs and however
// two threads meet, a kernel's limit is its greatest amount once the function has returned.

#include <condition_variable>
#include <cstdio>
#include <mutex>
#include <thread>

#include "esp_moe_launch.cuh"

namespace {

constexpr size_t kMost = 72 * 1024;
void first() {}
void second() {}

std::mutex mu;
std::condition_variable cv;
int limit = 0, calls = 0, inside = 0;
bool meet = false, refuse = false;

}  // namespace

extern "C" cudaError_t cudaFuncSetAttribute(const void *, cudaFuncAttribute attr, int v)
{
    std::unique_lock<std::mutex> l(mu);
    ++calls;
    if (attr != cudaFuncAttributeMaxDynamicSharedMemorySize || refuse)
        return cudaErrorInvalidValue;
    limit = v;
    ++inside;
    cv.notify_all();
    if (meet)   // both threads are here before either returns
        cv.wait(l, [] { return inside == 2; });
    return cudaSuccess;
}

extern "C" cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t *, const void *, void **) { return cudaSuccess; }

int main()
{
    using esp_moe_impl::allow_smem;
    refuse = true;
    if (allow_smem<first, kMost>(0) == cudaSuccess)
        return printf("a refusal is lost\n"), 1;
    refuse = false;
    if (allow_smem<first, kMost>(0) != cudaSuccess || limit != (int)kMost || calls != 2)
        return printf("the limit is not set after a refusal\n"), 1;
    if (allow_smem<first, kMost>(0) != cudaSuccess || calls != 2)
        return printf("the limit is set again\n"), 1;
    if (allow_smem<first, kMost>(1) != cudaSuccess || calls != 3)
        return printf("another device has a limit of its own\n"), 1;
    meet = true;
    inside = 0;
    limit = 0;
    std::thread a([] { allow_smem<second, kMost>(0); }), b([] { allow_smem<second, kMost>(0); });
    a.join();
    b.join();
    if (limit != (int)kMost)
        return printf("two threads leave a limit of %d\n", limit), 1;
    printf("ok\n");
    return 0;
}
