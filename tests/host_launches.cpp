// host_runtime.cpp with more for a test to see and to set: what launches are handed, how much memory is held, an allocation that fails,
// the current device.
#define hipMalloc plain_hipMalloc
#define hipLaunchKernel plain_hipLaunchKernel
#define hipGetDevice plain_hipGetDevice
#define hipSetDevice plain_hipSetDevice
#define hipDeviceSynchronize plain_hipDeviceSynchronize
#include "host_runtime.cpp"
#undef hipMalloc
#undef hipLaunchKernel
#undef hipGetDevice
#undef hipSetDevice
#undef hipDeviceSynchronize

#include <vector>

namespace {
size_t kept_bytes = 0;
std::vector<std::vector<char>> kept;
int mallocs_left = -1, device = 0;
int64_t synchronised[8] = {};
}  // namespace

extern "C" {
// ---- what a test asks for
// Every later launch leaves a copy of the first `bytes` bytes of its kernel's first argument (the argument has that many); 0: none.
void host_launches_keep(size_t bytes)
{
    kept_bytes = bytes;
    kept.clear();
}
int host_launches_kept() { return (int)kept.size(); }
int host_launches_holds(int launch, uint64_t word)  // as one of its 8-byte words
{
    const std::vector<char>& a = kept[launch];
    for (size_t i = 0; i + 8 <= a.size(); i += 8)
        if (!memcmp(&a[i], &word, 8)) return 1;
    return 0;
}
// The allocation after `n` further ones is refused, once (-1: none).
void host_launches_refuse_malloc(int n) { mallocs_left = n; }
int64_t host_launches_bytes_held()
{
    std::lock_guard<std::mutex> g(mu);
    int64_t n = 0;
    for (auto& a : allocations) n += (int64_t)a.second;
    return n;
}
int64_t host_launches_synchronised(int d) { return synchronised[d]; }

// ---- the runtime
int hipMalloc(void** p, size_t bytes)
{
    if (mallocs_left == 0) {
        mallocs_left = -1;
        return result(2);
    }
    if (mallocs_left > 0) --mallocs_left;
    return plain_hipMalloc(p, bytes);
}
int hipLaunchKernel(const void* f, Dim grid, Dim block, void** args, size_t lds, void* s)
{
    if (kept_bytes) kept.emplace_back((const char*)args[0], (const char*)args[0] + kept_bytes);
    return plain_hipLaunchKernel(f, grid, block, args, lds, s);
}
int hipGetDevice(int* d)
{
    *d = device;
    return 0;
}
int hipSetDevice(int d)
{
    device = d;
    return 0;
}
int hipDeviceSynchronize()
{
    ++synchronised[device];
    return 0;
}
}
