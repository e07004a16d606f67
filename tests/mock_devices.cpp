// Two GPUs for tests of the host side without one, loaded before mock_hip.cpp: what a kernel may use of dynamic LDS beyond 64 KB is declared for the GPU that
// is current, and a launch that has not been declared on its own is counted.
#include <stdint.h>

#include <cstddef>
#include <map>
#include <utility>

namespace {

struct Dim { uint32_t x, y, z; };
int g_device = 0, g_launches = 0, g_undeclared = 0;
std::map<std::pair<int, const void *>, int> g_most;

}  // namespace

extern "C" {

int hipGetDevice(int *dev) { *dev = g_device; return 0; }
int hipFuncSetAttribute(const void *fn, int, int value)
{
    g_most[{g_device, fn}] = value;
    return 0;
}
int hipLaunchKernel(const void *fn, Dim, Dim, void **, size_t lds, void *)
{
    const auto at = g_most.find({g_device, fn});
    ++g_launches;
    if (lds > 64 * 1024 && (at == g_most.end() || (size_t)at->second < lds)) ++g_undeclared;
    return 0;
}
void devices_use(int dev) { g_device = dev; }
int devices_launches() { return g_launches; }
int devices_undeclared() { return g_undeclared; }

}  // extern "C"
