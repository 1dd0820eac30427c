// A program that includes this stands in for the runtime's launch: it keeps what was launched, and does nothing.  Link with -rdynamic
// -ldl, so that the library's launches come here and a kernel's name can be asked for.
#ifndef LAUNCH_STUB_H
#define LAUNCH_STUB_H

#include <cstdint>
#include <string>
#include <vector>

#include <dlfcn.h>

struct LaunchDim { uint32_t x, y, z; };
struct Launched { std::string kernel;            // as the linker knows it
                  LaunchDim grid, block; };
static std::vector<Launched> g_launched;

extern "C" {
static struct { LaunchDim grid, block; size_t shared; void* stream; } g_next_launch;
unsigned __hipPushCallConfiguration(LaunchDim grid, LaunchDim block, size_t shared, void* stream) {
    g_next_launch = {grid, block, shared, stream};
    return 0;
}
int __hipPopCallConfiguration(LaunchDim* grid, LaunchDim* block, size_t* shared, void** stream) {
    *grid = g_next_launch.grid;
    *block = g_next_launch.block;
    *shared = g_next_launch.shared;
    *stream = g_next_launch.stream;
    return 0;
}
int hipLaunchKernel(const void* kernel, LaunchDim grid, LaunchDim block, void**, size_t, void*) {
    Dl_info info;
    const char* name = dladdr(kernel, &info) && info.dli_sname ? info.dli_sname : "";
    g_launched.push_back({name, grid, block});
    return 0;
}
int hipGetLastError(void) { return 0; }
}

#endif
