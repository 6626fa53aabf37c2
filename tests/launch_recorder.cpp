// The launch functions of the HIP runtime for a process without a GPU: they write down which kernel would run in which grid and
// launch nothing.  Loaded before the library, whose references then find these.  hipGetLastError gives the last error and clears
// it, as the runtime's does.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cxxabi.h>
#include <map>
#include <string>

namespace {
struct Grid {
    uint32_t x, y, z;
};
struct Launch {
    Grid grid, block;
    size_t shared;
    void* stream;
};
Launch configured;
std::map<const void*, std::string>& kernels() {
    static std::map<const void*, std::string> m;
    return m;
}
std::string written;
int until_failure = -1, last_error = 0;
constexpr int kInvalidConfiguration = 9;
}  // namespace

extern "C" {
void** __hipRegisterFatBinary(const void*) {
    static void* module;
    return &module;
}
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, void*, void*, int*) {
    int status;
    char* plain = abi::__cxa_demangle(name, nullptr, nullptr, &status);
    kernels()[host] = plain ? plain : name;
    free(plain);
}
int __hipPushCallConfiguration(Grid grid, Grid block, size_t shared, void* stream) {
    configured = {grid, block, shared, stream};
    return 0;
}
int __hipPopCallConfiguration(Grid* grid, Grid* block, size_t* shared, void** stream) {
    *grid = configured.grid, *block = configured.block, *shared = configured.shared, *stream = configured.stream;
    return 0;
}
int hipLaunchKernel(const void* kernel, Grid grid, Grid block, void**, size_t shared, void*) {
    char line[128];
    snprintf(line, sizeof line, "%u %u %u|%u|%zu|", grid.x, grid.y, grid.z, block.x * block.y * block.z, shared);
    written += line + kernels()[kernel] + "\n";
    if (until_failure >= 0 && until_failure-- == 0) return last_error = kInvalidConfiguration;
    return 0;
}
int hipGetLastError() {
    const int error = last_error;
    last_error = 0;
    return error;
}
// The kernels of the library, one a line.
const char* kernels_known() {
    static std::string all;
    all.clear();
    for (const auto& k : kernels()) all += k.second + "\n";
    return all.c_str();
}
// What was launched since the last call; the launch of that number from here on fails (-1: none).
const char* launches_taken(int fail) {
    static std::string taken;
    taken.swap(written);
    written.clear();
    last_error = 0;
    until_failure = fail;
    return taken.c_str();
}
}
