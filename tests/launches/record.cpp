// Stands in for the HIP runtime under the library's own objects: a launch is only
// written down.  Linked into a library of its own, which runs without a GPU.
#include <stdint.h>

#include <map>
#include <string>
#include <vector>

namespace {
struct Dim {
    uint32_t x, y, z;
};
struct Launch {
    Dim grid, block;
    uint64_t lds;
    const char* name;
};
std::map<const void*, std::string>& names() {
    static std::map<const void*, std::string> n;
    return n;
}
std::vector<Launch> launches;
Dim pushed_grid, pushed_block;
size_t pushed_lds;
void* pushed_stream;
void* module_handle;
}  // namespace

#define EXPORT extern "C" __attribute__((visibility("default")))

extern "C" {
void** __hipRegisterFatBinary(const void*) { return &module_handle; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*,
                           void*, void*, void*, int*) {
    names()[host] = name;
}
int __hipPushCallConfiguration(Dim grid, Dim block, size_t lds, void* stream) {
    pushed_grid = grid, pushed_block = block, pushed_lds = lds, pushed_stream = stream;
    return 0;
}
int __hipPopCallConfiguration(Dim* grid, Dim* block, size_t* lds, void** stream) {
    *grid = pushed_grid, *block = pushed_block, *lds = pushed_lds, *stream = pushed_stream;
    return 0;
}
int hipLaunchKernel(const void* host, Dim grid, Dim block, void**, size_t lds, void*) {
    launches.push_back({grid, block, lds, names()[host].c_str()});
    return 0;
}
int hipGetLastError() { return 0; }
int hipGetDevice(int* device) { return *device = 0; }
int hipFuncSetAttribute(const void*, int, int) { return 0; }
}

EXPORT void record_clear() { launches.clear(); }
EXPORT int64_t record_count() { return (int64_t)launches.size(); }
EXPORT const char* record_launch(int64_t k, uint32_t* dims, uint64_t* lds) {
    const Launch& l = launches[k];
    const uint32_t d[6] = {l.grid.x, l.grid.y, l.grid.z, l.block.x, l.block.y, l.block.z};
    for (int i = 0; i < 6; ++i) dims[i] = d[i];
    *lds = l.lds;
    return l.name;
}
