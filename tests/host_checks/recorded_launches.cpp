// A runtime that launches nothing: what the host side of a HIP source calls, with every launch written down instead.
//
// The host side of a source, compiled by itself and linked with this file alone, runs on any machine: its entry points check
// their arguments and choose their kernels as they always do.  recorded() gives the launches since it was last called, one a line: the
// kernel's name, its dynamic LDS in bytes, the limit that was asked for it (0: none was, and 64 KB are all that it may have with
// its static variables), its workgroups and their threads.
#include <cstddef>
#include <map>
#include <string>

// As HIP's C interface has them.
struct dim3 {
    unsigned x, y, z;
};
typedef int hipError_t;
typedef void* hipStream_t;
constexpr hipError_t hipSuccess = 0;

namespace {

struct Dims {
    dim3 grid, block;
    size_t lds;
    hipStream_t stream;
};
std::map<const void*, std::string>& names() { static std::map<const void*, std::string> m; return m; }
std::map<const void*, int>& limits() { static std::map<const void*, int> m; return m; }
std::string& lines() { static std::string s; return s; }
Dims now;

void write_down(const void* kernel, dim3 grid, dim3 block, size_t lds) {
    auto count = [](dim3 d) { return std::to_string((unsigned long long)d.x * d.y * d.z); };
    lines() += names()[kernel] + " " + std::to_string(lds) + " " + std::to_string(limits()[kernel]) + " " + count(grid) + " " + count(block) + "\n";
}

}  // namespace

extern "C" {

extern const char __hip_fatbin[1];
const char __hip_fatbin[1] = {0};       // the device code, of which there is none

void** __hipRegisterFatBinary(const void*) { static void* handle; return &handle; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* kernel, char*, const char* name, unsigned, void*, void*, void*, void*, int*) { names()[kernel] = name; }
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}

hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream) { now = {grid, block, lds, stream}; return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* stream) {
    *grid = now.grid; *block = now.block; *lds = now.lds; *stream = now.stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void* kernel, dim3 grid, dim3 block, void**, size_t lds, hipStream_t) { write_down(kernel, grid, block, lds); return hipSuccess; }
hipError_t hipFuncSetAttribute(const void* kernel, int, int value) { limits()[kernel] = value; return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipGetDevice(int* device) { *device = 0; return hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }

// The launches since the last call; limits are forgotten as well, so that each set of calls has to ask by itself.
const char* recorded() {
    static std::string out;
    out.swap(lines());
    lines().clear();
    limits().clear();
    return out.c_str();
}

}  // extern "C"
