// hip_recorder.cpp -- stands in for the HIP runtime on a machine without a
// GPU: preloaded before the library, it takes the library's runtime calls,
// keeps device memory in host memory and writes down every kernel launch (name,
// grid, the arguments asked for) instead of running it.  Tests read what it
// wrote down and check it against the call.
#include <hip/hip_runtime.h>

#include <cstdlib>
#include <cstring>
#include <map>
#include <string>
#include <vector>

namespace {

struct Launch {
    std::string name;
    dim3 grid, block;
    std::vector<std::vector<unsigned char>> args;
};
struct Block {
    size_t size, written;
};

std::map<const void*, std::string>& names() {
    static std::map<const void*, std::string> m;
    return m;
}
std::vector<std::pair<std::string, std::vector<size_t>>> g_wanted;
std::vector<Launch> g_launches;
std::map<char*, Block> g_blocks;
struct {
    dim3 grid, block;
    size_t lds;
    hipStream_t stream;
} g_next;
hipError_t g_last = hipSuccess;

hipError_t done(hipError_t e) {
    if (e != hipSuccess) g_last = e;
    return e;
}

// The block that holds p, or the end.
std::map<char*, Block>::iterator block_of(const void* p) {
    auto it = g_blocks.upper_bound((char*)p);
    if (it == g_blocks.begin()) return g_blocks.end();
    --it;
    return (char*)p < it->first + it->second.size ? it : g_blocks.end();
}

}  // namespace

extern "C" {

// ------------------------------------------------------ what tests read
// Keep `count` arguments of `bytes` each of kernels whose name holds `part`.
void recorder_want(const char* part, int count, const size_t* bytes) {
    g_wanted.push_back({part, std::vector<size_t>(bytes, bytes + count)});
}
int recorder_count() { return (int)g_launches.size(); }
void recorder_clear() { g_launches.clear(); }
const char* recorder_name(int i) { return g_launches[i].name.c_str(); }
void recorder_dims(int i, unsigned* out) {
    const Launch& l = g_launches[i];
    const unsigned d[6] = {l.grid.x, l.grid.y, l.grid.z, l.block.x, l.block.y, l.block.z};
    std::memcpy(out, d, sizeof(d));
}
const void* recorder_arg(int i, int a) { return g_launches[i].args[a].data(); }
// Bytes from p to the end of what was last copied into its block; -1: no block.
long long recorder_written_after(const void* p) {
    const auto it = block_of(p);
    return it == g_blocks.end() ? -1 : (long long)(it->first + it->second.written - (char*)p);
}

// ------------------------------------------------------------ the runtime
void** __hipRegisterFatBinary(const void*) {
    static void* handle;
    return &handle;
}
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, void*, void*,
                           int*) {
    names()[host] = name;
}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}

hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream) {
    g_next = {grid, block, lds, stream};
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* stream) {
    *grid = g_next.grid;
    *block = g_next.block;
    *lds = g_next.lds;
    *stream = g_next.stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t, hipStream_t) {
    // the runtime's own limits
    if (grid.x == 0 || grid.y == 0 || grid.z == 0 || (unsigned long long)grid.x * block.x >= (1ull << 32) ||
        grid.y > 65535 || grid.z > 65535 || block.x * block.y * block.z > 1024)
        return done(hipErrorInvalidConfiguration);
    Launch l{names()[f], grid, block, {}};
    for (const auto& [part, bytes] : g_wanted) {
        if (l.name.find(part) == std::string::npos) continue;
        for (size_t a = 0; a < bytes.size(); ++a)
            l.args.emplace_back((unsigned char*)args[a], (unsigned char*)args[a] + bytes[a]);
        break;
    }
    g_launches.push_back(l);
    return hipSuccess;
}
hipError_t hipExtLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t lds, hipStream_t s, hipEvent_t,
                              hipEvent_t, int) {
    return hipLaunchKernel(f, grid, block, args, lds, s);
}
hipError_t hipGetLastError() {
    const hipError_t e = g_last;
    g_last = hipSuccess;
    return e;
}

hipError_t hipMalloc(void** p, size_t n) {
    *p = std::malloc(n);
    std::memset(*p, 0xAB, n);
    g_blocks[(char*)*p] = {n, 0};
    return hipSuccess;
}
hipError_t hipFree(void* p) {
    g_blocks.erase((char*)p);
    std::free(p);
    return hipSuccess;
}
hipError_t hipHostMalloc(void** p, size_t n, unsigned) {
    *p = std::malloc(n);
    return hipSuccess;
}
hipError_t hipHostFree(void* p) {
    std::free(p);
    return hipSuccess;
}
hipError_t hipMemcpy(void* to, const void* from, size_t n, hipMemcpyKind) {
    std::memcpy(to, from, n);
    const auto it = block_of(to);
    if (it != g_blocks.end()) it->second.written = (size_t)((char*)to - it->first) + n;
    return hipSuccess;
}
hipError_t hipMemcpyAsync(void* to, const void* from, size_t n, hipMemcpyKind k, hipStream_t) {
    return hipMemcpy(to, from, n, k);
}

hipError_t hipEventCreateWithFlags(hipEvent_t* e, unsigned) {
    static int event;
    *e = (hipEvent_t)&event;
    return hipSuccess;
}
hipError_t hipEventDestroy(hipEvent_t) { return hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipSuccess; }
hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }
hipError_t hipStreamWaitEvent(hipStream_t, hipEvent_t, unsigned) { return hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int) { return hipSuccess; }

hipError_t hipGetDevice(int* d) {
    *d = 0;
    return hipSuccess;
}
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) {
    *v = 100000;
    return hipSuccess;
}
hipError_t hipGetDevicePropertiesR0600(hipDeviceProp_tR0600* p, int) {
    std::memset(p, 0, sizeof(*p));
    p->multiProcessorCount = 256;
    return hipSuccess;
}

}  // extern "C"
