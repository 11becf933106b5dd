// A stand-in for the CUDA runtime that runs nothing: every call succeeds, memory is made-up addresses, and each kernel launch
// is written down -- the kernel's name, the device that was current, the stream, the first bytes of its first argument.  Linked
// with the library's objects it lets the host side of the entry points run without a GPU (and without touching one).
#include <cuda_runtime_api.h>
#include <string.h>
#include <stdlib.h>

#include <map>
#include <string>
#include <utility>
#include <vector>

namespace {
struct Launch { std::string name; int device; void* stream; unsigned char arg[128]; };
std::vector<Launch> launches;
std::map<const void*, std::string>& names() { static std::map<const void*, std::string> m; return m; }
int device = 0;
unsigned long long next_address = 0x500000000000ull;
std::vector<std::pair<unsigned long long, size_t>> blocks;       // device memory handed out
struct { dim3 grid, block; size_t smem; void* stream; } pushed;

void note(const void* kernel, void* stream, void** args) {
    Launch l = {names()[kernel], device, stream, {}};
    // (only of the kernels whose arguments are looked at: one structure of at least as many bytes)
    if (l.name.find("page_select") != std::string::npos || l.name.find("attn_decode_pages") != std::string::npos) memcpy(l.arg, args[0], sizeof l.arg);
    launches.push_back(l);
}
int encode_tiled() { return 0; }
int handle;
}  // namespace

extern "C" {
// ---- what a test reads and sets
int host_launch_count() { return (int)launches.size(); }
const char* host_launch_name(int i) { return launches[i].name.c_str(); }
int host_launch_device(int i) { return launches[i].device; }
void* host_launch_stream(int i) { return launches[i].stream; }
const void* host_launch_arg(int i) { return launches[i].arg; }
void host_forget() { launches.clear(); }
void host_set_device(int d) { device = d; }
int host_device() { return device; }
int host_allocated(unsigned long long from, unsigned long long to) {       // is [from, to) part of one block
    for (auto& b : blocks) if (from >= b.first && to <= b.first + b.second) return 1;
    return 0;
}

// ---- the runtime
void** __cudaRegisterFatBinary(void*) { static void* h[1]; return h; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
void __cudaRegisterFunction(void**, const char* host, char*, const char* name, int, void*, void*, void*, void*, int*) { names()[host] = name; }
void __cudaRegisterVar(void**, char*, char*, const char*, int, size_t, int, int) {}
unsigned __cudaPushCallConfiguration(dim3 g, dim3 b, size_t s, void* st) { pushed = {g, b, s, st}; return 0; }
cudaError_t __cudaPopCallConfiguration(dim3* g, dim3* b, size_t* s, void* st) {
    *g = pushed.grid; *b = pushed.block; *s = pushed.smem;
    *(void**)st = pushed.stream;
    return cudaSuccess;
}
cudaError_t cudaLaunchKernel(const void* f, dim3, dim3, void** a, size_t, cudaStream_t st) { note(f, st, a); return cudaSuccess; }
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void* f, void** a) { note(f, c->stream, a); return cudaSuccess; }
cudaError_t cudaGetDevice(int* d) { *d = device; return cudaSuccess; }
cudaError_t cudaSetDevice(int d) { device = d; return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* v, cudaDeviceAttr, int) { *v = 148; return cudaSuccess; }
cudaError_t cudaGetDeviceProperties(cudaDeviceProp* p, int) {
    memset(p, 0, sizeof *p);
    p->major = 10;
    p->multiProcessorCount = 148;
    return cudaSuccess;
}
cudaError_t cudaMalloc(void** p, size_t n) {
    *p = (void*)next_address;
    blocks.push_back({next_address, n});
    next_address += (n + (2u << 20)) >> 21 << 21;
    return cudaSuccess;
}
cudaError_t cudaFree(void*) { return cudaSuccess; }
cudaError_t cudaHostAlloc(void** p, size_t n, unsigned) { *p = calloc(1, n); return cudaSuccess; }
cudaError_t cudaFreeHost(void* p) { free(p); return cudaSuccess; }
cudaError_t cudaMemset(void*, int, size_t) { return cudaSuccess; }
cudaError_t cudaMemsetAsync(void*, int, size_t, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaMemcpy(void*, const void*, size_t, cudaMemcpyKind) { return cudaSuccess; }
cudaError_t cudaMemcpyAsync(void*, const void*, size_t, cudaMemcpyKind, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaMemcpyPeerAsync(void*, int, const void*, int, size_t, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaStreamCreateWithFlags(cudaStream_t* s, unsigned) { static long n = 0x100; *s = (cudaStream_t)(n += 16); return cudaSuccess; }
cudaError_t cudaStreamDestroy(cudaStream_t) { return cudaSuccess; }
cudaError_t cudaStreamSynchronize(cudaStream_t) { return cudaSuccess; }
cudaError_t cudaStreamWaitEvent(cudaStream_t, cudaEvent_t, unsigned) { return cudaSuccess; }
cudaError_t cudaDeviceSynchronize() { return cudaSuccess; }
cudaError_t cudaEventCreate(cudaEvent_t* e) { *e = (cudaEvent_t)&handle; return cudaSuccess; }
cudaError_t cudaEventCreateWithFlags(cudaEvent_t* e, unsigned) { *e = (cudaEvent_t)&handle; return cudaSuccess; }
cudaError_t cudaEventDestroy(cudaEvent_t) { return cudaSuccess; }
cudaError_t cudaEventRecord(cudaEvent_t, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaEventSynchronize(cudaEvent_t) { return cudaSuccess; }
cudaError_t cudaEventElapsedTime(float* t, cudaEvent_t, cudaEvent_t) { *t = 0.f; return cudaSuccess; }
cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t cudaGetLastError() { return cudaSuccess; }
const char* cudaGetErrorString(cudaError_t) { return "stand-in"; }
cudaError_t cudaGetSymbolAddress(void** p, const void*) { return cudaMalloc(p, 16u << 20); }
cudaError_t cudaOccupancyMaxActiveClusters(int* n, const void*, const cudaLaunchConfig_t*) { *n = 16; return cudaSuccess; }
cudaError_t cudaGetDriverEntryPoint(const char*, void** p, unsigned long long, cudaDriverEntryPointQueryResult* r) {
    *p = (void*)&encode_tiled;
    if (r) *r = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}
}
