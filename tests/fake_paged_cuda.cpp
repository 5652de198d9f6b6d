// A CUDA runtime of one host process that counts what the paged calls ask of it; launches do nothing.  The test links it with the
// library's host objects; entry points that are neither here nor there return zero.
#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdlib>
#include <cstring>

#define FAKE extern "C" __attribute__((visibility("default")))

namespace {
struct Counts { int properties, attributes, launches, maps; };
Counts g_n{};
int g_fail_attribute = 0;
CUresult encode(CUtensorMap* m, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill)
{
    ++g_n.maps;
    std::memset(m, 0, sizeof *m);
    return CUDA_SUCCESS;
}
}  // namespace

FAKE Counts fake_counts() { return g_n; }
FAKE void fake_fail_attribute(int n) { g_fail_attribute = n; }       // the n-th setting of an attribute from now fails

FAKE cudaError_t cudaGetDeviceCount(int* n) { *n = 2; return cudaSuccess; }
FAKE cudaError_t cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
FAKE cudaError_t cudaGetDeviceProperties_v2(cudaDeviceProp* p, int)
{
    ++g_n.properties;
    std::memset(p, 0, sizeof *p);
    p->major = 10; p->multiProcessorCount = 148;
    return cudaSuccess;
}
FAKE cudaError_t cudaGetDriverEntryPoint(const char*, void** fn, unsigned long long, cudaDriverEntryPointQueryResult* r)
{
    *fn = (void*)encode; *r = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}
FAKE cudaError_t cudaMalloc(void** p, size_t n) { *p = std::malloc(n); return cudaSuccess; }
FAKE cudaError_t cudaFree(void* p) { std::free(p); return cudaSuccess; }
FAKE cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int)
{
    ++g_n.attributes;
    return g_fail_attribute > 0 && --g_fail_attribute == 0 ? cudaErrorInvalidValue : cudaSuccess;
}
FAKE cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t*, const void*, void**) { ++g_n.launches; return cudaSuccess; }
