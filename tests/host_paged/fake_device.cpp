// A device for the host code of the paged cache that launches nothing: the CUDA calls that the host code makes succeed,
// the launchers count themselves.  One device of 148 multiprocessors; fake_set_device changes the current one.
#include <cuda_runtime.h>

#include "xkv_paged_internal.cuh"

static int g_device = 0, g_launches = 0;

extern "C" {
void fake_set_device(int d) { g_device = d; }
int fake_launches() { return g_launches; }

// registration of the (absent) device code
void** __cudaRegisterFatBinary(void*) { static void* h; return &h; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
char __cudaInitModule(void**) { return 0; }

cudaError_t cudaGetDevice(int* d) { *d = g_device; return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* v, cudaDeviceAttr, int) { *v = 148; return cudaSuccess; }
cudaError_t cudaMemsetAsync(void*, int, size_t, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaMemcpyAsync(void*, const void*, size_t, cudaMemcpyKind, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaStreamSynchronize(cudaStream_t) { return cudaSuccess; }
cudaError_t cudaGetLastError() { return cudaSuccess; }
}

namespace xkv {
static cudaError_t launched() { ++g_launches; return cudaSuccess; }
cudaError_t launch_tokens(const TokenArgs&, int, int, cudaStream_t) { return launched(); }
cudaError_t launch_evict(const EvictArgs&, cudaStream_t) { return launched(); }
cudaError_t evict_device_setup() { return cudaSuccess; }
cudaError_t make_pool_maps(const PagedView&, int, int, int, PoolMaps*) { return cudaSuccess; }
cudaError_t attn_few_setup() { return cudaSuccess; }
cudaError_t launch_attn_few(const PagedAttnArgs&, const PoolMaps&, const PagedScratch&, int, int, int, cudaStream_t) { return launched(); }
size_t attn_chunk_cut_bytes() { return 32; }
cudaError_t attn_chunk_setup() { return cudaSuccess; }
cudaError_t launch_attn_chunk(const PagedAttnArgs&, const PoolMaps&, const PagedScratch&, void*, int, int, int, cudaStream_t) { return launched(); }
cudaError_t launch_paged_attn_simple(const PagedAttnArgs&, int, int, cudaStream_t) { return launched(); }
cudaError_t weights_setup() { return cudaSuccess; }
cudaError_t launch_paged_weights(const PagedWeightArgs&, const PoolMaps&, int, int, int, cudaStream_t) { return launched(); }
}  // namespace xkv
