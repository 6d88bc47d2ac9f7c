// What follows a launch that is refused.  The runtime's launch calls (and what else a call asks of the runtime) are replaced by the
// linker (--wrap) with fakes, so nothing reaches a GPU: the n-th launch of a call is refused, and the launches are counted.
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdio.h>

#include "fd_internal.cuh"
#include "fd_prompt.cuh"

static int launches, refused;
static cudaError_t next() { return ++launches == refused ? cudaErrorLaunchOutOfResources : cudaSuccess; }
static CUresult encode_any() { return CUDA_SUCCESS; }

extern "C" {
cudaError_t __wrap_cudaLaunchKernelExC(const cudaLaunchConfig_t*, const void*, void**) { return next(); }
cudaError_t __wrap_cudaLaunchKernel(const void*, dim3, dim3, void**, size_t, cudaStream_t) { return next(); }
unsigned __wrap___cudaPushCallConfiguration(dim3, dim3, size_t, void*) { return 0; }
cudaError_t __wrap___cudaPopCallConfiguration(dim3*, dim3*, size_t*, void*) { return cudaSuccess; }
cudaError_t __wrap_cudaGetDriverEntryPoint(const char*, void** f, unsigned long long, cudaDriverEntryPointQueryResult*) {
    *f = reinterpret_cast<void*>(encode_any);
    return cudaSuccess;
}
cudaError_t __wrap_cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t __wrap_cudaFuncGetAttributes(cudaFuncAttributes* a, const void*) {
    a->numRegs = 168;
    return cudaSuccess;
}
}

// "name refused: launches attempted, what the call said"
template <class F>
static void report(const char* name, int kernels, F call) {
    for (refused = 0; refused <= kernels; ++refused) {
        launches = 0;
        const int said = call();
        printf("%s %d: %d %d\n", name, refused, launches, said);
    }
}

int main() {
    fd::CompactParams c = {};
    c.batch = 4; c.num_pages = 100; c.max_pages = 8; c.n_sms = 148;
    report("compact", 2, [&] { return fd::launch_kv_compact(c, nullptr); });
    c.num_pages = 100000;
    report("compact in a cluster", 2, [&] { return fd::launch_kv_compact(c, nullptr); });
    fd::FreeParams f = {};
    f.n_seqs = 512; f.max_pages = 300; f.n_sms = 148;
    report("free", 4, [&] { return fd::launch_kv_free(f, nullptr); });
    fd::PromptParams p = {};
    p.batch = 40; p.total_q = 64; p.total_kv = 9000; p.Hq = 8; p.Hkv = 2; p.G = 4; p.d = 128; p.tile_tokens = 32; p.n_ctas = 148;
    p.q_stride = 1024; p.kv_stride = 256;
    p.split = reinterpret_cast<fd::PromptSplit*>(16);
    void* state = nullptr;
    if (fd::prompt_tc_prepare(&state, p) != cudaSuccess) return 1;
    report("prompt", 2, [&] {
        int n = 0;
        const cudaError_t e = fd::launch_prompt_tc(state, p, &n, nullptr);
        return e == cudaSuccess ? n : -n - 1;
    });
    fd::prompt_tc_free(state);
}
