/* The host side of the expert FFN's gradient on a runtime that is faked here, so that it runs without a GPU and a launch can fail.
 * Linked with director_ffn_grad.cu.  "Device memory" is host memory; a launch does to the two work-item counters what the
 * kernels do: it leaves its own claims in its counter and clears the other launch's. */
#include <cstdint>
static int32_t atomicCAS(int32_t*, int32_t, int32_t) { return 0; }      /* named by a device function that the host does not call */
#include "director_common.cuh"

#include <cuda.h>

#include <cstdio>
#include <cstring>

namespace director {
int ffn_grad_init(director_ctx*);
}

static unsigned int counters[2];
static int launches, fail_at, unclean;

extern "C" {
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t*, const void*, void**) {
    const int n = launches++;
    if (n == fail_at) return cudaErrorLaunchOutOfResources;
    const int phase = n & 1;
    if (counters[phase] != 0) ++unclean;               /* items would be taken for claimed already */
    counters[phase] = 100 + n;
    counters[1 - phase] = 0;
    return cudaSuccess;
}
cudaError_t cudaMemsetAsync(void* p, int v, size_t n, cudaStream_t) { memset(p, v, n); return cudaSuccess; }
cudaError_t cudaStreamIsCapturing(cudaStream_t, cudaStreamCaptureStatus* s) { *s = cudaStreamCaptureStatusNone; return cudaSuccess; }
cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t cudaLaunchKernel(const void*, dim3, dim3, void**, size_t, cudaStream_t) { return cudaErrorUnknown; }
cudaError_t cudaEventCreate(cudaEvent_t*) { return cudaErrorUnknown; }
cudaError_t cudaEventRecord(cudaEvent_t, cudaStream_t) { return cudaErrorUnknown; }
cudaError_t __cudaPopCallConfiguration(dim3*, dim3*, size_t*, void*) { return cudaErrorUnknown; }
void** __cudaRegisterFatBinary(void*) { static void* handle; return &handle; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
void __cudaRegisterFunction(void**, const char*, char*, const char*, int, uint3*, uint3*, dim3*, dim3*, int*) {}
}

static CUresult encode(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                       const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill) {
    return CUDA_SUCCESS;
}

int main() {
    using namespace director;
    director_ctx ctx;
    ctx.shape = director_shape{64, 256, 128, 8, 2, 0, 4, 3};
    ctx.pair_clusters = 74;
    ctx.n_replicas = 8;
    ctx.encode_tiled = reinterpret_cast<void*>(&encode);
    ctx.d_grad_sched = counters;
    static uint16_t data[64];
    const Checkpoint kept{reinterpret_cast<int8_t*>(data), data, 128};
    const FfnGrad routed{data, data, kept, data, data, data, data, data, data, data}, none{};
    /* call 0 succeeds; the second launch of call 1 fails; call 2 succeeds again (launches 4 and 5) */
    fail_at = 3;
    const int a = launch_expert_ffn_backward(&ctx, nullptr, routed, none, nullptr);
    const int b = launch_expert_ffn_backward(&ctx, nullptr, routed, none, nullptr);
    const int c = launch_expert_ffn_backward(&ctx, nullptr, routed, none, nullptr);
    printf("%d %d %d launches %d unclean %d\n", a, b, c, launches, unclean);
    return a == DIRECTOR_OK && b == DIRECTOR_ERR_CUDA && c == DIRECTOR_OK && launches == 6 && unclean == 0 ? 0 : 1;
}
