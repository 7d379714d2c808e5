/* AdamW's tables with masters and moments at any address, on a runtime that is faked here, so that it runs without a GPU.  All five
 * arrays of every chunk are walked as the kernels walk them: each element once, inside its tensor, and whole accesses (32 bytes of fp32,
 * 16 of bf16) only where the address allows them. */
#include "../../paper_2607_08782_b200/csrc/director_update.cu"

#include <cstdio>
#include <map>
#include <vector>

using namespace director;

static int bad, small_updates, updates, whole_states, odd_states;
static std::map<uintptr_t, std::vector<unsigned char>> seen;         /* address of an array -> how often each element was touched */

static void expect(bool ok, const char* what) {
    if (!ok && bad++ < 10) printf("failed: %s\n", what);
}
template <typename TABLE>
static void walk(const TABLE& t, unsigned grid) {
    for (unsigned c = 0; c < grid; ++c) {
        const Place p = place_of(t, (int)c, kChunk);
        const bool master = p.kind & kOutBf16;
        (p.kind & kStateWhole ? whole_states : odd_states)++;
        expect((t.at[2][p.k] != nullptr) == master, "a master for a bf16 weight");
        for (int a = 0; a < 5; ++a) {
            if (a == 2 && !master) continue;
            const bool bf16 = (a == 0 && (p.kind & kGradBf16)) || (a == 1 && (p.kind & kOutBf16));
            const int bit = a == 0 ? kGradWhole : a == 1 ? kOutWhole : kStateWhole, width = bf16 ? 2 : 4;
            const uintptr_t base = reinterpret_cast<uintptr_t>(t.at[a][p.k]);
            auto& n = seen[base];
            n.resize((size_t)t.numel[p.k]);
            for (int e = 0; e < kChunk; e += 8) {
                const int lo = p.lo(e), hi = p.hi(e);
                expect(lo == 0, "a step's chunks begin inside the tensor");
                for (int i = lo; i < hi; ++i) {
                    const long long at = p.at + e + i;
                    expect(at >= 0 && at < t.numel[p.k], "an element of the tensor");
                    if (at >= 0 && at < t.numel[p.k]) ++n[(size_t)at];
                }
                if ((p.kind & bit) && hi == 8) expect((base + (uintptr_t)(p.at + e) * width) % (width * 8) == 0, "a whole access is aligned");
            }
        }
    }
}

extern "C" {
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* cfg, const void* f, void** a) {
    if (f == (const void*)update_kernel) {
        ++updates;
        walk(*(const Table<5, kUpdateTensors>*)a[0], cfg->gridDim.x);
    } else if (f == (const void*)update_small_kernel) {
        ++small_updates;
        walk(*(const Table<5, kFewTensors>*)a[0], cfg->gridDim.x);
    }
    return cudaSuccess;
}
#ifndef __CUDA_ARCH__        /* the device pass has these from a header */
cudaError_t cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* v, cudaDeviceAttr, int) { *v = 148; return cudaSuccess; }
cudaError_t cudaEventRecord(cudaEvent_t, cudaStream_t) { return cudaErrorUnknown; }
#endif
cudaError_t cudaStreamIsCapturing(cudaStream_t, cudaStreamCaptureStatus* s) { *s = cudaStreamCaptureStatusNone; return cudaSuccess; }
cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t cudaLaunchKernel(const void*, dim3, dim3, void**, size_t, cudaStream_t) { return cudaErrorUnknown; }
cudaError_t cudaEventCreate(cudaEvent_t*) { return cudaErrorUnknown; }
cudaError_t __cudaPopCallConfiguration(dim3*, dim3*, size_t*, void*) { return cudaErrorUnknown; }
void** __cudaRegisterFatBinary(void*) { static void* handle; return &handle; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
void __cudaRegisterFunction(void**, const char*, char*, const char*, int, uint3*, uint3*, dim3*, dim3*, int*) {}
}

static uintptr_t next_room = 1ull << 40;                             /* addresses that nobody looks at */
static void* room(long long numel, int type, int shift) {
    const uintptr_t at = next_room + (uintptr_t)shift * width_of(type);
    next_room = (at + (uintptr_t)numel * width_of(type) + 511) / 256 * 256;
    return reinterpret_cast<void*>(at);
}

int main() {
    alignas(16) static unsigned char work[sizeof(Workspace)];
    static float norm;
    static int64_t steps;
    /* each of the five arrays shifted in turn by 0 to 7 elements (array 5: all of them), for the one launch and for the several */
    for (const double max_norm : {1.0, (double)INFINITY})
        for (const long long most : {5000ll, 400000ll})
            for (int which = 0; which <= 5; ++which)
                for (int shift = 0; shift < 8; ++shift) {
                    const director_adamw h{1e-3, 0.9, 0.99, 1e-8, 0.0, max_norm};
                    std::vector<director_tensor> g;
                    std::vector<director_param> p;
                    const auto at = [&](int array) { return array == which || which == 5 ? shift : 0; };
                    for (const long long numel : {1ll, 7ll, 9ll, 2047ll, 2048ll, 2049ll, most})
                        for (int kinds = 0; kinds < 4; ++kinds) {
                            const int gt = kinds & 1, wt = kinds >> 1;
                            g.push_back({room(numel, gt, at(0)), numel, gt, 0});
                            p.push_back({room(numel, wt, at(1)), wt == DIRECTOR_BF16 ? (float*)room(numel, 0, at(2)) : nullptr,
                                         (float*)room(numel, 0, at(3)), (float*)room(numel, 0, at(4)), numel, wt, 0});
                        }
                    seen.clear();
                    expect(director_adamw_step((int)g.size(), g.data(), p.data(), &h, nullptr, &steps, max_norm == 1.0 ? &norm : nullptr, nullptr,
                                               work, nullptr) == DIRECTOR_OK, "step");
                    const auto once = [&](const void* array, long long numel) {
                        const auto& n = seen[reinterpret_cast<uintptr_t>(array)];
                        expect((long long)n.size() == numel, "every array is walked");
                        for (unsigned char c : n) expect(c == 1, "every element once");
                    };
                    for (size_t i = 0; i < g.size(); ++i) {
                        once(g[i].data, g[i].numel), once(p[i].weight, g[i].numel);
                        once(p[i].exp_avg, g[i].numel), once(p[i].exp_avg_sq, g[i].numel);
                        if (p[i].master != nullptr) once(p[i].master, g[i].numel);
                    }
                }
    printf("update %d/%d, states whole %d odd %d, %d bad\n", updates, small_updates, whole_states, odd_states, bad);
    return bad != 0 || !updates || !small_updates || !whole_states || !odd_states;
}
