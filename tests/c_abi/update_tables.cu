/* The host side of norm, clipping and AdamW on a runtime that is faked here, so that it runs without a GPU: the tables that the
 * launches get are walked as the kernels walk them.  Every element of every tensor has to belong to exactly one thread, inside its
 * tensor, with whole accesses only where the address allows them; and a call whose launch fails must not have counted its step. */
#include "../../paper_2607_08782_b200/csrc/director_update.cu"

#include <cstdio>
#include <cstring>
#include <map>
#include <vector>

using namespace director;

static int launches, fail_at = -1, bad, norms, finishes, clips, updates, small_clips, small_updates, clusters, counted;
static std::map<uintptr_t, std::vector<unsigned char>> seen;         // address of an array -> how often each element was touched

static void expect(bool ok, const char* what) {
    if (!ok && bad++ < 10) printf("failed: %s\n", what);
}
template <typename TABLE>
static void walk(const TABLE& t, unsigned grid, int chunk, int array, bool bf16_bit, int whole_bit) {
    expect((int)grid == t.first[t.n], "a CTA for every chunk");
    for (unsigned c = 0; c < grid; ++c) {
        const Place p = place_of(t, (int)c, chunk);
        const bool bf16 = p.kind & (bf16_bit ? kOutBf16 : kGradBf16);
        const uintptr_t base = reinterpret_cast<uintptr_t>(t.at[array][p.k]);
        auto& n = seen[base];
        n.resize((size_t)t.numel[p.k]);
        for (int e = 0; e < chunk; e += 8) {
            const int lo = p.lo(e), hi = p.hi(e);
            for (int i = lo; i < hi; ++i) {
                const long long at = p.at + e + i;
                expect(at >= 0 && at < t.numel[p.k], "an element of the tensor");
                if (at >= 0 && at < t.numel[p.k]) ++n[(size_t)at];
            }
            const bool whole = (p.kind & whole_bit) && lo == 0 && hi == 8;
            if (whole) expect((base + (p.at + e) * (bf16 ? 2 : 4)) % (bf16 ? 16 : 32) == 0, "a whole access is aligned");
            if (p.full(chunk)) expect(lo == 0 && hi == 8, "a full chunk is full");
        }
    }
}
/* the norm: the chunks of squares_of_chunk, with its head and tail */
template <typename TABLE>
static void walk_norm(const TABLE& t, int per) {
    for (int k = 0; k < t.n; ++k) {
        const long long n = t.numel[k];
        const bool bf16 = t.kind[k] == DIRECTOR_BF16;
        const long long head = bf16 ? head_of<__nv_bfloat16>(t.at[0][k], n) : head_of<float>(t.at[0][k], n), width = bf16 ? 8 : 4;
        const long long vecs = (n - head) / width, chunks = t.first[k + 1] - t.first[k];
        expect(head <= 32 && n - head - vecs * width <= 32, "ragged ends fit a warp each");
        expect(chunks >= 1 && chunks * per >= vecs && (chunks - 1) * per < std::max(vecs, 1ll), "the chunks hold the vectors");
        if (vecs > 0) expect((reinterpret_cast<uintptr_t>(t.at[0][k]) + head * (bf16 ? 2 : 4)) % 16 == 0, "vectors are aligned");
        for (int c = t.first[k]; c < t.first[k + 1]; ++c) expect(tensor_of(t, c) == k, "a chunk's tensor");
    }
}

extern "C" {
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* cfg, const void* f, void** a) {
    if (launches++ == fail_at) return cudaErrorLaunchOutOfResources;
    const unsigned grid = cfg->gridDim.x;
    if (f == (const void*)norm_kernel) {
        ++norms;
        walk_norm(*(const Table<1, kNormTensors>*)a[0], kThreads * kNormUnroll);
        expect(grid >= 1 && grid <= kSlots, "a slot for every CTA");
    } else if (f == (const void*)norm_cluster_kernel) {
        ++clusters;
        walk_norm(*(const Table<1, kFewTensors>*)a[0], kClusterThreads * kClusterUnroll);
    } else if (f == (const void*)finish_kernel) {
        ++finishes;
        const Call& q = *(const Call*)a[0];
        counted += *(const bool*)a[2] && q.steps != nullptr;
    } else if (f == (const void*)clip_kernel) {
        ++clips;
        walk(*(const Table<2, kClipTensors>*)a[0], grid, kClipChunk, 1, true, kOutWhole);
        walk(*(const Table<2, kClipTensors>*)a[0], grid, kClipChunk, 0, false, kGradWhole);
    } else if (f == (const void*)clip_small_kernel) {
        ++small_clips;
        walk(*(const Table<2, kFewTensors>*)a[0], grid, kClipChunk, 1, true, kOutWhole);
        walk(*(const Table<2, kFewTensors>*)a[0], grid, kClipChunk, 0, false, kGradWhole);
    } else if (f == (const void*)update_kernel) {
        ++updates;
        walk(*(const Table<5, kUpdateTensors>*)a[0], grid, kChunk, 1, true, kOutWhole);
        walk(*(const Table<5, kUpdateTensors>*)a[0], grid, kChunk, 0, false, kGradWhole);
        counted += *(const bool*)a[3];
    } else if (f == (const void*)update_small_kernel) {
        ++small_updates;
        walk(*(const Table<5, kFewTensors>*)a[0], grid, kChunk, 1, true, kOutWhole);
        walk(*(const Table<5, kFewTensors>*)a[0], grid, kChunk, 0, false, kGradWhole);
        ++counted;
    } else {
        expect(false, "a kernel of this file");
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

static uint64_t state = 88172645463325252ull;
static long long draw(long long n) {
    state ^= state << 13, state ^= state >> 7, state ^= state << 17;
    return (long long)(state % (uint64_t)n);
}

struct Set {
    std::vector<director_tensor> g, out;
    std::vector<director_param> p;
    uintptr_t next = 1ull << 40;                                     /* addresses that nobody looks at */
    void* room(long long numel, int type, bool odd) {
        const uintptr_t at = next + (odd ? (uintptr_t)draw(8) * width_of(type) : 0);
        next = (at + (uintptr_t)numel * width_of(type) + 511) / 256 * 256;
        return reinterpret_cast<void*>(at);
    }
    Set(int n, long long most, bool odd, bool in_place) {
        for (int i = 0; i < n; ++i) {
            const long long numel = draw(5) == 0 ? draw(20) : draw(most);
            const int gt = (int)draw(2), wt = (int)draw(2);
            g.push_back({room(numel, gt, odd), numel, gt, 0});
            out.push_back(in_place ? g.back() : director_tensor{room(numel, wt, odd), numel, wt, 0});
            p.push_back({room(numel, wt, odd), wt == DIRECTOR_BF16 ? (float*)room(numel, 0, false) : nullptr, (float*)room(numel, 0, false),
                         (float*)room(numel, 0, odd && draw(3) == 0), numel, wt, 0});
        }
    }
    /* every array of the kind touched once an element */
    void once(const std::vector<director_tensor>& which) {
        for (auto& t : which)
            if (t.numel > 0)
                for (unsigned char c : seen[reinterpret_cast<uintptr_t>(t.data)]) expect(c == 1, "every element once");
    }
};

int main() {
    alignas(16) static unsigned char room[sizeof(Workspace)];
    static float norm;
    static int64_t steps;
    const director_adamw h{1e-3, 0.9, 0.99, 1e-8, 0.0, 1.0};
    for (int n : {0, 1, 5, 63, 64, 65, 199, 200, 201, 361, 481, 700})
        for (long long most : {100ll, 9000ll, 70000ll})
            for (int odd = 0; odd < 2; ++odd) {
                if (n > 201 && most > 9000) continue;
                Set s(n, most, odd, odd && n % 2);
                seen.clear();
                expect(director_grad_norm(n, s.g.data(), &norm, room, nullptr) == DIRECTOR_OK, "norm");
                expect(director_clip_grads(n, s.g.data(), s.out.data(), 1.0f, &norm, room, nullptr) == DIRECTOR_OK, "clip");
                if (!(odd && n % 2)) s.once(s.out), s.once(s.g);
                seen.clear();
                counted = 0;
                expect(director_adamw_step(n, s.g.data(), s.p.data(), &h, nullptr, &steps, &norm, nullptr, room, nullptr) == DIRECTOR_OK, "step");
                expect(counted == 1, "a step is counted once");
                s.once(s.g);
                std::vector<director_tensor> weights;
                for (auto& p : s.p) weights.push_back({p.weight, p.numel, p.type, 0});
                s.once(weights);
            }
    /* each launch of a step of 450 tensors fails in turn: an error, and nothing counted */
    Set s(450, 3000, true, false);
    for (fail_at = 0; fail_at < 10; ++fail_at) {
        launches = counted = 0;
        const int rc = director_adamw_step(450, s.g.data(), s.p.data(), &h, nullptr, &steps, &norm, nullptr, room, nullptr);
        if (rc == DIRECTOR_OK) break;
        expect(rc == DIRECTOR_ERR_CUDA && counted == 0, "a failed step is not counted");
    }
    expect(fail_at >= 4 && fail_at < 10, "norm, finish and the tables of weights");
    printf("norm %d cluster %d finish %d clip %d/%d update %d/%d, %d bad\n", norms, clusters, finishes, clips, small_clips, updates, small_updates, bad);
    return bad != 0 || !norms || !clusters || !finishes || !clips || !small_clips || !updates || !small_updates;
}
