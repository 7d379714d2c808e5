// From a model's gradients to its next weights: the global norm, clipping by it, and AdamW with the clipping on the way (training; the
// paper serves).  A call takes any number of tensors; their addresses and lengths travel as kernel parameters, up to kTensors to a
// launch, so that nothing has to be copied to the device ahead of a call and a captured call keeps its own table.
//
// All of it is HBM-bound elementwise work over the concatenation of the tensors.  That is cut into chunks which the CTAs of a grid
// that fills the GPU once take in turn; the sums of squares are joined in a fixed order, so that a call gives the same bits again.
#include "director_common.cuh"

#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

namespace director {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kSlots = 1024;                     // CTAs of the norm's grid at most: one partial sum each
constexpr int kNormUnroll = 4;                   // 16-byte loads of a thread and chunk of the norm
constexpr int kVec = 8;                          // elements of a thread and chunk of the two others
constexpr int kChunk = kThreads * kVec;
constexpr long long kMostElements = 1ll << 40;

// What a call keeps between its launches, in the caller's workspace.
struct Workspace {
    double partial[kSlots];                      // sums of squares
    double bias1, bias2;                         // 1 - beta^t of the step under way
};

// The tensors of one launch: P arrays of CAP tensors, and the first chunk of each tensor.
template <int P, int CAP>
struct Table {
    void* at[P][CAP];
    long long numel[CAP];
    int first[CAP + 1];
    unsigned char kind[CAP];
    int n;
};
constexpr int kFewTensors = 16, kTensors = 160;

// The tensor that chunk c lies in.
template <typename TABLE>
__device__ __forceinline__ int tensor_of(const TABLE& t, int c) {
    int lo = 0, hi = t.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= c) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
}

// the sum over the CTA, in every thread; in a fixed order
__device__ __forceinline__ double block_sum(double v) {
    __shared__ double s_part[kWarps];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = v;
    __syncthreads();
    double sum = 0.0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) sum += s_part[w];
    return sum;
}

// ---- the sum of squares --------------------------------------------------------------------------------------------
//
// A thread squares and adds up to 32 elements in fp32 and carries the sum in fp64 from there.  Where that fp32 sum shows that squares
// left the range - it is infinite, or so small that some may have vanished - the same elements are summed in fp64.

constexpr float kSquaresLowest = 1e-26f, kSquaresHighest = 3e38f;

template <typename T>
__device__ __forceinline__ float element(uint4 v, int i);
template <>
__device__ __forceinline__ float element<float>(uint4 v, int i) {
    return __uint_as_float(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w);
}
template <>
__device__ __forceinline__ float element<__nv_bfloat16>(uint4 v, int i) {
    const uint32_t u = (i >> 1) == 0 ? v.x : (i >> 1) == 1 ? v.y : (i >> 1) == 2 ? v.z : v.w;
    return (i & 1) ? bf16_hi(u) : bf16_lo(u);
}
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }

// elements in front of the first 16-byte boundary
template <typename T>
__host__ __device__ inline long long head_of(const void* p, long long n) {
    const long long head = (long long)(((16u - (unsigned)(reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) / sizeof(T));
    return head < n ? head : n;
}
template <typename T>
inline long long norm_chunks(const void* p, long long n) {
    const long long vecs = (n - head_of<T>(p, n)) / (16 / (int)sizeof(T)), per = kThreads * kNormUnroll;
    return n == 0 ? 0 : vecs == 0 ? 1 : (vecs + per - 1) / per;
}

template <typename T>
__device__ __forceinline__ double squares_of_chunk(const T* __restrict__ p, long long n, int chunk) {
    constexpr int kPer = 16 / sizeof(T);
    const int tid = threadIdx.x;
    const long long head = head_of<T>(p, n), vecs = (n - head) / kPer;
    double sum = 0.0;
    if (chunk == 0) {                                      // the ragged ends: fewer than kPer elements each
        const int tail = (int)(n - head - vecs * kPer);
        float v = 0.0f;
        if (tid < head) v = to_float(p[tid]);
        else if (tid >= 32 && tid < 32 + tail) v = to_float(p[n - tail + tid - 32]);
        sum = (double)v * (double)v;
    }
    const uint4* q = reinterpret_cast<const uint4*>(p + head);
    const long long v0 = (long long)chunk * (kThreads * kNormUnroll) + tid;
    uint4 x[kNormUnroll];
#pragma unroll
    for (int u = 0; u < kNormUnroll; ++u)
        x[u] = v0 + u * kThreads < vecs ? __ldg(q + v0 + u * kThreads) : make_uint4(0u, 0u, 0u, 0u);
    float s = 0.0f;
#pragma unroll
    for (int u = 0; u < kNormUnroll; ++u)
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const float v = element<T>(x[u], i);
            s = fmaf(v, v, s);
        }
    if (s >= kSquaresLowest && s <= kSquaresHighest) return sum + (double)s;
#pragma unroll
    for (int u = 0; u < kNormUnroll; ++u)
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const double v = (double)element<T>(x[u], i);
            sum = fma(v, v, sum);
        }
    return sum;
}

struct StepStart {                               // what the first launch of an AdamW step does besides
    long long* steps;
    double beta1, beta2;
};

__device__ __forceinline__ void start_step(const StepStart& s, Workspace* ws) {
    const long long t = *s.steps + 1;
    *s.steps = t;
    ws->bias1 = 1.0 - pow(s.beta1, (double)t);
    ws->bias2 = 1.0 - pow(s.beta2, (double)t);
}

// Partial sum blockIdx.x of the workspace, added to it where an earlier launch of the call has written it (blockIdx.x < filled).
template <int CAP>
__global__ void __launch_bounds__(kThreads, 4)
norm_kernel(const __grid_constant__ Table<1, CAP> t, Workspace* ws, int filled, const StepStart start) {
    chain_prologue();
    if (start.steps != nullptr && blockIdx.x == 0 && threadIdx.x == 0) start_step(start, ws);
    double sum = 0.0;
    for (int c = blockIdx.x; c < t.first[t.n]; c += gridDim.x) {
        const int k = tensor_of(t, c);
        sum += t.kind[k] == DIRECTOR_BF16
                   ? squares_of_chunk(static_cast<const __nv_bfloat16*>(t.at[0][k]), t.numel[k], c - t.first[k])
                   : squares_of_chunk(static_cast<const float*>(t.at[0][k]), t.numel[k], c - t.first[k]);
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) ws->partial[blockIdx.x] = (int)blockIdx.x < filled ? ws->partial[blockIdx.x] + sum : sum;
}

// The norm from the partial sums, in every thread of the CTA.
__device__ __forceinline__ double norm_of(const Workspace* ws, int slots) {
    double v = 0.0;
    for (int i = threadIdx.x; i < slots; i += kThreads) v += __ldcg(&ws->partial[i]);
    return sqrt(block_sum(v));
}

__global__ void __launch_bounds__(kThreads) norm_finish_kernel(const Workspace* ws, int slots, float* norm) {
    chain_prologue();
    const double v = norm_of(ws, slots);
    if (threadIdx.x == 0) *norm = (float)v;
}

__global__ void start_step_kernel(Workspace* ws, const StepStart start) {
    chain_prologue();
    start_step(start, ws);
}

// ---- eight elements ------------------------------------------------------------------------------------------------
//
// fp32 elements move as one 32-byte access, bf16 as one of 16 bytes, where the address allows it.

__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]) : "l"(p) : "memory");
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&v)[8]) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    v[0] = bf16_lo(u.x), v[1] = bf16_hi(u.x), v[2] = bf16_lo(u.y), v[3] = bf16_hi(u.y);
    v[4] = bf16_lo(u.z), v[5] = bf16_hi(u.z), v[6] = bf16_lo(u.w), v[7] = bf16_hi(u.w);
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    asm volatile("st.global.v8.f32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                 :: "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "l"(p) : "memory");
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}
template <typename T>
__device__ __forceinline__ void load_some(const T* p, int n, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? to_float(p[i]) : 0.0f;
}
__device__ __forceinline__ void store_one(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_one(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
template <typename T>
__device__ __forceinline__ void store_some(T* p, int n, const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) store_one(p + i, v[i]);
}
template <typename T>
inline bool whole(const void* p) { return (reinterpret_cast<uintptr_t>(p) & (8 * sizeof(T) - 1)) == 0; }

// kind bits of a tensor: its types, and which addresses allow whole accesses
enum { kGradBf16 = 1, kOutBf16 = 2, kGradWhole = 4, kOutWhole = 8 };

// ---- clipping ------------------------------------------------------------------------------------------------------
//
// The chunks run backwards: the norm has read the last tensors last, and what of them is still in L2 is not fetched again.

template <typename S, typename D>
__device__ __forceinline__ void scale_chunk(const S* src, D* dst, long long n, int chunk, float scale, int kind) {
    const long long at = (long long)chunk * kChunk + threadIdx.x * kVec;
    if (at >= n) return;
    float v[8];
    const int some = (int)min(n - at, 8ll);
    if (some == 8 && (kind & kGradWhole)) load8(src + at, v);
    else load_some(src + at, some, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= scale;
    if (some == 8 && (kind & kOutWhole)) store8(dst + at, v);
    else store_some(dst + at, some, v);
}

template <int CAP>
__global__ void __launch_bounds__(kThreads, 4)
clip_kernel(const __grid_constant__ Table<2, CAP> t, const Workspace* ws, int slots, float max_norm, float* norm) {
    chain_prologue();
    const double total = norm_of(ws, slots);
    const float scale = total > (double)max_norm && isfinite((float)total) ? (float)((double)max_norm / total) : 1.0f;
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)total;
    for (int c = t.first[t.n] - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {
        const int k = tensor_of(t, c), kind = t.kind[k], chunk = c - t.first[k];
        const void* src = t.at[0][k];
        void* dst = t.at[1][k];
        if (scale == 1.0f && src == dst) continue;
        const long long n = t.numel[k];
        if (kind & kGradBf16) {
            if (kind & kOutBf16) scale_chunk(static_cast<const __nv_bfloat16*>(src), static_cast<__nv_bfloat16*>(dst), n, chunk, scale, kind);
            else scale_chunk(static_cast<const __nv_bfloat16*>(src), static_cast<float*>(dst), n, chunk, scale, kind);
        } else {
            if (kind & kOutBf16) scale_chunk(static_cast<const float*>(src), static_cast<__nv_bfloat16*>(dst), n, chunk, scale, kind);
            else scale_chunk(static_cast<const float*>(src), static_cast<float*>(dst), n, chunk, scale, kind);
        }
    }
}

// ---- AdamW ---------------------------------------------------------------------------------------------------------

struct AdamW {
    float beta1, rest1, beta2, rest2, eps, decay;          // rest = 1 - beta, decay = lr * weight_decay
    float scale, rate, root;                               // the clipping factor, lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
};

template <typename G, typename W>
__device__ __forceinline__ void update_chunk(const G* grad, W* weight, float* master, float* exp_avg, float* exp_avg_sq, long long n,
                                             int chunk, const AdamW& a, int kind) {
    const long long at = (long long)chunk * kChunk + threadIdx.x * kVec;
    if (at >= n) return;
    const int some = (int)min(n - at, 8ll);
    const bool all = some == 8 && (kind & kOutWhole);
    float g[8], w[8], m[8], v[8];
    if (some == 8 && (kind & kGradWhole)) load8(grad + at, g);
    else load_some(grad + at, some, g);
    float* const w32 = sizeof(W) == 2 ? master : reinterpret_cast<float*>(weight);
    if (all) {
        load8(exp_avg + at, m);
        load8(exp_avg_sq + at, v);
        load8(w32 + at, w);
    } else {
        load_some(exp_avg + at, some, m);
        load_some(exp_avg_sq + at, some, v);
        load_some(w32 + at, some, w);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x = g[i] * a.scale;
        m[i] = fmaf(a.beta1, m[i], a.rest1 * x);
        v[i] = fmaf(a.beta2, v[i], a.rest2 * x * x);
        w[i] = fmaf(-a.decay, w[i], w[i]) - a.rate * m[i] / fmaf(sqrtf(v[i]), a.root, a.eps);
    }
    if (all) {
        store8(exp_avg + at, m);
        store8(exp_avg_sq + at, v);
        store8(w32 + at, w);
        if (sizeof(W) == 2) store8(weight + at, w);
    } else {
        store_some(exp_avg + at, some, m);
        store_some(exp_avg_sq + at, some, v);
        store_some(w32 + at, some, w);
        if (sizeof(W) == 2) store_some(weight + at, some, w);
    }
}

struct StepRest {
    float beta1, rest1, beta2, rest2, eps;
    double lr, weight_decay, max_norm;
    const float* lr_dev;
    float* norm;
    long long* steps;
    int32_t* status;
    int slots;           // partial sums of the norm; 0: it was not taken
    bool last;           // of the call's launches
};

template <int CAP>
__global__ void __launch_bounds__(kThreads, 4)
update_kernel(const __grid_constant__ Table<5, CAP> t, const Workspace* ws, const StepRest r) {
    chain_prologue();
    AdamW a;
    a.beta1 = r.beta1, a.rest1 = r.rest1, a.beta2 = r.beta2, a.rest2 = r.rest2, a.eps = r.eps;
    a.scale = 1.0f;
    const bool first = blockIdx.x == 0 && threadIdx.x == 0 && r.last;
    if (r.slots > 0) {
        const double total = norm_of(ws, r.slots);
        if (first && r.norm != nullptr) *r.norm = (float)total;
        if (!isfinite((float)total)) {
            if (first) {
                *r.steps -= 1;                             // no other thread of the launch reads it
                if (r.status != nullptr) director_set_status(r.status, DIRECTOR_ERR_NONFINITE);
            }
            return;
        }
        if (total > r.max_norm) a.scale = (float)(r.max_norm / total);
    }
    const double lr = r.lr_dev != nullptr ? (double)__ldg(r.lr_dev) : r.lr;
    a.decay = (float)(lr * r.weight_decay);
    a.rate = (float)(lr / __ldcg(&ws->bias1));
    a.root = (float)(1.0 / sqrt(__ldcg(&ws->bias2)));
    for (int c = t.first[t.n] - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {
        const int k = tensor_of(t, c), kind = t.kind[k], chunk = c - t.first[k];
        const long long n = t.numel[k];
        const void* grad = t.at[0][k];
        void* weight = t.at[1][k];
        float* master = static_cast<float*>(t.at[2][k]);
        float* exp_avg = static_cast<float*>(t.at[3][k]);
        float* exp_avg_sq = static_cast<float*>(t.at[4][k]);
        if (kind & kGradBf16) {
            const __nv_bfloat16* g = static_cast<const __nv_bfloat16*>(grad);
            if (kind & kOutBf16) update_chunk(g, static_cast<__nv_bfloat16*>(weight), master, exp_avg, exp_avg_sq, n, chunk, a, kind);
            else update_chunk(g, static_cast<float*>(weight), master, exp_avg, exp_avg_sq, n, chunk, a, kind);
        } else {
            const float* g = static_cast<const float*>(grad);
            if (kind & kOutBf16) update_chunk(g, static_cast<__nv_bfloat16*>(weight), master, exp_avg, exp_avg_sq, n, chunk, a, kind);
            else update_chunk(g, static_cast<float*>(weight), master, exp_avg, exp_avg_sq, n, chunk, a, kind);
        }
    }
}

// ---- host ----------------------------------------------------------------------------------------------------------

size_t width_of(int type) { return type == DIRECTOR_BF16 ? 2 : 4; }

bool valid_array(const void* p, long long numel, int type) {
    if (numel < 0 || (type != DIRECTOR_FP32 && type != DIRECTOR_BF16)) return false;
    if (numel == 0) return true;
    return p != nullptr && reinterpret_cast<uintptr_t>(p) % width_of(type) == 0;
}

// What a call reads and writes: no array that is written may overlap another of the call.
class Extents {
public:
    explicit Extents(int most) : e_(new (std::nothrow) Extent[most > 0 ? most : 1]) {}
    bool made() const { return e_ != nullptr; }
    void add(const void* p, long long numel, int type, bool written) {
        if (numel == 0) return;
        const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
        e_[n_++] = {lo, lo + (uintptr_t)numel * width_of(type), written};
    }
    bool apart() {
        std::sort(e_.get(), e_.get() + n_, [](const Extent& a, const Extent& b) { return a.lo < b.lo; });
        uintptr_t any = 0, written = 0;                    // ends of what lies before
        for (int i = 0; i < n_; ++i) {
            if (e_[i].lo < (e_[i].written ? any : written)) return false;
            any = std::max(any, e_[i].hi);
            if (e_[i].written) written = std::max(written, e_[i].hi);
        }
        return true;
    }

private:
    struct Extent {
        uintptr_t lo, hi;
        bool written;
    };
    std::unique_ptr<Extent[]> e_;
    int n_ = 0;
};

int check_tensors(int32_t n, const director_tensor* g) {
    if (n < 0 || (n > 0 && g == nullptr)) return DIRECTOR_ERR_INVALID_ARG;
    for (int i = 0; i < n; ++i) {
        if (!valid_array(g[i].data, g[i].numel, g[i].type)) return DIRECTOR_ERR_INVALID_ARG;
        if (g[i].numel > kMostElements) return DIRECTOR_ERR_UNSUPPORTED;
    }
    return DIRECTOR_OK;
}

bool sm_count(int* out) {
    int dev = 0;
    return cudaGetDevice(&dev) == cudaSuccess && cudaDeviceGetAttribute(out, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess;
}

template <typename... KArgs>
cudaError_t launch(void (*kernel)(KArgs...), unsigned grid, unsigned threads, cudaStream_t st, const KArgs&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = chain_allowed(st) ? 1 : 0;
    void* at[] = {const_cast<void*>(static_cast<const void*>(&args))...};      // the tables are copied once, by the runtime
    return cudaLaunchKernelExC(&cfg, reinterpret_cast<const void*>(kernel), at);
}

// Puts the tensors i = 0 .. n-1 that have chunks (chunks_of(i)) into tables (fill(table, slot, i)) and launches each table that is
// full, and the last one even if it is empty: run(table, chunks, last).
template <typename TABLE, int CAP, typename Chunks, typename Fill, typename Run>
int in_tables(int n, Chunks&& chunks_of, Fill&& fill, Run&& run) {
    TABLE t;
    t.n = 0;
    t.first[0] = 0;
    for (int i = 0; i < n; ++i) {
        const long long chunks = chunks_of(i);
        if (chunks == 0) continue;
        if (t.n == CAP || t.first[t.n] + chunks > (1ll << 30)) {
            const int rc = run(t, t.first[t.n], false);
            if (rc != DIRECTOR_OK) return rc;
            t.n = 0;
        }
        fill(t, t.n, i);
        t.first[t.n + 1] = (int)(t.first[t.n] + chunks);
        ++t.n;
    }
    return run(t, t.first[t.n], true);
}

unsigned grid_of(int chunks, int sms) {
    const int most = std::min(4 * sms, kSlots);
    return (unsigned)std::max(1, std::min(chunks, most));
}

// The launches that leave the partial sums in the workspace; *slots: how many.
template <int CAP>
int norm_launches(int n, const director_tensor* g, Workspace* ws, const StepStart& start, int sms, int* slots, cudaStream_t st) {
    *slots = 0;
    StepStart s = start;
    return in_tables<Table<1, CAP>, CAP>(
        n,
        [&](int i) {
            return g[i].type == DIRECTOR_BF16 ? norm_chunks<__nv_bfloat16>(g[i].data, g[i].numel) : norm_chunks<float>(g[i].data, g[i].numel);
        },
        [&](Table<1, CAP>& t, int k, int i) {
            t.at[0][k] = g[i].data;
            t.numel[k] = g[i].numel;
            t.kind[k] = (unsigned char)g[i].type;
        },
        [&](const Table<1, CAP>& t, int chunks, bool) {
            const unsigned grid = grid_of(chunks, sms);
            const cudaError_t e = launch(norm_kernel<CAP>, grid, kThreads, st, t, ws, *slots, s);
            *slots = std::max(*slots, (int)grid);
            s.steps = nullptr;
            return cuda_status(e);
        });
}
int take_norm(int n, const director_tensor* g, Workspace* ws, const StepStart& start, int sms, int* slots, cudaStream_t st) {
    return n <= kFewTensors ? norm_launches<kFewTensors>(n, g, ws, start, sms, slots, st)
                            : norm_launches<kTensors>(n, g, ws, start, sms, slots, st);
}

template <int CAP>
int clip_launches(int n, const director_tensor* g, const director_tensor* out, const Workspace* ws, int slots, float max_norm, float* norm,
                  int sms, cudaStream_t st) {
    return in_tables<Table<2, CAP>, CAP>(
        n, [&](int i) { return (g[i].numel + kChunk - 1) / kChunk; },
        [&](Table<2, CAP>& t, int k, int i) {
            t.at[0][k] = g[i].data;
            t.at[1][k] = out[i].data;
            t.numel[k] = g[i].numel;
            const bool sb = g[i].type == DIRECTOR_BF16, db = out[i].type == DIRECTOR_BF16;
            t.kind[k] = (unsigned char)((sb ? kGradBf16 : 0) | (db ? kOutBf16 : 0) |
                                        ((sb ? whole<__nv_bfloat16>(g[i].data) : whole<float>(g[i].data)) ? kGradWhole : 0) |
                                        ((db ? whole<__nv_bfloat16>(out[i].data) : whole<float>(out[i].data)) ? kOutWhole : 0));
        },
        [&](const Table<2, CAP>& t, int chunks, bool) {
            return cuda_status(launch(clip_kernel<CAP>, grid_of(chunks, sms), kThreads, st, t, ws, slots, max_norm, norm));
        });
}

template <int CAP>
int update_launches(int n, const director_tensor* g, const director_param* p, const Workspace* ws, StepRest rest, int sms, cudaStream_t st) {
    return in_tables<Table<5, CAP>, CAP>(
        n, [&](int i) { return (g[i].numel + kChunk - 1) / kChunk; },
        [&](Table<5, CAP>& t, int k, int i) {
            t.at[0][k] = g[i].data;
            t.at[1][k] = p[i].weight;
            t.at[2][k] = p[i].master;
            t.at[3][k] = p[i].exp_avg;
            t.at[4][k] = p[i].exp_avg_sq;
            t.numel[k] = g[i].numel;
            const bool gb = g[i].type == DIRECTOR_BF16, wb = p[i].type == DIRECTOR_BF16;
            const bool state = whole<float>(p[i].exp_avg) && whole<float>(p[i].exp_avg_sq) &&
                               (wb ? whole<__nv_bfloat16>(p[i].weight) && whole<float>(p[i].master) : whole<float>(p[i].weight));
            t.kind[k] = (unsigned char)((gb ? kGradBf16 : 0) | (wb ? kOutBf16 : 0) | (state ? kOutWhole : 0) |
                                        ((gb ? whole<__nv_bfloat16>(g[i].data) : whole<float>(g[i].data)) ? kGradWhole : 0));
        },
        [&](const Table<5, CAP>& t, int chunks, bool last) {
            rest.last = last;
            return cuda_status(launch(update_kernel<CAP>, grid_of(chunks, sms), kThreads, st, t, ws, rest));
        });
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace

}  // namespace director

using namespace director;

extern "C" {

int64_t director_grad_workspace_bytes(void) { return (int64_t)sizeof(Workspace); }

int director_grad_norm(int32_t n, const director_tensor* grads, float* norm, void* workspace, void* stream) {
    const int rc = check_tensors(n, grads);
    if (rc != DIRECTOR_OK) return rc;
    if (norm == nullptr || !aligned4(norm) || workspace == nullptr || !aligned16(workspace)) return DIRECTOR_ERR_INVALID_ARG;
    int sms = 0, slots = 0;
    if (!sm_count(&sms)) return DIRECTOR_ERR_CUDA;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    Workspace* ws = static_cast<Workspace*>(workspace);
    const int done = take_norm(n, grads, ws, StepStart{}, sms, &slots, st);
    if (done != DIRECTOR_OK) return done;
    return cuda_status(launch(norm_finish_kernel, 1u, kThreads, st, static_cast<const Workspace*>(ws), slots, norm));
}

int director_clip_grads(int32_t n, const director_tensor* grads, const director_tensor* out, float max_norm, float* norm,
                        void* workspace, void* stream) {
    int rc = check_tensors(n, grads);
    if (rc == DIRECTOR_OK && out != nullptr) rc = check_tensors(n, out);
    if (rc != DIRECTOR_OK) return rc;
    if (norm == nullptr || !aligned4(norm) || workspace == nullptr || !aligned16(workspace) || !(max_norm > 0.0f))
        return DIRECTOR_ERR_INVALID_ARG;
    if (out == nullptr) out = grads;
    Extents extents(2 * n + 2);
    if (!extents.made()) return DIRECTOR_ERR_WORKSPACE;
    for (int i = 0; i < n; ++i) {
        if (out[i].numel != grads[i].numel) return DIRECTOR_ERR_INVALID_ARG;
        extents.add(out[i].data, out[i].numel, out[i].type, true);
        if (out[i].data != grads[i].data || out[i].type != grads[i].type) extents.add(grads[i].data, grads[i].numel, grads[i].type, false);
    }
    extents.add(norm, 1, DIRECTOR_FP32, true);
    extents.add(workspace, sizeof(Workspace) / 4, DIRECTOR_FP32, true);
    if (!extents.apart()) return DIRECTOR_ERR_INVALID_ARG;
    int sms = 0, slots = 0;
    if (!sm_count(&sms)) return DIRECTOR_ERR_CUDA;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    Workspace* ws = static_cast<Workspace*>(workspace);
    rc = take_norm(n, grads, ws, StepStart{}, sms, &slots, st);
    if (rc != DIRECTOR_OK) return rc;
    return n <= kFewTensors ? clip_launches<kFewTensors>(n, grads, out, ws, slots, max_norm, norm, sms, st)
                            : clip_launches<kTensors>(n, grads, out, ws, slots, max_norm, norm, sms, st);
}

int director_adamw_step(int32_t n, const director_tensor* grads, const director_param* params, const director_adamw* h,
                        const float* lr, int64_t* steps, float* norm, int32_t* device_status, void* workspace, void* stream) {
    int rc = check_tensors(n, grads);
    if (rc != DIRECTOR_OK) return rc;
    if ((n > 0 && params == nullptr) || h == nullptr || steps == nullptr || (reinterpret_cast<uintptr_t>(steps) & 7u) ||
        !aligned4(lr) || !aligned4(norm) || !aligned4(device_status) || workspace == nullptr || !aligned16(workspace))
        return DIRECTOR_ERR_INVALID_ARG;
    if (!(h->beta1 >= 0.0 && h->beta1 < 1.0) || !(h->beta2 >= 0.0 && h->beta2 < 1.0) || !(h->eps >= 0.0) || !(h->max_norm > 0.0) ||
        !std::isfinite(h->eps) || !std::isfinite(h->weight_decay) || (lr == nullptr && !std::isfinite(h->lr)))
        return DIRECTOR_ERR_INVALID_ARG;
    Extents extents(5 * n + 5);
    if (!extents.made()) return DIRECTOR_ERR_WORKSPACE;
    for (int i = 0; i < n; ++i) {
        const director_param& p = params[i];
        const bool wb = p.type == DIRECTOR_BF16;
        if (!valid_array(p.weight, p.numel, p.type) || !valid_array(p.exp_avg, p.numel, DIRECTOR_FP32) ||
            !valid_array(p.exp_avg_sq, p.numel, DIRECTOR_FP32) || (wb && !valid_array(p.master, p.numel, DIRECTOR_FP32)) ||
            (!wb && p.master != nullptr))
            return DIRECTOR_ERR_INVALID_ARG;
        if (grads[i].numel != p.numel && !(grads[i].numel == 0 && grads[i].data == nullptr)) return DIRECTOR_ERR_INVALID_ARG;
        extents.add(grads[i].data, grads[i].numel, grads[i].type, false);
        extents.add(p.weight, p.numel, p.type, true);
        if (wb) extents.add(p.master, p.numel, DIRECTOR_FP32, true);
        extents.add(p.exp_avg, p.numel, DIRECTOR_FP32, true);
        extents.add(p.exp_avg_sq, p.numel, DIRECTOR_FP32, true);
    }
    extents.add(steps, 2, DIRECTOR_FP32, true);
    if (norm != nullptr) extents.add(norm, 1, DIRECTOR_FP32, true);
    if (lr != nullptr) extents.add(lr, 1, DIRECTOR_FP32, false);
    if (device_status != nullptr) extents.add(device_status, 1, DIRECTOR_FP32, true);
    extents.add(workspace, sizeof(Workspace) / 4, DIRECTOR_FP32, true);
    if (!extents.apart()) return DIRECTOR_ERR_INVALID_ARG;
    int sms = 0;
    if (!sm_count(&sms)) return DIRECTOR_ERR_CUDA;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    Workspace* ws = static_cast<Workspace*>(workspace);
    StepRest rest = {};
    rest.beta1 = (float)h->beta1, rest.rest1 = (float)(1.0 - h->beta1);
    rest.beta2 = (float)h->beta2, rest.rest2 = (float)(1.0 - h->beta2);
    rest.eps = (float)h->eps;
    rest.lr = h->lr, rest.weight_decay = h->weight_decay, rest.max_norm = h->max_norm;
    rest.lr_dev = lr;
    rest.norm = norm;
    rest.steps = reinterpret_cast<long long*>(steps);
    rest.status = device_status;
    const StepStart start{rest.steps, h->beta1, h->beta2};
    if (norm != nullptr || std::isfinite(h->max_norm)) rc = take_norm(n, grads, ws, start, sms, &rest.slots, st);
    else rc = cuda_status(launch(start_step_kernel, 1u, 1u, st, ws, start));
    if (rc != DIRECTOR_OK) return rc;
    return n <= kFewTensors ? update_launches<kFewTensors>(n, grads, params, ws, rest, sms, st)
                            : update_launches<kTensors>(n, grads, params, ws, rest, sms, st);
}

}  // extern "C"
