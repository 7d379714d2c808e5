// From a model's gradients to its next weights: the global norm, clipping by it, and AdamW with the clipping on the way (training; the
// paper serves).  A call takes any number of tensors; their addresses and lengths travel as kernel parameters, a few hundred to a
// launch, so that nothing has to be copied to the device ahead of a call and a captured call keeps its own table.
//
// All of it is HBM-bound elementwise work over the concatenation of the tensors, which is cut into chunks.  A call is
//   the sum of squares, by a grid that fills the GPU once;
//   the norm, by one CTA that joins the partial sums;
//   the elementwise part, a CTA to a chunk: handed out in order, the CTAs under way stay close together in memory (an update of 210 M
//   weights 859 us; by a grid that fills the GPU and takes chunks in turns 1018, with three CTAs an SM instead of four 926).
// Where the chunks are few (kSmallCtas) all of it is one cooperative launch, and the norm alone of small tensors is one cluster's
// (DIRECTOR_SMALL_BYTES): launches are what those cost.
// Sums are joined in a fixed order, so that a call gives the same bits again.
#include "director_common.cuh"

#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

namespace director {

namespace {

constexpr int kThreads = 256;
// CTAs of an SM in the norm's grid (eight, as many as an SM holds, read 1.41 G bf16 gradients in 414 us, six in 393), and CTAs of a grid
// at most, one partial sum each.
constexpr int kNormCtas = 6, kSlots = 1024;
constexpr int kNormUnroll = 4;                   // 16-byte loads of a thread and chunk of the norm
constexpr int kClusterCtas = 16, kClusterThreads = 1024, kClusterUnroll = 8;
constexpr int kChunk = kThreads * 8;             // elements of a chunk of the update
constexpr int kClipUnroll = 4, kClipChunk = kThreads * 8 * kClipUnroll;
// CTAs of an SM, and so chunks, up to which norm and elementwise part are one cooperative launch.  Against three launches, four tensors:
// a step of 0.26 M weights 7.9 and 13.1 us a call (6.5 and 7.2 from a graph), of 0.5 M 8.6 and 13.2 (7.9 both); clipping of 1 M 9.7 and
// 15.5.  With four CTAs an SM a step of 1 M (512 chunks) would take 10.3 instead of 13.1 us a call, but 9.4 instead of 9.3 from a graph.
constexpr int kSmallCtas = 2;
constexpr long long kMostElements = 1ll << 40;   // of a tensor
constexpr int kMostTensors = 1 << 24;            // of a call

// What a call keeps between its launches, in the caller's workspace.
struct Workspace {
    double partial[kSlots];                      // sums of squares
    // What all elements have in common.  Read as one vector through L1: with loads from L2, those of a few hundred thousand CTAs
    // queue up at one line (an update of 603 M weights: 3157 instead of 2640 us).
    float scale;                                 // the clipping factor, kNotFinite for a norm that is none
    float decay, rate, root;                     // AdamW: lr * weight_decay, lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
};

constexpr float kNotFinite = -1.0f;

// chain_prologue() in two halves, for the kernels that come before a norm: they let the next kernel come when their own work is done (at
// their end, where they do not say so themselves), not when it begins.  The CTAs of a norm that comes earlier go where some of its
// predecessor's have left first, more than kNormCtas to an SM and fewer to others, and the SMs stay unevenly filled as long as it runs
// (back to back, 336 tensors 56 us instead of 43, as from a graph; 1.41 G elements 419 instead of 387).
__device__ __forceinline__ void chain_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void chain_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// The tensors of one launch: P arrays of CAP tensors, and the first chunk of each tensor.
template <int P, int CAP>
struct Table {
    void* at[P][CAP];
    long long numel[CAP];
    int first[CAP + 1];
    unsigned char kind[CAP];
    int n;
};
constexpr int kFewTensors = DIRECTOR_SMALL_TENSORS, kNormTensors = 480, kClipTensors = 360, kUpdateTensors = 200;     // about 10 KB each

// The tensor that chunk c lies in.
template <typename TABLE>
__host__ __device__ __forceinline__ int tensor_of(const TABLE& t, int c) {
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

// the sum over the lanes in each of them, and over the CTA in every thread; in a fixed order
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
template <int THREADS>
__device__ __forceinline__ double block_sum(double v) {
    __shared__ double s_part[THREADS / 32];
    v = warp_sum(v);
    if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = v;
    __syncthreads();
    if constexpr (THREADS > 256) {
        const int lane = threadIdx.x & 31;
        return warp_sum(lane < THREADS / 32 ? s_part[lane] : 0.0);
    } else {                                               // of eight, faster than five shuffles
        double sum = 0.0;
#pragma unroll
        for (int w = 0; w < THREADS / 32; ++w) sum += s_part[w];
        return sum;
    }
}

// ---- the sum of squares --------------------------------------------------------------------------------------------
//
// A thread squares and adds up to 32 elements in fp32 and carries the sum in fp64 from there.  Where that fp32 sum shows that squares
// left the range - it is infinite, or so small that some may have vanished - the same elements are summed in fp64.

constexpr float kSquaresLowest = 1e-26f, kSquaresHighest = 3e38f;

__device__ __forceinline__ double squares_of(const float (&v)[8]) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf(v[i], v[i], s);
    if (s >= kSquaresLowest && s <= kSquaresHighest) return (double)s;
    double d = 0.0;                                        // as in far_squares
#pragma unroll
    for (int i = 0; i < 8; ++i) d = fma((double)v[i], (double)v[i], d);
    return d;
}

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
inline long long norm_chunks(const void* p, long long n, int per) {
    const long long vecs = (n - head_of<T>(p, n)) / (16 / (int)sizeof(T));
    return n == 0 ? 0 : vecs == 0 ? 1 : (vecs + per - 1) / per;
}

// The same four vectors once more in fp64, all zeros apart (an expert without tokens, the places behind a tensor's end).  They are
// read again and out of line, so that the common way has the registers.
template <typename T>
__device__ __noinline__ double far_squares(const uint4* q, long long v, int step, long long vecs) {
    constexpr uint32_t kMagnitude = sizeof(T) == 2 ? 0x7FFF7FFFu : 0x7FFFFFFFu;
    double sum = 0.0;
    for (int u = 0; u < 4 && v < vecs; ++u, v += step) {
        const uint4 x = __ldg(q + v);
        if (((x.x | x.y | x.z | x.w) & kMagnitude) == 0) continue;
#pragma unroll
        for (int i = 0; i < 16 / (int)sizeof(T); ++i) {
            const double e = (double)element<T>(x, i);
            sum = fma(e, e, sum);
        }
    }
    return sum;
}

// What a thread of a CTA of THREADS adds for chunk `chunk` of a tensor: UNROLL 16-byte loads, a multiple of four.
template <typename T, int THREADS, int UNROLL>
__device__ __forceinline__ double squares_of_chunk(const T* __restrict__ p, long long n, int chunk) {
    constexpr int kPer = 16 / sizeof(T);
    const int tid = threadIdx.x;
    const long long head = head_of<T>(p, n), vecs = (n - head) / kPer;
    const uint4* q = reinterpret_cast<const uint4*>(p + head);
    const long long v0 = (long long)chunk * (THREADS * UNROLL) + tid;
    uint4 x[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u)
        x[u] = v0 + u * THREADS < vecs ? __ldg(q + v0 + u * THREADS) : make_uint4(0u, 0u, 0u, 0u);
    double sum = 0.0;
    if (chunk == 0) {                                      // the ragged ends: fewer than kPer elements each
        const int tail = (int)(n - head - vecs * kPer);
        float v = 0.0f;
        if (tid < head) v = to_float(p[tid]);
        else if (tid >= 32 && tid < 32 + tail) v = to_float(p[n - tail + tid - 32]);
        sum = (double)v * (double)v;
    }
#pragma unroll
    for (int u0 = 0; u0 < UNROLL; u0 += 4) {               // up to 32 elements
        float s = 0.0f;
#pragma unroll
        for (int u = u0; u < u0 + 4; ++u)
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const float v = element<T>(x[u], i);
                s = fmaf(v, v, s);
            }
        if (s >= kSquaresLowest && s <= kSquaresHighest) {
            sum += (double)s;
            continue;
        }
        sum += far_squares<T>(q, v0 + u0 * THREADS, THREADS, vecs);
    }
    return sum;
}

// What CTA `cta` of `ctas` has of the table: every ctas-th chunk.
template <int THREADS, int UNROLL, typename TABLE>
__device__ __forceinline__ double squares_of_table(const TABLE& t, int cta, int ctas) {
    double sum = 0.0;
    const int chunks = t.first[t.n];
    for (int c = cta; c < chunks;) {
        const int k = tensor_of(t, c), first = t.first[k], end = t.first[k + 1];
        const long long n = t.numel[k];
        if (t.kind[k] == DIRECTOR_BF16) {
            const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(t.at[0][k]);
            for (; c < end; c += ctas) sum += squares_of_chunk<__nv_bfloat16, THREADS, UNROLL>(p, n, c - first);
        } else {
            const float* p = static_cast<const float*>(t.at[0][k]);
            for (; c < end; c += ctas) sum += squares_of_chunk<float, THREADS, UNROLL>(p, n, c - first);
        }
    }
    return sum;
}

// What a call makes of the norm.  A step (AdamW) is started by the call's first launch and counted by its last one, so that a call
// whose later launches fail has not counted it.
struct Call {
    Workspace* ws;
    float* norm;                 // or NULL
    double max_norm;
    long long* steps;            // AdamW; NULL: clipping
    double lr, beta1, beta2, weight_decay;
    const float* lr_dev;
    int32_t* status;
};

// beta^t by squaring.  Every rounding grows with the powers taken of it, to t 2^-53 of the result at most, and t beta^t is below
// 1 / (1 - beta): 1 - beta^t is good to 1e-12 for any t and any beta below 0.9999.  pow() takes 0.4 to 0.7 us longer, of a step's 7.
__device__ __forceinline__ double power(double beta, long long t) {
    double r = 1.0;
    for (; t > 0; t >>= 1, beta *= beta)
        if (t & 1) r *= beta;
    return r;
}
__device__ __forceinline__ void start_step(const Call& q) {
    const long long t = *q.steps + 1;
    const double lr = q.lr_dev != nullptr ? (double)*q.lr_dev : q.lr;
    q.ws->decay = (float)(lr * q.weight_decay);
    q.ws->rate = (float)(lr / (1.0 - power(q.beta1, t)));
    q.ws->root = (float)(1.0 / sqrt(1.0 - power(q.beta2, t)));
}
__device__ __forceinline__ float scale_of(const Call& q, double norm) {
    return !isfinite((float)norm) ? kNotFinite : norm > q.max_norm ? (float)(q.max_norm / norm) : 1.0f;
}
__device__ __forceinline__ void finish(const Call& q, double norm) {
    if (q.norm != nullptr) *q.norm = (float)norm;
    if (q.steps != nullptr && q.status != nullptr && !isfinite((float)norm)) director_set_status(q.status, DIRECTOR_ERR_NONFINITE);
}
// One thread of the call's last launch, which nobody else reads *q.steps in; a norm that is not finite: the step is not taken.
__device__ __forceinline__ void count_step(const Call& q, float scale) {
    if (scale != kNotFinite) *q.steps += 1;
}

// The sum of squares: one read of the gradients, HBM-bound.  Four 16-byte loads a thread are under way, a chunk of 16 KB a CTA; 1.41 G
// bf16 gradients take 387 us, 7.3 TB/s (a CTA to a chunk would leave 172 thousand sums to join).
// Partial sum blockIdx.x of the workspace, added to it where an earlier launch of the call has written it (blockIdx.x < filled).
__global__ void __launch_bounds__(kThreads, kNormCtas)
norm_kernel(const __grid_constant__ Table<1, kNormTensors> t, const Call q, int filled) {
    chain_wait();
    if (filled == 0 && q.steps != nullptr && blockIdx.x == gridDim.x - 1 && threadIdx.x == kThreads - 1) start_step(q);
    const double sum = block_sum<kThreads>(squares_of_table<kThreads, kNormUnroll>(t, blockIdx.x, gridDim.x));
    chain_release();
    double* const mine = q.ws->partial + blockIdx.x;
    if (threadIdx.x == 0) *mine = (int)blockIdx.x < filled ? *mine + sum : sum;
}

__device__ __forceinline__ double norm_of_slots(const Workspace* ws, int slots) {
    double v = 0.0;
    for (int i = threadIdx.x; i < slots; i += kThreads) v += __ldcg(&ws->partial[i]);
    return sqrt(block_sum<kThreads>(v));
}

// The norm from the partial sums; with none of them: a norm of 0, and the step is started here.  last: no launch of the call follows.
__global__ void __launch_bounds__(kThreads) finish_kernel(const Call q, int slots, bool last) {
    chain_wait();
    const double norm = norm_of_slots(q.ws, slots);
    if (threadIdx.x != 0) return;
    if (slots == 0 && q.steps != nullptr) start_step(q);
    const float scale = scale_of(q, norm);
    q.ws->scale = scale;
    finish(q, norm);
    if (last && q.steps != nullptr) count_step(q, scale);
}

// The norm alone of small tensors: the CTAs of one cluster hand their sums to its first through distributed shared memory - one
// launch instead of two, and no workspace.  Sixteen SMs read little: 1 MB takes 4.5 us and 4 MB 5.9 us from a graph, where the two
// launches take 3.8 and 4.2, but 6.6 instead of 11.1 us a call.
__global__ void __cluster_dims__(kClusterCtas, 1, 1) __launch_bounds__(kClusterThreads, 1)
norm_cluster_kernel(const __grid_constant__ Table<1, kFewTensors> t, float* norm) {
    __shared__ double s_sums[kClusterCtas];
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    chain_prologue();
    const double sum = block_sum<kClusterThreads>(squares_of_table<kClusterThreads, kClusterUnroll>(t, blockIdx.x, kClusterCtas));
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");      // every CTA of the cluster is there
    if (threadIdx.x == 0) {
        uint32_t at;
        const uint32_t mine = (uint32_t)__cvta_generic_to_shared(&s_sums[blockIdx.x]);
        asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(at) : "r"(mine));
        asm volatile("st.shared::cluster.f64 [%0], %1;" :: "r"(at), "d"(sum) : "memory");
    }
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (blockIdx.x == 0 && threadIdx.x < 32) {
        const double v = warp_sum(threadIdx.x < kClusterCtas ? s_sums[threadIdx.x] : 0.0);
        if (threadIdx.x == 0) *norm = (float)sqrt(v);
    }
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
// Elements [lo, hi) of eight, the others zero; `whole`: the address allows whole accesses.
template <typename T>
__device__ __forceinline__ void load_some(const T* p, int lo, int hi, bool whole, float (&v)[8]) {
    if (whole && lo == 0 && hi == 8) {
        load8(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i >= lo && i < hi ? to_float(p[i]) : 0.0f;
}
__device__ __forceinline__ void store_one(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_one(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
template <typename T>
__device__ __forceinline__ void store_some(T* p, int lo, int hi, bool whole, const float (&v)[8]) {
    if (whole && lo == 0 && hi == 8) {
        store8(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i >= lo && i < hi) store_one(p + i, v[i]);
}
// Elements of an array in front of its address that would make whole accesses of it possible from there.
template <typename T>
inline int pad_of(const void* p) { return (int)(reinterpret_cast<uintptr_t>(p) / sizeof(T) % 8); }
inline int pad_of(const void* p, int type) { return type == DIRECTOR_BF16 ? pad_of<__nv_bfloat16>(p) : pad_of<float>(p); }

// kind of a tensor: its types, which addresses allow whole accesses, and how many elements in front of it its first chunk begins
enum { kGradBf16 = 1, kOutBf16 = 2, kGradWhole = 4, kOutWhole = 8, kStateWhole = 16, kPadShift = 5 };

// What all elements have in common: (scale, decay, rate, root) of the workspace.
__device__ __forceinline__ float4 common_of(const Call& q) { return *reinterpret_cast<const float4*>(&q.ws->scale); }

// The chunks run backwards: the norm has read the last tensors last, and what of them is still in L2 is not fetched again.
struct Place {
    int k, kind;                 // tensor
    long long at, end;           // the chunk's first element (negative in front of the tensor), and the tensor's end from there
    __host__ __device__ bool full(int chunk) const { return at >= 0 && end >= chunk; }
    // of the eight elements at e, those of the tensor: [lo, hi)
    __host__ __device__ int lo(int e) const { return at + e >= 0 ? 0 : at + e > -8 ? (int)-(at + e) : 8; }
    __host__ __device__ int hi(int e) const { return end - e >= 8 ? 8 : end > e ? (int)(end - e) : 0; }
};
template <typename TABLE>
__host__ __device__ __forceinline__ Place place_of(const TABLE& t, int c, int chunk) {
    const int k = tensor_of(t, c);
    const long long at = (long long)(c - t.first[k]) * chunk - (t.kind[k] >> kPadShift);
    return {k, t.kind[k], at, t.numel[k] - at};
}

// The norm inside a cooperative launch: a CTA sums the squares of its chunk, and every CTA joins the partial sums behind the grid's
// barrier.  Array 0 of the table holds the gradients.
template <typename T, int UNROLL>
__device__ __forceinline__ double squares_of_place(const void* grad, const Place& p) {
    const T* g = static_cast<const T*>(grad) + p.at;
    const bool whole = p.kind & kGradWhole, full = whole && p.full(UNROLL * kThreads * 8);
    float v[UNROLL][8];
    if (full) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) load8(g + (u * kThreads + threadIdx.x) * 8, v[u]);
    } else {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int e = (u * kThreads + threadIdx.x) * 8;
            load_some(g + e, p.lo(e), p.hi(e), whole, v[u]);
        }
    }
    double sum = 0.0;
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) sum += squares_of(v[u]);
    return sum;
}
template <int UNROLL, typename TABLE>
__device__ __forceinline__ double norm_in_launch(const TABLE& t, const Call& q, const Place& p) {
    double sum = (p.kind & kGradBf16) ? squares_of_place<__nv_bfloat16, UNROLL>(t.at[0][p.k], p) : squares_of_place<float, UNROLL>(t.at[0][p.k], p);
    if (q.steps != nullptr && blockIdx.x == gridDim.x - 1 && threadIdx.x == kThreads - 1) start_step(q);
    sum = block_sum<kThreads>(sum);
    if (threadIdx.x == 0) q.ws->partial[blockIdx.x] = sum;
    cooperative_groups::this_grid().sync();
    const double norm = norm_of_slots(q.ws, gridDim.x);
    if (blockIdx.x == 0 && threadIdx.x == 0) finish(q, norm);
    return norm;
}

// ---- clipping ------------------------------------------------------------------------------------------------------

// One read and one write, HBM-bound, with the norm's read before it: 571 M bf16 gradients to fp32 in 680 us, 156 of them the norm's; the
// rest moves 3.43 GB at 6.5 TB/s.  Chunks of 4096 elements 692 us, of 2048 892: a CTA then has too few bytes under way.
// A chunk: kClipUnroll x eight elements a thread, asked for together.  FULL: all of them exist, and go out whole; SW: and come in whole.
template <bool FULL, bool SW, typename S, typename D>
__device__ __forceinline__ void clip_chunk(const S* src, D* dst, const Place& p, float scale) {
    float v[kClipUnroll][8];
#pragma unroll
    for (int u = 0; u < kClipUnroll; ++u) {
        const int e = (u * kThreads + threadIdx.x) * 8;
        if (FULL && SW) load8(src + e, v[u]);
        else if (FULL) load_some(src + e, 0, 8, false, v[u]);
        else load_some(src + e, p.lo(e), p.hi(e), p.kind & kGradWhole, v[u]);
    }
    const bool same = scale == kNotFinite || scale == 1.0f;
    if (same && static_cast<const void*>(src) == dst) return;
#pragma unroll
    for (int u = 0; u < kClipUnroll; ++u) {
        const int e = (u * kThreads + threadIdx.x) * 8;
        if (!same)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[u][i] *= scale;
        if (FULL) store8(dst + e, v[u]);
        else store_some(dst + e, p.lo(e), p.hi(e), p.kind & kOutWhole, v[u]);
    }
}
template <typename S, typename D>
__device__ __forceinline__ void clip_any(const void* src, void* dst, const Place& p, float scale) {
    const S* s = static_cast<const S*>(src) + p.at;
    D* d = static_cast<D*>(dst) + p.at;
    const bool full = p.full(kClipChunk) && (p.kind & kOutWhole);
    if (full && (p.kind & kGradWhole)) clip_chunk<true, true>(s, d, p, scale);
    else if (full) clip_chunk<true, false>(s, d, p, scale);
    else clip_chunk<false, false>(s, d, p, scale);
}

template <typename TABLE>
__device__ __forceinline__ void clip_place(const TABLE& t, const Place& p, float scale) {
    const void* src = t.at[0][p.k];
    void* dst = t.at[1][p.k];
    if (p.kind & kGradBf16) {
        if (p.kind & kOutBf16) clip_any<__nv_bfloat16, __nv_bfloat16>(src, dst, p, scale);
        else clip_any<__nv_bfloat16, float>(src, dst, p, scale);
    } else {
        if (p.kind & kOutBf16) clip_any<float, __nv_bfloat16>(src, dst, p, scale);
        else clip_any<float, float>(src, dst, p, scale);
    }
}

__global__ void __launch_bounds__(kThreads, 4)
clip_kernel(const __grid_constant__ Table<2, kClipTensors> t, const Call q, bool in_place) {
    chain_wait();
    const float scale = common_of(q).x;
    if (in_place && (scale == kNotFinite || scale == 1.0f)) return;
    clip_place(t, place_of(t, gridDim.x - 1 - blockIdx.x, kClipChunk), scale);
}

// Few chunks: norm and clipping in one cooperative launch.
__global__ void __launch_bounds__(kThreads, kSmallCtas)
clip_small_kernel(const __grid_constant__ Table<2, kFewTensors> t, const Call q) {
    const Place p = place_of(t, blockIdx.x, kClipChunk);
    clip_place(t, p, scale_of(q, norm_in_launch<kClipUnroll>(t, q, p)));
}

// ---- AdamW ---------------------------------------------------------------------------------------------------------

struct Betas {
    float beta1, rest1, beta2, rest2, eps;                 // rest = 1 - beta
};
struct Arrays {
    const void* grad;
    void* weight;
    float *master, *exp_avg, *exp_avg_sq;
};

// Four arrays read, four written, 28 bytes a bf16 weight, HBM-bound: 604 M weights in 2630 us with the norm (170 us), 6.87 TB/s.  Eight
// elements a thread and not more: 112 bytes under way are enough at 1024 threads an SM, and the registers are full.
// A chunk: eight elements a thread.  FULL: all of them exist and the state's addresses allow whole accesses; GW, WW: the gradient's and
// the weight's do.
template <bool FULL, bool GW, bool WW, typename G, typename W>
__device__ __forceinline__ void update_chunk(const Arrays& a, const Place& p, float4 common, const Betas& b) {
    constexpr bool kMaster = sizeof(W) == 2;
    const int e = threadIdx.x * 8;
    const long long at = p.at + e;
    const int hi = FULL ? 8 : p.hi(e);
    const bool state = FULL || (p.kind & kStateWhole), grad = FULL ? GW : (p.kind & kGradWhole) != 0, weight = FULL ? WW : (p.kind & kOutWhole) != 0;
    const float scale = common.x, decay = common.y, rate = common.z, root = common.w;
    float g[8], w[8], m[8], v[8];
    load_some(a.exp_avg + at, 0, hi, state, m);
    load_some(a.exp_avg_sq + at, 0, hi, state, v);
    if (kMaster) load_some(a.master + at, 0, hi, state, w);
    else load_some(static_cast<const float*>(a.weight) + at, 0, hi, weight, w);
    load_some(static_cast<const G*>(a.grad) + at, 0, hi, grad, g);
    if (scale == kNotFinite) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x = g[i] * scale;
        m[i] = fmaf(b.beta1, m[i], b.rest1 * x);
        v[i] = fmaf(b.beta2, v[i], b.rest2 * x * x);
        w[i] = fmaf(-decay, w[i], w[i]) - rate * m[i] / fmaf(sqrtf(v[i]), root, b.eps);
    }
    store_some(a.exp_avg + at, 0, hi, state, m);
    store_some(a.exp_avg_sq + at, 0, hi, state, v);
    if (kMaster) store_some(a.master + at, 0, hi, state, w);
    store_some(static_cast<W*>(a.weight) + at, 0, hi, weight, w);
}
template <typename G, typename W>
__device__ __forceinline__ void update_any(const Arrays& a, const Place& p, float4 common, const Betas& b) {
    const bool gw = p.kind & kGradWhole, ww = p.kind & kOutWhole;
    if (!p.full(kChunk) || !(p.kind & kStateWhole)) update_chunk<false, false, false, G, W>(a, p, common, b);
    else if (gw && ww) update_chunk<true, true, true, G, W>(a, p, common, b);
    else if (ww) update_chunk<true, false, true, G, W>(a, p, common, b);
    else if (gw) update_chunk<true, true, false, G, W>(a, p, common, b);
    else update_chunk<true, false, false, G, W>(a, p, common, b);
}

template <typename TABLE>
__device__ __forceinline__ void update_place(const TABLE& t, const Place& p, float4 common, const Betas& b) {
    const Arrays a{t.at[0][p.k], t.at[1][p.k], static_cast<float*>(t.at[2][p.k]), static_cast<float*>(t.at[3][p.k]),
                   static_cast<float*>(t.at[4][p.k])};
    if (p.kind & kGradBf16) {
        if (p.kind & kOutBf16) update_any<__nv_bfloat16, __nv_bfloat16>(a, p, common, b);
        else update_any<__nv_bfloat16, float>(a, p, common, b);
    } else {
        if (p.kind & kOutBf16) update_any<float, __nv_bfloat16>(a, p, common, b);
        else update_any<float, float>(a, p, common, b);
    }
}

__global__ void __launch_bounds__(kThreads, 4)
update_kernel(const __grid_constant__ Table<5, kUpdateTensors> t, const Call q, const Betas b, bool last) {
    chain_wait();
    const float4 common = common_of(q);
    if (last && blockIdx.x == 0 && threadIdx.x == 0) count_step(q, common.x);
    update_place(t, place_of(t, gridDim.x - 1 - blockIdx.x, kChunk), common, b);
}

// Few chunks: norm and step in one cooperative launch.
__global__ void __launch_bounds__(kThreads, kSmallCtas)
update_small_kernel(const __grid_constant__ Table<5, kFewTensors> t, const Call q, const Betas b) {
    const Place p = place_of(t, blockIdx.x, kChunk);
    const double norm = norm_in_launch<1>(t, q, p);
    float4 common = common_of(q);
    common.x = scale_of(q, norm);
    if (blockIdx.x == 0 && threadIdx.x == 0) count_step(q, common.x);
    update_place(t, p, common, b);
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
    if (n > kMostTensors) return DIRECTOR_ERR_UNSUPPORTED;
    for (int i = 0; i < n; ++i) {
        if (!valid_array(g[i].data, g[i].numel, g[i].type)) return DIRECTOR_ERR_INVALID_ARG;
        if (g[i].numel > kMostElements) return DIRECTOR_ERR_UNSUPPORTED;
    }
    return DIRECTOR_OK;
}

template <typename... KArgs>
cudaError_t launch_as(bool cooperative, void (*kernel)(KArgs...), unsigned grid, unsigned threads, cudaStream_t st, const KArgs&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    if (cooperative) {
        attr[0].id = cudaLaunchAttributeCooperative;
        attr[0].val.cooperative = 1;
    } else {
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
    }
    cfg.attrs = attr;
    cfg.numAttrs = cooperative || chain_allowed(st) ? 1 : 0;
    void* at[] = {const_cast<void*>(static_cast<const void*>(&args))...};      // the tables are copied once, by the runtime
    return cudaLaunchKernelExC(&cfg, reinterpret_cast<const void*>(kernel), at);
}
template <typename... KArgs>
cudaError_t launch(void (*kernel)(KArgs...), unsigned grid, unsigned threads, cudaStream_t st, const KArgs&... args) {
    return launch_as(false, kernel, grid, threads, st, args...);
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

// Whether one cluster takes the sum of squares.
bool in_one_cluster(int n, const director_tensor* g) {
    if (n > kFewTensors) return false;
    long long bytes = 0;
    for (int i = 0; i < n; ++i) {
        if (g[i].numel > DIRECTOR_SMALL_BYTES) return false;
        bytes += g[i].numel * (long long)width_of(g[i].type);
    }
    return bytes <= DIRECTOR_SMALL_BYTES;
}

template <int CAP, typename Run>
int norm_tables(int n, const director_tensor* g, int per, Run&& run) {
    return in_tables<Table<1, CAP>, CAP>(
        n,
        [&](int i) {
            return g[i].type == DIRECTOR_BF16 ? norm_chunks<__nv_bfloat16>(g[i].data, g[i].numel, per)
                                              : norm_chunks<float>(g[i].data, g[i].numel, per);
        },
        [&](Table<1, CAP>& t, int k, int i) {
            t.at[0][k] = g[i].data;
            t.numel[k] = g[i].numel;
            t.kind[k] = (unsigned char)g[i].type;
        },
        run);
}

bool sm_count(int* out) {
    int dev = 0;
    return cudaGetDevice(&dev) == cudaSuccess && cudaDeviceGetAttribute(out, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess;
}

// Leaves *slots partial sums in the workspace.
int sum_squares(int n, const director_tensor* g, const Call& q, int* slots, cudaStream_t st) {
    int sms = 0;
    if (!sm_count(&sms)) return DIRECTOR_ERR_CUDA;
    *slots = 0;
    return norm_tables<kNormTensors>(n, g, kThreads * kNormUnroll, [&](const Table<1, kNormTensors>& t, int chunks, bool) {
        const int grid = std::max(1, std::min({chunks, kNormCtas * sms, kSlots}));
        const cudaError_t e = launch(norm_kernel, (unsigned)grid, kThreads, st, t, q, *slots);
        *slots = std::max(*slots, grid);
        return cuda_status(e);
    });
}

int finish_call(const Call& q, int slots, bool last, cudaStream_t st) {
    return cuda_status(launch(finish_kernel, 1u, kThreads, st, q, slots, last));
}

// The norm, finished.
int take_norm(int n, const director_tensor* g, const Call& q, bool last, cudaStream_t st) {
    int slots = 0;
    const int rc = sum_squares(n, g, q, &slots, st);
    return rc != DIRECTOR_OK ? rc : finish_call(q, slots, last, st);
}

// Whether the norm and the elementwise part, of chunks_of(i) chunks a tensor, go into one launch: all CTAs run at once.
template <typename Chunks>
bool in_one_launch(int n, Chunks&& chunks_of) {
    int sms = 0;
    if (n > kFewTensors || !sm_count(&sms)) return false;
    long long chunks = 0;
    for (int i = 0; i < n; ++i) chunks += chunks_of(i);
    return chunks > 0 && chunks <= std::min(kSmallCtas * sms, kSlots);
}

// Chunks of a gradient to be clipped into `out`: they begin where that allows whole accesses.
long long clip_chunks(const director_tensor& out) {
    return out.numel == 0 ? 0 : (out.numel + pad_of(out.data, out.type) + kClipChunk - 1) / kClipChunk;
}
template <int CAP, typename Run>
int clip_tables(int n, const director_tensor* g, const director_tensor* out, Run&& run) {
    return in_tables<Table<2, CAP>, CAP>(
        n, [&](int i) { return clip_chunks(out[i]); },
        [&](Table<2, CAP>& t, int k, int i) {
            t.at[0][k] = g[i].data;
            t.at[1][k] = out[i].data;
            t.numel[k] = g[i].numel;
            const int pad = pad_of(out[i].data, out[i].type);
            t.kind[k] = (unsigned char)((g[i].type == DIRECTOR_BF16 ? kGradBf16 : 0) | (out[i].type == DIRECTOR_BF16 ? kOutBf16 : 0) |
                                        (pad_of(g[i].data, g[i].type) == pad ? kGradWhole : 0) | kOutWhole | pad << kPadShift);
        },
        run);
}
long long update_chunks(const director_tensor& g) { return (g.numel + kChunk - 1) / kChunk; }
template <int CAP, typename Run>
int update_tables(int n, const director_tensor* g, const director_param* p, Run&& run) {
    return in_tables<Table<5, CAP>, CAP>(
        n, [&](int i) { return update_chunks(g[i]); },
        [&](Table<5, CAP>& t, int k, int i) {
            t.at[0][k] = g[i].data;
            t.at[1][k] = p[i].weight;
            t.at[2][k] = p[i].master;
            t.at[3][k] = p[i].exp_avg;
            t.at[4][k] = p[i].exp_avg_sq;
            t.numel[k] = g[i].numel;
            const bool wb = p[i].type == DIRECTOR_BF16;
            const bool state = pad_of<float>(p[i].exp_avg) == 0 && pad_of<float>(p[i].exp_avg_sq) == 0 && (!wb || pad_of<float>(p[i].master) == 0);
            t.kind[k] = (unsigned char)((g[i].type == DIRECTOR_BF16 ? kGradBf16 : 0) | (wb ? kOutBf16 : 0) | (state ? kStateWhole : 0) |
                                        (pad_of(p[i].weight, p[i].type) == 0 ? kOutWhole : 0) | (pad_of(g[i].data, g[i].type) == 0 ? kGradWhole : 0));
        },
        run);
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
    if (norm == nullptr || !aligned4(norm) || !aligned16(workspace) || (workspace == nullptr && !in_one_cluster(n, grads)))
        return DIRECTOR_ERR_INVALID_ARG;
    const auto apart = [](const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
        const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
        return x + a_bytes <= y || y + b_bytes <= x;
    };
    const size_t room = workspace == nullptr ? 0 : sizeof(Workspace);
    if (room > 0 && !apart(norm, sizeof(float), workspace, room)) return DIRECTOR_ERR_INVALID_ARG;
    for (int i = 0; i < n; ++i) {
        const size_t bytes = (size_t)grads[i].numel * width_of(grads[i].type);
        if (bytes == 0) continue;
        if (!apart(grads[i].data, bytes, norm, sizeof(float)) || (room > 0 && !apart(grads[i].data, bytes, workspace, room)))
            return DIRECTOR_ERR_INVALID_ARG;
    }
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (in_one_cluster(n, grads)) {
        if (cudaFuncSetAttribute(norm_cluster_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return DIRECTOR_ERR_CUDA;
        return norm_tables<kFewTensors>(n, grads, kClusterThreads * kClusterUnroll, [&](const Table<1, kFewTensors>& t, int, bool) {
            return cuda_status(launch(norm_cluster_kernel, kClusterCtas, kClusterThreads, st, t, norm));
        });
    }
    Call q = {};
    q.ws = static_cast<Workspace*>(workspace);
    q.norm = norm;
    return take_norm(n, grads, q, true, st);
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
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    Call q = {};
    q.ws = static_cast<Workspace*>(workspace);
    q.norm = norm;
    q.max_norm = max_norm;
    if (in_one_launch(n, [&](int i) { return clip_chunks(out[i]); }))
        return clip_tables<kFewTensors>(n, grads, out, [&](const Table<2, kFewTensors>& t, int chunks, bool) {
            return cuda_status(launch_as(true, clip_small_kernel, (unsigned)chunks, kThreads, st, t, q));
        });
    rc = take_norm(n, grads, q, false, st);
    if (rc != DIRECTOR_OK) return rc;
    return clip_tables<kClipTensors>(n, grads, out, [&](const Table<2, kClipTensors>& t, int chunks, bool) {
        return chunks == 0 ? DIRECTOR_OK : cuda_status(launch(clip_kernel, (unsigned)chunks, kThreads, st, t, q, out == grads));
    });
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
        if (p.numel > kMostElements) return DIRECTOR_ERR_UNSUPPORTED;
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
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    Call q = {};
    q.ws = static_cast<Workspace*>(workspace);
    q.norm = norm;
    q.max_norm = h->max_norm;
    q.steps = reinterpret_cast<long long*>(steps);
    q.lr = h->lr, q.beta1 = h->beta1, q.beta2 = h->beta2, q.weight_decay = h->weight_decay;
    q.lr_dev = lr;
    q.status = device_status;
    Betas b = {};
    b.beta1 = (float)h->beta1, b.rest1 = (float)(1.0 - h->beta1);
    b.beta2 = (float)h->beta2, b.rest2 = (float)(1.0 - h->beta2);
    b.eps = (float)h->eps;
    bool none = true;                                      // no weight has a gradient
    for (int i = 0; i < n && none; ++i) none = grads[i].numel == 0;
    if (norm != nullptr || std::isfinite(h->max_norm)) {
        if (in_one_launch(n, [&](int i) { return update_chunks(grads[i]); }))
            return update_tables<kFewTensors>(n, grads, params, [&](const Table<5, kFewTensors>& t, int chunks, bool) {
                return cuda_status(launch_as(true, update_small_kernel, (unsigned)chunks, kThreads, st, t, q, b));
            });
        rc = take_norm(n, grads, q, none, st);
    } else {
        rc = finish_call(q, 0, none, st);
    }
    if (rc != DIRECTOR_OK) return rc;
    return update_tables<kUpdateTensors>(n, grads, params, [&](const Table<5, kUpdateTensors>& t, int chunks, bool last) {
        return chunks == 0 ? DIRECTOR_OK : cuda_status(launch(update_kernel, (unsigned)chunks, kThreads, st, t, q, b, last));
    });
}

}  // extern "C"
