// The router's balance term (training; the paper balances by placement instead, Section VI): per-expert counts, the loss that pulls
// the router's mean scores towards an even load, and its gradient.
//
//   N valid tokens, f_e = counts_e / (K N), p_t = softmax(logits_t), P_e = sum_t p_te / N:   loss = E sum_e f_e P_e
//   dlogits_te = dloss E/N p_te (f_e - sum_j f_j p_tj)          (the counts are piecewise constant)
//
// A row of up to 256 logits lies in the registers of LPR lanes, sixteen values each, so that a pass over the logits is one read;
// max and sum of the softmax take log2(LPR) shuffles for the 32 / LPR rows that a warp has at a time, and a lane keeps its columns from
// row to row, so that the sums over tokens are adds in registers.  Sixteen and not eight values a lane: half the shuffles (131072 x
// 256, the forward 28 and 30 us).  HBM bounds the large batches, the call the small ones: 131072 tokens, 256 experts, 27 us the forward
// (138 MB, 5.2 TB/s; 3 us of them are the last CTAs' sums) and 44 us the gradient (268 MB, 6.1 TB/s); 8192 tokens, 64 experts, 5.6
// and 3.1 us; 48 tokens, 8 experts, 3.1 and 2.5 us.
#include "director_common.cuh"

#include <cmath>

namespace director {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kVals = 16;
constexpr int kMostPasses = 64;      // rows that a lane sees in one CTA at most: the forward's fp32 sums stay short
// CTAs of the forward that an SM holds, and that the batch is cut for: they all run at once (131072 x 256: 28 us; four and 64 registers
// 28, five 41).  The backward sums nothing, and many small CTAs keep the addresses that are under way close together: 43.8 us with 24
// an SM of which four run, 44.8 with 16, 45.8 with 8, 50 with 4, 47 with 64.
constexpr int kForwardCtas = 3, kBackwardCtas = 24;

// The expert of a lane's value i: groups of four LPR groups apart where a row can be read in 16-byte words, values LPR apart where
// it cannot, so that the lanes of a row touch neighbours in either case.
template <int LPR, bool VEC>
__device__ __forceinline__ int expert_of(int i, int sub) {
    return VEC ? 4 * ((i / 4) * LPR + sub) + i % 4 : i * LPR + sub;
}

// The sixteen values of lane `sub` of its row, -inf behind the last expert.
template <int LPR, bool VEC>
__device__ __forceinline__ void load_row(const float* __restrict__ row, int E, int sub, float (&x)[kVals]) {
#pragma unroll
    for (int j = 0; j < kVals / 4; ++j) {
        if (VEC) {
            const int e = 4 * (j * LPR + sub);
            const float4 v = e < E ? __ldg(reinterpret_cast<const float4*>(row + e)) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
            x[4 * j] = v.x, x[4 * j + 1] = v.y, x[4 * j + 2] = v.z, x[4 * j + 3] = v.w;
        } else {
#pragma unroll
            for (int i = 4 * j; i < 4 * j + 4; ++i) {
                const int e = expert_of<LPR, VEC>(i, sub);
                x[i] = e < E ? __ldg(row + e) : -INFINITY;
            }
        }
    }
}

__device__ __forceinline__ float power_of_two(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// x -> exp(x - max), up to a factor that all have in common; returns their sum, NaN for a row with a NaN, a +inf or nothing but
// -inf.  One product and one power of two: 2^(x log2(e) - max log2(e)).  The second product's rounding, 2^-24 of it, is the common
// factor's exponent, which has to stay small; the difference's is 2^-24 of the distance from the maximum, in the exponent: what it moves
// is as small as exp(-distance).
template <int LPR>
__device__ __forceinline__ float softmax_terms(float (&x)[kVals]) {
    constexpr float kLog2E = 1.4426950408889634f;
    float m = x[0];
#pragma unroll
    for (int i = 1; i < kVals; ++i) m = fmaxf(m, x[i]);
#pragma unroll
    for (int o = 1; o < LPR; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    if (fabsf(m) > 1e6f) {                                 // the common factor would be more than 2^0.1 from one
#pragma unroll
        for (int i = 0; i < kVals; ++i) x[i] -= m;
        m -= m;
    }
    m *= kLog2E;
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < kVals; ++i) {
        x[i] = power_of_two(fmaf(x[i], kLog2E, -m));
        s += x[i];
    }
#pragma unroll
    for (int o = 1; o < LPR; o <<= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    return s;
}

// Loss and counts.  A CTA sums its tokens' p in registers (fp32, at most kMostPasses rows a lane), then over lanes and warps (the
// latter in fp64), and adds the sums to the context's 64-bit integers as fixed point (2^`shift` to one; T 2^shift < 2^62), whose
// order makes no difference: the loss has the same bits on every run.  The last CTA to arrive writes the results and leaves zeros.
struct BalanceSums {
    unsigned long long p[kMaxE];
    unsigned long long count[kMaxE + 1];     // [kMaxE]: valid tokens
    unsigned int ticket;
};

template <int LPR, bool VEC>
__global__ void __launch_bounds__(kThreads, kForwardCtas)
balance_loss_kernel(const float* __restrict__ logits, const int32_t* __restrict__ topk_idx, const uint8_t* __restrict__ mask, int T,
                    int E, int K, int rows, int shift, BalanceSums* __restrict__ sums, float* __restrict__ loss,
                    int64_t* __restrict__ counts, int32_t* status) {
    constexpr int kGroups = 32 / LPR;                      // rows a warp has at a time
    __shared__ float s_p[kWarps][LPR * kVals];
    __shared__ int s_count[kMaxE + 1];
    __shared__ double s_term[kWarps];
    __shared__ bool s_last;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane % LPR;
    for (int e = tid; e <= kMaxE; e += kThreads) s_count[e] = 0;
    chain_prologue();
    __syncthreads();
    const int r0 = blockIdx.x * rows, n_rows = min(rows, T - r0);

    float acc[kVals] = {}, next[kVals] = {};
    int valid = 0;
    const auto fetch = [&](int base) {                     // the lane's part of its row of the pass at `base`
        const int row = r0 + base + lane / LPR;
        const bool live = base + lane / LPR < n_rows && (mask == nullptr || __ldg(mask + row) != 0);
        if (live) load_row<LPR, VEC>(logits + (size_t)row * E, E, sub, next);
        return live;
    };
    bool next_live = fetch(warp * kGroups);

    // The counts, four choices a thread and pass, fetched a pass ahead like the rows.  r0 is a multiple of four, so that a CTA's
    // choices start on 16 bytes.
    const unsigned n_chosen = (unsigned)n_rows * K;
    const int32_t* const chosen = topk_idx + (size_t)r0 * K;
    unsigned at = 4 * tid;
    int4 four = make_int4(0, 0, 0, 0);
    const auto fetch_four = [&] {
        if (at + 4 <= n_chosen) {
            four = __ldg(reinterpret_cast<const int4*>(chosen + at));
        } else if (at < n_chosen) {
            four.x = __ldg(chosen + at);
            if (at + 1 < n_chosen) four.y = __ldg(chosen + at + 1);
            if (at + 2 < n_chosen) four.z = __ldg(chosen + at + 2);
        }
    };
    const auto count_one = [&](unsigned a, int e) {
        if (a >= n_chosen || (mask != nullptr && __ldg(mask + r0 + a / (unsigned)K) == 0)) return;
        if ((unsigned)e < (unsigned)E) atomicAdd(&s_count[e], 1);
        else director_set_status(status, DIRECTOR_ERR_BAD_INDEX);
    };
    const auto count_four = [&] {
        if (at >= n_chosen) return;
        count_one(at, four.x), count_one(at + 1, four.y), count_one(at + 2, four.z), count_one(at + 3, four.w);
        at += 4 * kThreads;
        fetch_four();
    };
    fetch_four();

    for (int base = warp * kGroups; base < n_rows; base += kWarps * kGroups) {
        const bool live = next_live;
        float x[kVals];
#pragma unroll
        for (int i = 0; i < kVals; ++i) x[i] = next[i];
        next_live = fetch(base + kWarps * kGroups);
        const float s = softmax_terms<LPR>(x);
        const float inv = __fdividef(1.0f, s);
        if (live) {
            valid += sub == 0;
            if (s > 0.0f) {
#pragma unroll
                for (int i = 0; i < kVals; ++i) acc[i] = fmaf(x[i], inv, acc[i]);
            } else if (sub == 0) {
                director_set_status(status, DIRECTOR_ERR_NONFINITE);
            }
        }
        count_four();
    }
    while (at < n_chosen) count_four();
#pragma unroll
    for (int o = LPR; o < 32; o <<= 1)
#pragma unroll
        for (int i = 0; i < kVals; ++i) acc[i] += __shfl_xor_sync(0xFFFFFFFFu, acc[i], o);
    if (lane < LPR)
#pragma unroll
        for (int i = 0; i < kVals; ++i) s_p[warp][expert_of<LPR, VEC>(i, sub)] = acc[i];
    valid = __reduce_add_sync(0xFFFFFFFFu, valid);
    if (lane == 0 && valid) atomicAdd(&s_count[kMaxE], valid);
    __syncthreads();

    double p = 0.0;                                        // of expert tid, below
    if (tid < E)
#pragma unroll
        for (int w = 0; w < kWarps; ++w) p += (double)s_p[w][tid];
    long long count = tid < E ? s_count[tid] : 0, n = s_count[kMaxE];
    if (gridDim.x > 1) {
        if (tid < E) {
            atomicAdd(&sums->p[tid], (unsigned long long)__double2ll_rn(ldexp(p, shift)));
            if (count) atomicAdd(&sums->count[tid], (unsigned long long)count);
        }
        if (tid == 0 && n) atomicAdd(&sums->count[kMaxE], (unsigned long long)n);
        __syncthreads();
        if (tid == 0) {                                    // one fence behind the barrier covers what the whole CTA has added
            __threadfence();
            s_last = atomicAdd(&sums->ticket, 1u) == gridDim.x - 1;
            __threadfence();
        }
        __syncthreads();
        if (!s_last) return;
        if (tid < E) {
            p = ldexp((double)(long long)__ldcg(&sums->p[tid]), -shift);
            count = (long long)__ldcg(&sums->count[tid]);
            sums->p[tid] = 0ull;
            sums->count[tid] = 0ull;
        }
        n = (long long)__ldcg(&sums->count[kMaxE]);
        __syncthreads();
        if (tid == 0) {
            sums->count[kMaxE] = 0ull;
            sums->ticket = 0u;
        }
    }
    if (tid < E) counts[tid] = count;
    double term = tid < E ? (double)count * p : 0.0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) term += __shfl_xor_sync(0xFFFFFFFFu, term, o);
    if (lane == 0) s_term[warp] = term;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < kWarps; ++w) term += s_term[w];
        counts[E] = n;
        *loss = n > 0 ? (float)(E * term / ((double)K * (double)n * (double)n)) : 0.0f;
    }
}

// The gradient.  A row is read, its softmax taken again (keeping it would cost the forward another array) and its gradient written.
// f enters less its mean, (E counts_e - sum counts) / (E K N) from whole numbers: the difference f_e - sum_j f_j p_tj is
// the same, and a router that is nearly balanced does not lose it to the rounding of two nearly equal numbers.
template <int LPR, bool VEC>
__global__ void __launch_bounds__(kThreads, VEC ? 4 : 3)
balance_backward_kernel(const float* __restrict__ logits, const int64_t* __restrict__ counts, const uint8_t* __restrict__ mask,
                        const float* __restrict__ dloss, const float* added, float* dlogits, int T, int E, int K, int rows,
                        int32_t* status) {
    constexpr int kGroups = 32 / LPR;
    __shared__ float s_f[LPR * kVals];
    __shared__ long long s_total[kWarps];
    chain_prologue();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane % LPR;
    const int r0 = (int)(gridDim.x - 1 - blockIdx.x) * rows, n_rows = min(rows, T - r0);
    float x[kVals] = {};
    const auto fetch = [&](int base) {                     // the lane's part of its row of the pass at `base`
        const int row = r0 + base + lane / LPR;
        const bool live = base + lane / LPR < n_rows && (mask == nullptr || __ldg(mask + row) != 0);
        if (live) load_row<LPR, VEC>(logits + (size_t)row * E, E, sub, x);
        return live;
    };
    bool live = fetch(warp * kGroups);

    // f, while the first rows are on their way
    const long long count = tid < E ? __ldg(counts + tid) : 0;
    const double n = (double)__ldg(counts + E);
    long long total = count;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, o);
    if (lane == 0) s_total[warp] = total;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) total += s_total[w];
    if (tid < LPR * kVals) s_f[tid] = n > 0 ? (float)((double)(E * count - total) / ((double)E * K * n)) : 0.0f;
    __syncthreads();
    float f[kVals];
#pragma unroll
    for (int i = 0; i < kVals; ++i) f[i] = s_f[expert_of<LPR, VEC>(i, sub)];
    const float factor = n > 0 ? (float)((double)__ldg(dloss) * E / n) : 0.0f;

    for (int base = warp * kGroups; base < n_rows; base += kWarps * kGroups) {
        const int row = r0 + base + lane / LPR;
        const float s = softmax_terms<LPR>(x);
        const bool good = live && s > 0.0f;
        if (!good) {                                       // no gradient: padding, or a row that is not finite
            if (live && sub == 0) director_set_status(status, DIRECTOR_ERR_NONFINITE);
#pragma unroll
            for (int i = 0; i < kVals; ++i) x[i] = 0.0f;
        }
        float mean = 0.0f;
#pragma unroll
        for (int i = 0; i < kVals; ++i) mean = fmaf(x[i], f[i], mean);
#pragma unroll
        for (int o = 1; o < LPR; o <<= 1) mean += __shfl_xor_sync(0xFFFFFFFFu, mean, o);
        // chosen, not multiplied by zero: a factor that is not finite (a scaled loss that overflowed) leaves such rows alone
        const float inv = good ? __fdividef(1.0f, s) : 0.0f, scale = good ? factor * inv : 0.0f, shift = mean * inv * scale;
        float d[kVals];
#pragma unroll
        for (int i = 0; i < kVals; ++i) d[i] = x[i] * fmaf(f[i], scale, -shift);
        const bool here = base + lane / LPR < n_rows;
        live = fetch(base + kWarps * kGroups);
        if (!here) continue;
#pragma unroll
        for (int j = 0; j < kVals / 4; ++j) {
            if (VEC) {
                const int e = 4 * (j * LPR + sub);
                if (e >= E) continue;
                const size_t at = (size_t)row * E + e;
                float4 v = make_float4(d[4 * j], d[4 * j + 1], d[4 * j + 2], d[4 * j + 3]);
                if (added != nullptr) {
                    const float4 a = *reinterpret_cast<const float4*>(added + at);
                    v.x += a.x, v.y += a.y, v.z += a.z, v.w += a.w;
                }
                *reinterpret_cast<float4*>(dlogits + at) = v;
            } else {
#pragma unroll
                for (int i = 4 * j; i < 4 * j + 4; ++i) {
                    const int e = expert_of<LPR, VEC>(i, sub);
                    if (e >= E) continue;
                    const size_t at = (size_t)row * E + e;
                    dlogits[at] = added != nullptr ? added[at] + d[i] : d[i];
                }
            }
        }
    }
}

// Rows of a CTA: whole passes of its warps, `most` at most, so many that about `ctas` CTAs cover the batch.
int rows_of_cta(int T, int lpr, int ctas, int most) {
    const int pass = kWarps * (32 / lpr), passes = ((T - 1) / pass) / ctas + 1;
    return pass * (passes < most ? passes : most);
}
unsigned ctas_of(int T, int rows) { return (unsigned)((T - 1) / rows) + 1; }

// calls f<LPR, VEC>: the fewest lanes that hold a row, float4 loads where every row starts on 16 bytes
template <typename F>
int by_width(int E, F&& f) {
    const bool vec = E % 4 == 0;
#define DIRECTOR_WIDTH(L) \
    if (E <= L * kVals) return vec ? f(std::integral_constant<int, L>{}, std::true_type{}) : f(std::integral_constant<int, L>{}, std::false_type{})
    DIRECTOR_WIDTH(1);
    DIRECTOR_WIDTH(2);
    DIRECTOR_WIDTH(4);
    DIRECTOR_WIDTH(8);
    DIRECTOR_WIDTH(16);
#undef DIRECTOR_WIDTH
    return DIRECTOR_ERR_UNSUPPORTED;
}

}  // namespace

size_t balance_workspace_bytes() { return sizeof(BalanceSums); }

int launch_balance_loss(director_ctx* ctx, int T, const float* logits, const int32_t* topk_idx, const uint8_t* mask, float* loss,
                        int64_t* counts, cudaStream_t st) {
    StageScope stage(ctx, st, "stage_balance_loss");
    const director_shape& s = ctx->shape;
    int shift = 62;
    for (int t = T; t > 0; t >>= 1) --shift;               // T 2^shift < 2^62
    return by_width(s.E, [&](auto lpr, auto vec) {
        constexpr int L = decltype(lpr)::value;
        const int rows = rows_of_cta(T, L, kForwardCtas * ctx->sm_count, kMostPasses);
        LaunchScope scope(ctx, st, "balance_loss_kernel");
        return cuda_status(launch_chained(balance_loss_kernel<L, decltype(vec)::value>, dim3(ctas_of(T, rows)), dim3(kThreads), 0, st,
                                          logits, topk_idx, mask, T, (int)s.E, (int)s.K, rows, shift,
                                          static_cast<BalanceSums*>(ctx->d_balance), loss, counts, ctx->d_status));
    });
}

int launch_balance_backward(director_ctx* ctx, int T, const float* logits, const int64_t* counts, const uint8_t* mask,
                            const float* dloss, const float* added, float* dlogits, cudaStream_t st) {
    StageScope stage(ctx, st, "stage_balance_backward");
    const director_shape& s = ctx->shape;
    return by_width(s.E, [&](auto lpr, auto vec) {
        constexpr int L = decltype(lpr)::value;
        const int rows = rows_of_cta(T, L, kBackwardCtas * ctx->sm_count, kMostPasses);
        LaunchScope scope(ctx, st, "balance_backward_kernel");
        return cuda_status(launch_chained(balance_backward_kernel<L, decltype(vec)::value>, dim3(ctas_of(T, rows)), dim3(kThreads), 0, st,
                                          logits, counts, mask, dloss, added, dlogits, T, (int)s.E, (int)s.K, rows, ctx->d_status));
    });
}

}  // namespace director
