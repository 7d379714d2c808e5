// The router's balance term (training; the paper balances by placement instead, Section VI): per-expert counts, the loss that pulls
// the router's mean scores towards an even load, and its gradient.
//
//   N valid tokens, f_e = counts_e / (K N), p_t = softmax(logits_t), P_e = sum_t p_te / N:   loss = E sum_e f_e P_e
//   dlogits_te = dloss E/N p_te (f_e - sum_j f_j p_tj)          (the counts are piecewise constant)
//
// A row of up to 256 logits lies in the registers of LPR lanes, sixteen values each, so that a pass over the logits is one read;
// max and sum of the softmax take log2(LPR) shuffles for the 32 / LPR rows that a warp has at a time, and a lane keeps its columns from
// row to row, so that the sums over tokens are adds in registers.  HBM bounds the large batches, the launch the small ones.
#include "director_common.cuh"

#include <cmath>

namespace director {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kVals = 16;
constexpr int kForwardRows = 64;     // most rows of a lane's registers in one CTA of the forward: its fp32 sums stay short

// The sixteen values of lane `sub` of its row: groups of four, LPR groups apart.  -inf behind the last expert.
template <int LPR, bool VEC>
__device__ __forceinline__ void load_row(const float* __restrict__ row, int E, int sub, float (&x)[kVals]) {
#pragma unroll
    for (int j = 0; j < kVals / 4; ++j) {
        const int e = 4 * (j * LPR + sub);
        if (VEC) {
            const float4 v = e < E ? __ldg(reinterpret_cast<const float4*>(row + e)) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
            x[4 * j] = v.x, x[4 * j + 1] = v.y, x[4 * j + 2] = v.z, x[4 * j + 3] = v.w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[4 * j + i] = e + i < E ? __ldg(row + e + i) : -INFINITY;
        }
    }
}

// x -> exp(x - max); returns their sum, NaN for a row with a NaN, a +inf or nothing but -inf.  __expf's error grows with the
// distance from the maximum, 2^-24 a unit: what it moves is as small as exp(-distance).
template <int LPR>
__device__ __forceinline__ float softmax_terms(float (&x)[kVals]) {
    float m = x[0];
#pragma unroll
    for (int i = 1; i < kVals; ++i) m = fmaxf(m, x[i]);
#pragma unroll
    for (int o = 1; o < LPR; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < kVals; ++i) {
        x[i] = __expf(x[i] - m);
        s += x[i];
    }
#pragma unroll
    for (int o = 1; o < LPR; o <<= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    return s;
}

// Loss and counts.  A CTA sums its tokens' p in registers (fp32, at most kForwardRows rows a lane), then over lanes and warps (the
// latter in fp64), and adds the sums to the context's 64-bit integers as fixed point (2^`shift` to one; T 2^shift < 2^62), whose
// order makes no difference: the loss has the same bits on every run.  The last CTA to arrive writes the results and leaves zeros.
struct BalanceSums {
    unsigned long long p[kMaxE];
    unsigned long long count[kMaxE + 1];     // [kMaxE]: valid tokens
    unsigned int ticket;
};

template <int LPR, bool VEC>
__global__ void __launch_bounds__(kThreads)
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

    for (unsigned a = tid; a < (unsigned)(n_rows * K); a += kThreads) {
        if (mask != nullptr && __ldg(mask + r0 + a / (unsigned)K) == 0) continue;
        const int e = __ldg(topk_idx + (size_t)r0 * K + a);
        if ((unsigned)e < (unsigned)E) atomicAdd(&s_count[e], 1);
        else director_set_status(status, DIRECTOR_ERR_BAD_INDEX);
    }

    float acc[kVals] = {};
    int valid = 0;
    for (int base = warp * kGroups; base < n_rows; base += kWarps * kGroups) {
        const bool here = base + lane / LPR < n_rows;
        const int row = r0 + base + lane / LPR;
        const bool live = here && (mask == nullptr || __ldg(mask + row) != 0);
        float x[kVals] = {};
        if (live) load_row<LPR, VEC>(logits + (size_t)row * E, E, sub, x);
        const float s = softmax_terms<LPR>(x);
        const bool good = live && s > 0.0f;
        if (live && !good && sub == 0) director_set_status(status, DIRECTOR_ERR_NONFINITE);
        valid += live && sub == 0;
        const float inv = 1.0f / s;
#pragma unroll
        for (int i = 0; i < kVals; ++i) acc[i] += good ? x[i] * inv : 0.0f;
    }
#pragma unroll
    for (int o = LPR; o < 32; o <<= 1)
#pragma unroll
        for (int i = 0; i < kVals; ++i) acc[i] += __shfl_xor_sync(0xFFFFFFFFu, acc[i], o);
    if (lane < LPR)
#pragma unroll
        for (int i = 0; i < kVals; ++i) s_p[warp][4 * ((i / 4) * LPR + sub) + i % 4] = acc[i];
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
        __threadfence();
        __syncthreads();
        if (tid == 0) s_last = atomicAdd(&sums->ticket, 1u) == gridDim.x - 1;
        __syncthreads();
        if (!s_last) return;
        __threadfence();
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

// The gradient.  f enters less its mean, (E counts_e - sum counts) / (E K N) from whole numbers: the difference f_e - sum_j f_j p_tj is
// the same, and a router that is nearly balanced does not lose it to the rounding of two nearly equal numbers.
template <int LPR, bool VEC>
__global__ void __launch_bounds__(kThreads)
balance_backward_kernel(const float* __restrict__ logits, const int64_t* __restrict__ counts, const uint8_t* __restrict__ mask,
                        const float* __restrict__ dloss, const float* added, float* dlogits, int T, int E, int K, int rows,
                        int32_t* status) {
    constexpr int kGroups = 32 / LPR;
    chain_prologue();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % LPR;
    float f[kVals];
    float factor;
    {
        long long c[kVals], total = 0;
#pragma unroll
        for (int i = 0; i < kVals; ++i) {
            const int e = 4 * ((i / 4) * LPR + sub) + i % 4;
            c[i] = e < E ? __ldg(counts + e) : 0;
            total += c[i];
        }
#pragma unroll
        for (int o = 1; o < LPR; o <<= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, o);
        const double n = (double)__ldg(counts + E), scale = n > 0 ? 1.0 / ((double)E * K * n) : 0.0;
#pragma unroll
        for (int i = 0; i < kVals; ++i) f[i] = (float)((double)(E * c[i] - total) * scale);
        factor = n > 0 ? (float)((double)__ldg(dloss) * E / n) : 0.0f;
    }
    const int r0 = blockIdx.x * rows, n_rows = min(rows, T - r0);
    for (int base = warp * kGroups; base < n_rows; base += kWarps * kGroups) {
        const bool here = base + lane / LPR < n_rows;
        const int row = r0 + base + lane / LPR;
        const bool live = here && (mask == nullptr || __ldg(mask + row) != 0);
        float x[kVals] = {};
        if (live) load_row<LPR, VEC>(logits + (size_t)row * E, E, sub, x);
        const float s = softmax_terms<LPR>(x);
        const bool good = live && s > 0.0f;
        if (live && !good && sub == 0) director_set_status(status, DIRECTOR_ERR_NONFINITE);
        float mean = 0.0f;
#pragma unroll
        for (int i = 0; i < kVals; ++i) mean = fmaf(x[i], f[i], mean);
#pragma unroll
        for (int o = 1; o < LPR; o <<= 1) mean += __shfl_xor_sync(0xFFFFFFFFu, mean, o);
        const float inv = 1.0f / s, scale = factor * inv;
        mean *= inv;
        if (!here) continue;
#pragma unroll
        for (int j = 0; j < kVals / 4; ++j) {
            const int e = 4 * (j * LPR + sub);
            float d[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) d[i] = good ? scale * x[4 * j + i] * (f[4 * j + i] - mean) : 0.0f;
            const size_t at = (size_t)row * E + e;
            if (VEC) {
                if (e >= E) continue;
                if (added != nullptr) {
                    const float4 a = *reinterpret_cast<const float4*>(added + at);
                    d[0] += a.x, d[1] += a.y, d[2] += a.z, d[3] += a.w;
                }
                *reinterpret_cast<float4*>(dlogits + at) = make_float4(d[0], d[1], d[2], d[3]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (e + i < E) dlogits[at + i] = added != nullptr ? added[at + i] + d[i] : d[i];
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
        const int rows = rows_of_cta(T, L, 2 * ctx->sm_count, kForwardRows);
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
        const int rows = rows_of_cta(T, L, 4 * ctx->sm_count, 32);
        LaunchScope scope(ctx, st, "balance_backward_kernel");
        return cuda_status(launch_chained(balance_backward_kernel<L, decltype(vec)::value>, dim3(ctas_of(T, rows)), dim3(kThreads), 0, st,
                                          logits, counts, mask, dloss, added, dlogits, T, (int)s.E, (int)s.K, rows, ctx->d_status));
    });
}

}  // namespace director
