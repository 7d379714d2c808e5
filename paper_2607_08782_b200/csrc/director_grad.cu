// The row-moving and gating half of the layer's backward pass (the forward's Section II-A weighted sum and gate, Section II-B
// exchanges, differentiated; the paper itself serves and does not train).  The expert products' gradients are in
// director_ffn_grad.cu.  All four kernels move data once and compute almost nothing: HBM bounds them.
#include "director_common.cuh"

#include <cuda_bf16.h>

namespace director {

namespace {

__device__ __forceinline__ float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
}

// ---- gradient of the combine -------------------------------------------------------------------------------------
//
//   y[t] = sum_s w[t,s] yp[r(t,s)]:   dyp[r(t,s)] = w[t,s] dy[t],   dw[t,s] = <dy[t], yp[r(t,s)]>
//
// One warp per assignment (t, s): it reads dy[t] and the row of yp once, writes the row of dyp, and the dot product is a sum
// over its lanes - no atomics, so dw has the same bits on every run.  The K warps of a token sit next to each other in a CTA,
// so that dy[t] comes from HBM once and from L1 or L2 after that.  T = 32768, H = 2048, K = 8: 352-358 us, 6.4-6.5 TB/s.  Tried there: CTAs
// of 8 warps + 1 %, 16 + 4 %; rows of yp loaded as streaming (evict first) + 4 %, dyp stored so + 11 %; four pieces of a row per
// lane asked for together + 4 % (registers cost occupancy), and no faster for a small batch, whose call is launch-bound.
constexpr int kRowWarps = 4;

__global__ void __launch_bounds__(kRowWarps * 32)
combine_backward_kernel(const uint4* __restrict__ dy, const uint4* __restrict__ yp, const int32_t* __restrict__ inv_row,
                        const float* __restrict__ topk_w, uint4* __restrict__ dyp, float* __restrict__ dtopk_w, int A, int K,
                        int row_vec, int32_t* status) {
    chain_prologue();
    const int lane = threadIdx.x & 31;
    const long long item = (long long)blockIdx.x * kRowWarps + (threadIdx.x >> 5);
    if (item >= A) return;
    const int t = (int)(item / K);
    const int row = __ldg(inv_row + item);
    const float w = __ldg(topk_w + item);
    if ((unsigned)row >= (unsigned)A) {       // an assignment that the dispatch skipped (-1), or no row of this batch
        if (lane == 0) {
            dtopk_w[item] = 0.0f;
            if (row >= 0) director_set_status(status, DIRECTOR_ERR_BAD_INDEX);
        }
        return;
    }
    const uint4* g = dy + (size_t)t * row_vec;
    const uint4* y = yp + (size_t)row * row_vec;
    uint4* o = dyp + (size_t)row * row_vec;
    float dot = 0.0f;
    for (int v = lane; v < row_vec; v += 32) {
        const uint4 a = __ldg(g + v), b = __ldg(y + v);
        const uint32_t ga[4] = {a.x, a.y, a.z, a.w}, yb[4] = {b.x, b.y, b.z, b.w};
        uint32_t r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            dot = fmaf(bf16_lo(ga[i]), bf16_lo(yb[i]), dot);
            dot = fmaf(bf16_hi(ga[i]), bf16_hi(yb[i]), dot);
            r[i] = pack_bf16x2(w * bf16_lo(ga[i]), w * bf16_hi(ga[i]));
        }
        o[v] = make_uint4(r[0], r[1], r[2], r[3]);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, d);
    if (lane == 0) dtopk_w[item] = dot;
}

// ---- gradient of the gate ----------------------------------------------------------------------------------------
//
//   w = softmax over the K chosen logits:   dlogits[t, idx[t,s]] = w[t,s] (dw[t,s] - sum_j w[t,j] dw[t,j]),  0 elsewhere
//
// One warp per four tokens, eight lanes a token (K <= 8): a lane holds one choice, the weighted mean is a sum over the eight, the
// warp clears its four rows of dlogits (4 E floats, a 16-byte aligned block for every E) and each lane then stores its one
// value.  T = 32768, E = 128, K = 8: 6.0 us a call, launch-bound; comparing every entry with the K choices instead took 8.1 us, a
// tile in shared memory 6.4 us.
constexpr int kGateWarps = 4;

__global__ void __launch_bounds__(kGateWarps * 32)
route_backward_kernel(const int32_t* __restrict__ topk_idx, const float* __restrict__ topk_w, const float* __restrict__ dtopk_w,
                      float* __restrict__ dlogits, int T, int K, int E, int32_t* status) {
    chain_prologue();
    const int lane = threadIdx.x & 31, s = lane & 7;
    const int t0 = (blockIdx.x * kGateWarps + (threadIdx.x >> 5)) * 4, t = t0 + (lane >> 3);
    if (t0 >= T) return;
    int idx = -1;
    float w = 0.0f, dw = 0.0f;
    if (s < K && t < T) {
        const size_t i = (size_t)t * K + s;
        idx = __ldg(topk_idx + i);
        w = __ldg(topk_w + i);
        dw = __ldg(dtopk_w + i);
        if ((unsigned)idx >= (unsigned)E) director_set_status(status, DIRECTOR_ERR_BAD_INDEX);
    }
    float* const rows = dlogits + (size_t)t0 * E;
    const int total = min(4, T - t0) * E;
    for (int i = lane; i < total / 4; i += 32) reinterpret_cast<float4*>(rows)[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int i = total / 4 * 4 + lane; i < total; i += 32) rows[i] = 0.0f;
    float mean = w * dw;
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) mean += __shfl_xor_sync(0xFFFFFFFFu, mean, o);   // lanes without a choice hold zeros
    __syncwarp();                                                                    // the zeros come before the values
    if ((unsigned)idx < (unsigned)E) dlogits[(size_t)t * E + idx] = w * (dw - mean);
}

// ---- the 8-bit checkpoint as numbers -----------------------------------------------------------------------------
//
// A CTA takes 32 rows x 16 blocks of 16 features: the exponents, which lie along the rows, go through shared memory; a lane
// turns half a block - 16 bytes of codes - into 8 gate and 8 up values, so that a warp reads 512 and writes 2 x 512
// consecutive bytes.  Codes of seven bits and a sign times a power of two are exact in bf16.  HBM-bound: 69 M values of each in
// 69 us, 6.1 TB/s (a thread per block of 16, its exponent read across the rows, took a fifth longer).
constexpr int kDecodeRows = 32, kDecodeBlocks = 16;

__global__ void __launch_bounds__(256)
checkpoint_decode_kernel(const uint4* __restrict__ codes, const uint16_t* __restrict__ exps, uint4* __restrict__ gate,
                         uint4* __restrict__ up, int rows, int blocks, int row_tiles) {
    __shared__ uint16_t s_exp[kDecodeBlocks][kDecodeRows];
    chain_prologue();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int row0 = (int)(blockIdx.x % row_tiles) * kDecodeRows, b0 = (int)(blockIdx.x / row_tiles) * kDecodeBlocks;
    for (int b = warp; b < kDecodeBlocks; b += 8)
        s_exp[b][lane] = b0 + b < blocks && row0 + lane < rows ? __ldg(exps + (size_t)(b0 + b) * rows + row0 + lane) : 0;
    const int half = 2 * b0 + lane;                           // which 8 features of the row
    uint4 c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = row0 + warp * 4 + i;
        c[i] = half < 2 * blocks && row < rows ? __ldcs(codes + (size_t)row * (2 * blocks) + half) : make_uint4(0u, 0u, 0u, 0u);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = row0 + warp * 4 + i;
        if (half >= 2 * blocks || row >= rows) continue;
        const uint32_t e = s_exp[lane >> 1][warp * 4 + i];
        const float sg = checkpoint_scale(e & 255u), su = checkpoint_scale(e >> 8);
        const uint32_t w[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
        uint32_t g[4], u[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t biased = w[j] ^ 0x80808080u;
            g[j] = pack_bf16x2(checkpoint_value(biased, 0, sg), checkpoint_value(biased, 2, sg));
            u[j] = pack_bf16x2(checkpoint_value(biased, 1, su), checkpoint_value(biased, 3, su));
        }
        const size_t at = (size_t)row * (2 * blocks) + half;
        gate[at] = make_uint4(g[0], g[1], g[2], g[3]);
        up[at] = make_uint4(u[0], u[1], u[2], u[3]);
    }
}

}  // namespace

int launch_combine_backward(director_ctx* ctx, int T, const void* dy, const void* yp, const int32_t* inv_row,
                            const float* topk_w, void* dyp, float* dtopk_w, cudaStream_t st) {
    StageScope stage(ctx, st, "stage_combine_backward");
    const director_shape& s = ctx->shape;
    const int A = T * s.K;
    const unsigned grid = ((unsigned)A + kRowWarps - 1) / kRowWarps;
    LaunchScope scope(ctx, st, "combine_backward_kernel");
    return cuda_status(launch_chained(combine_backward_kernel, dim3(grid), dim3(kRowWarps * 32), 0, st,
                                      static_cast<const uint4*>(dy), static_cast<const uint4*>(yp), inv_row, topk_w,
                                      static_cast<uint4*>(dyp), dtopk_w, A, s.K, s.H * 2 / 16, ctx->d_status));
}

int launch_route_backward(director_ctx* ctx, int T, const int32_t* topk_idx, const float* topk_w, const float* dtopk_w,
                          float* dlogits, cudaStream_t st) {
    StageScope stage(ctx, st, "stage_route_backward");
    const director_shape& s = ctx->shape;
    const unsigned grid = ((unsigned)T + 4 * kGateWarps - 1) / (4 * kGateWarps);
    LaunchScope scope(ctx, st, "route_backward_kernel");
    return cuda_status(launch_chained(route_backward_kernel, dim3(grid), dim3(kGateWarps * 32), 0, st, topk_idx, topk_w, dtopk_w,
                                      dlogits, T, (int)s.K, (int)s.E, ctx->d_status));
}

int launch_checkpoint_decode(director_ctx* ctx, int rows, int F, const Checkpoint& kept, void* gate, void* up,
                             cudaStream_t st) {
    const int blocks = F / kCheckpointBlock;
    const int row_tiles = (rows + kDecodeRows - 1) / kDecodeRows;
    const unsigned grid = (unsigned)row_tiles * (unsigned)((blocks + kDecodeBlocks - 1) / kDecodeBlocks);
    LaunchScope scope(ctx, st, "checkpoint_decode_kernel");
    return cuda_status(launch_chained(checkpoint_decode_kernel, dim3(grid), dim3(256), 0, st,
                                      reinterpret_cast<const uint4*>(kept.codes), static_cast<const uint16_t*>(kept.exps),
                                      static_cast<uint4*>(gate), static_cast<uint4*>(up), rows, blocks, row_tiles));
}

}  // namespace director
