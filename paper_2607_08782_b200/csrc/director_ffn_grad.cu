// Gradients of the grouped expert FFN (Section II-A's expert FFNs, differentiated; the paper itself does not train).
//
// For the rows i of an expert's segments, with g, u the kept gate and up values (8 bits, director_checkpoint.cuh), s = sigmoid(g):
//   GRAD_ACT    da = dyp . Wd              contraction over H;   epilogue: act = g s u, du = da g s, dg = da u s (1 + g (1 - s))
//   GRAD_DX     dxp = dg . Wg + du . Wu    contraction over 2F: F steps of (Wg, dg), then F of (Wu, du), one accumulator
//   GRAD_GATEUP dWg = dg^T . xp, dWu = du^T . xp    contraction over the expert's rows
//   GRAD_DOWN   dWd = dyp^T . act                   contraction over the expert's rows
// dg, du and act are rounded to bf16 between the products (the tensor cores' operand type): an error of the size of the
// outputs' own rounding.  All sums are fp32 in tensor memory, in a fixed order.
//
// CTA pairs as in the forward kernel (tcgen05.mma cta_group::2, M = 256: 128 rows of D per CTA, accumulators of up to 256
// columns, two of them), operands by TMA through a ring of 32 KB stages.  What differs is the operands' direction: no matrix
// is transposed in memory.  An operand whose rows run along the contraction (Wd, Wg, Wu as the left operand; everything in
// the weight gradients) is loaded as boxes of 64 contraction rows x 64 columns and handed to the tensor core as an
// MN-major tile.
//   GRAD_ACT / GRAD_DX: D[feature, token], as in the forward: 256 weight columns x up to 256 tokens, the token count a runtime
//     operand in steps of 32, so a segment's ragged end costs little.
//   GRAD_GATEUP: D[h, f]: 256 columns of xp x 128 features of dg and the same 128 of du - the left tile serves both products,
//     and each CTA of the pair supplies one of the right ones.   GRAD_DOWN: D[h, f]: 256 columns of dyp x up to 256 of act.
//     The contraction runs over the segments of all of an expert's replicas.  Where a segment ends inside a 64-row step the
//     rows behind it belong to another expert: the step issues only the MMAs it needs (16 rows each), and a warp of each CTA
//     zeroes the rows behind the end inside the last one, in both operands (a zero times another expert's infinity would be
//     NaN).  Experts are taken by descending length, so that the longest contractions do not end the launch.
//     An expert without rows gets zeros.
// Work items are claimed from a global counter and handed to all roles through a small ring, as in the forward kernel.
// Every wait is bounded; an expired one raises DIRECTOR_ERR_TIMEOUT.
#include "director_common.cuh"
#include "director_umma.cuh"

#include <cuda_bf16.h>

namespace director {

using namespace umma;

namespace {

enum GradKind { GRAD_ACT = 0, GRAD_DX = 1, GRAD_GATEUP = 2, GRAD_DOWN = 3 };

constexpr int G_STAGES = 6;
constexpr int G_BOX_BYTES = 64 * 128;                  // 64 rows of 64 bf16 columns
constexpr int G_STAGE_BYTES = 4 * G_BOX_BYTES;         // 16 KB of each operand
constexpr int G_EPI_WARPS = 8;                         // two per TMEM lane quadrant
constexpr int G_THREADS = 128 + 32 * G_EPI_WARPS;      // producer, MMA, scheduler and tail warps + epilogue
constexpr int G_TILE = 256;                            // tokens per full tile; accumulators are this many columns apart
constexpr int G_SLOTS = 4;                             // ring of work items
constexpr int G_CLAIM_LEAD = 32;                       // k-steps of claimed work ahead of the producer

struct GradHeader {
    uint64_t full[G_STAGES], empty[G_STAGES];
    uint64_t part[G_STAGES];                           // this CTA's loads of a step that still has rows to be zeroed
    uint64_t tfull[2], tempty[2], sched_full[G_SLOTS], sched_empty[G_SLOTS];
    int4 item[G_SLOTS];
    uint32_t tmem;
    int abort;
    int prod_k;                                        // k-steps issued by the scheduler CTA's producer
    int warp_sum[8];
};
constexpr int grad_smem_bytes(int n_rep, int E) {
    return 1024 + G_STAGES * G_STAGE_BYTES + (int)sizeof(GradHeader) + 8 * n_rep + 4 * (2 * (E + 1) + 2 * E);
}
static_assert(grad_smem_bytes(kMaxG, kMaxE) <= 232448, "the ring does not fit with the largest tables");
static_assert(kMaxE <= G_THREADS, "one thread per expert builds the tables");

constexpr uint32_t G_IDESC_BASE = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) /* left operand MN-major */ |
                                  ((uint32_t)(256 >> 4) << 24);
constexpr uint32_t G_IDESC_B_MN = 1u << 16;

// Shared-memory matrix descriptor of an MN-major tile, 128-byte swizzle: boxes of 64 columns x 64 contraction rows, a row 128
// bytes; the next 64 columns 8192 bytes on (LBO), the next 8 rows 1024 bytes on (SBO).  16 contraction rows - one MMA - are
// 2048 bytes.
__device__ __forceinline__ uint64_t smem_desc_mn(uint32_t addr) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(G_BOX_BYTES >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}

struct GradParams {
    const int32_t* seg_offsets;    // [G+1], clamped to [0, rows]
    const int32_t* rep_start;      // [E+1] replicas of expert e: rep_slot[rep_start[e] .. rep_start[e+1])
    const int32_t* rep_slot;
    int E, n_rep;
    int rows;                      // rows of the permuted operands
    int dense;                     // 1: one expert whose only segment is [0, rows); the three tables are not read
    int H, F;
    int m_blocks;                  // blocks of 256 D rows (per expert)
    int n_blocks;                  // weight gradients: blocks of D columns per expert
    int k_steps;                   // GRAD_ACT, GRAD_DX
    const int8_t* codes;           // GRAD_ACT: the checkpoint
    const uint16_t* exps;
    uint16_t* out0;                // dg | dxp | dWg | dWd
    uint16_t* out1;                // du |  -  | dWu |  -
    uint16_t* out2;                // act
    int32_t* status;
    unsigned int* counter;
};

struct GradItem {
    int a, valid, e, b;            // tokens: first row, rows (0: end), expert, block;   weights: h block, 1, expert, f block
};

__device__ __forceinline__ uint16_t to_bf16(float v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v)); }

template <int KIND>
__global__ void __launch_bounds__(G_THREADS, 1)
grouped_grad_kernel(const __grid_constant__ CUtensorMap tm_a0, const __grid_constant__ CUtensorMap tm_a1,
                    const __grid_constant__ CUtensorMap tm_b0, const __grid_constant__ CUtensorMap tm_b1, const GradParams p) {
    constexpr bool WEIGHTS = KIND == GRAD_GATEUP || KIND == GRAD_DOWN;
    extern __shared__ uint8_t smem_raw[];
    chain_prologue();
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t ring = (raw + 1023u) & ~1023u;
    GradHeader& hd = *reinterpret_cast<GradHeader*>(smem_raw + (ring - raw) + G_STAGES * G_STAGE_BYTES);
    const int E = p.E;
    int32_t* const s_rep = reinterpret_cast<int32_t*>(&hd + 1);        // [E+1] first replica of every expert
    int32_t* const s_pre = s_rep + (E + 1);                            // [E+1] token tiles before expert e
    int32_t* const s_steps = s_pre + (E + 1);                          // [E] weight gradients: 64-row steps of expert e
    int32_t* const s_order = s_steps + E;                              // [E] weight gradients: experts, longest first
    int32_t* const s_lo = s_order + E;                                 // [n_rep] rows of every replica
    int32_t* const s_hi = s_lo + p.n_rep;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = cluster_ctarank();
    const bool leader = rank == 0;
    volatile int* const abort_flag = &hd.abort;
    volatile int* const prod_k = &hd.prod_k;
    const uint32_t abort_addr = smem_u32(&hd.abort);

    // ---- tables and barriers ----
    for (int r = tid; r < p.n_rep; r += G_THREADS) {
        int lo = 0, hi = p.rows;
        if (!p.dense) {
            const int g = __ldg(p.rep_slot + r);
            lo = min(max(__ldg(p.seg_offsets + g), 0), p.rows);
            hi = min(max(__ldg(p.seg_offsets + g + 1), lo), p.rows);
        }
        s_lo[r] = lo;
        s_hi[r] = hi;
    }
    for (int e = tid; e <= E; e += G_THREADS) s_rep[e] = p.dense ? e : __ldg(p.rep_start + e);
    if (tid == 0) {
        *abort_flag = 0;
        *prod_k = 0;
        for (int s = 0; s < G_STAGES; ++s) {
            mbar_init(smem_u32(&hd.full[s]), 2);
            mbar_init(smem_u32(&hd.empty[s]), 1);
            mbar_init(smem_u32(&hd.part[s]), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(smem_u32(&hd.tfull[a]), 1);
            mbar_init(smem_u32(&hd.tempty[a]), 2 * G_EPI_WARPS);
        }
        // readers of an item: the MMA warp, both producers, all epilogue warps, for the weight gradients both tail warps
        for (int q = 0; q < G_SLOTS; ++q) {
            mbar_init(smem_u32(&hd.sched_full[q]), 1);
            mbar_init(smem_u32(&hd.sched_empty[q]), 3 + 2 * G_EPI_WARPS + (WEIGHTS ? 2 : 0));
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    {
        int mine = 0;                                   // token tiles (or 64-row steps) of expert tid
        if (tid < E)
            for (int r = s_rep[tid]; r < s_rep[tid + 1]; ++r)
                mine += WEIGHTS ? (s_hi[r] - s_lo[r] + 63) / 64 : (s_hi[r] - s_lo[r] + G_TILE - 1) / G_TILE;
        if constexpr (WEIGHTS) {
            if (tid < E) s_steps[tid] = mine;
            __syncthreads();
            if (tid < E) {
                int before = 0;
                for (int e = 0; e < E; ++e) before += s_steps[e] > mine || (s_steps[e] == mine && e < tid) ? 1 : 0;
                s_order[before] = tid;
            }
        } else {
            int incl = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
                if (lane >= o) incl += v;
            }
            if (warp < 8 && lane == 31) hd.warp_sum[warp] = incl;
            __syncthreads();
            for (int w = 0; w < min(warp, 8); ++w) incl += hd.warp_sum[w];
            if (tid < E) s_pre[tid + 1] = incl;
            if (tid == 0) s_pre[0] = 0;
        }
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&hd.tmem)), "r"(TMEM_COLS)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem_base = hd.tmem;

    // ---- work items: claimed by one thread of the leader CTA, read by every role of both ----
    auto take_item = [&](int i, GradItem& it) -> bool {
        const int q = i & (G_SLOTS - 1);
        const uint32_t par = ((uint32_t)i / G_SLOTS) & 1u, bar = smem_u32(&hd.sched_full[q]);
        const bool ok = leader ? mbar_wait(bar, par, abort_flag) : mbar_wait_acquire_cluster(bar, par, abort_flag);
        if (ok) {
            const int4 v = hd.item[q];
            it = GradItem{v.x, v.y, v.z, v.w};
        }
        return ok;
    };
    auto release_item = [&](int i) {
        const uint32_t bar = smem_u32(&hd.sched_empty[i & (G_SLOTS - 1)]);
        if (leader) mbar_arrive(bar);
        else mbar_arrive_cluster(map_to_cta(bar, 0));
    };
    auto take_item_warp = [&](int i, GradItem& it) -> bool {      // for a warp that runs its loop in lock step
        const bool ok = __all_sync(0xFFFFFFFFu, take_item(i, it));
        it.a = __shfl_sync(0xFFFFFFFFu, it.a, 0);
        it.valid = __shfl_sync(0xFFFFFFFFu, it.valid, 0);
        it.e = __shfl_sync(0xFFFFFFFFu, it.e, 0);
        it.b = __shfl_sync(0xFFFFFFFFu, it.b, 0);
        if (ok && lane == 0) release_item(i);
        return ok && it.valid != 0;
    };
    auto columns_of = [&](const GradItem& it) -> int {            // N of the item's MMAs
        if (KIND == GRAD_GATEUP) return 256;
        if (KIND == GRAD_DOWN) return min(256, p.F - it.b * 256);
        return (it.valid + 31) / 32 * 32;
    };

    GradItem it{};
    if (warp == 0) {
        // ---- operand producer, both CTAs ----
        const uint32_t lead_lane = elect_one() ? 1u : 0u;
        int stage = 0, issued_k = 0;
        uint32_t phase = 0, bad = 0;
        for (int i = 0; take_item_warp(i, it); ++i) {
            if constexpr (WEIGHTS) {
                const int m_col = it.a * 256 + (int)rank * 128;
                const int half = columns_of(it) >> 1;             // columns of the right operand this CTA supplies: 128 or 64
                const int n_col = KIND == GRAD_GATEUP ? it.b * 128 : it.b * 256 + (int)rank * half;
                const CUtensorMap* mb = KIND == GRAD_GATEUP && rank ? &tm_b1 : &tm_b0;
                const uint32_t tx = 2 * G_BOX_BYTES + half * 128;
                for (int r = s_rep[it.e]; r < s_rep[it.e + 1]; ++r) {
                    const int hi = s_hi[r];
                    for (int k0 = s_lo[r]; k0 < hi; k0 += 64) {
                        // a step whose last MMA reaches past the segment is reported to this CTA's tail warp first
                        const bool tail = hi - k0 < 64 && ((hi - k0) & 15) != 0;
                        const uint32_t dst = ring + stage * G_STAGE_BYTES;
                        const uint32_t bar = tail ? map_to_cta(smem_u32(&hd.part[stage]), rank) : map_to_cta(smem_u32(&hd.full[stage]), 0);
                        bad = mbar_wait_conv(smem_u32(&hd.empty[stage]), phase ^ 1u, abort_addr, bad, lead_lane);
                        ++issued_k;
                        if (lead_lane && !bad) {
                            mbar_expect_tx_cluster(bar, tx);
                            tma_load_2d_pair(dst, &tm_a0, bar, m_col, k0);
                            tma_load_2d_pair(dst + G_BOX_BYTES, &tm_a0, bar, m_col + 64, k0);
                            tma_load_2d_pair(dst + 2 * G_BOX_BYTES, mb, bar, n_col, k0);
                            if (half > 64) tma_load_2d_pair(dst + 3 * G_BOX_BYTES, mb, bar, n_col + 64, k0);
                            if (leader) *prod_k = issued_k;
                        }
                        if (++stage == G_STAGES) { stage = 0; phase ^= 1u; }
                    }
                }
            } else {
                const int m_col = it.b * 256 + (int)rank * 128;
                const int x_row = it.a + (int)rank * (columns_of(it) >> 1);
                for (int kb = 0; kb < p.k_steps; ++kb) {
                    const bool second = KIND == GRAD_DX && kb >= p.k_steps / 2;
                    const int k = (second ? kb - p.k_steps / 2 : kb) * 64;
                    const int w_row = it.e * (KIND == GRAD_ACT ? p.H : p.F) + k;
                    const CUtensorMap* ma = second ? &tm_a1 : &tm_a0;
                    const CUtensorMap* mb = second ? &tm_b1 : &tm_b0;
                    const uint32_t dst = ring + stage * G_STAGE_BYTES;
                    const uint32_t bar = map_to_cta(smem_u32(&hd.full[stage]), 0);
                    bad = mbar_wait_conv(smem_u32(&hd.empty[stage]), phase ^ 1u, abort_addr, bad, lead_lane);
                    ++issued_k;
                    if (lead_lane && !bad) {
                        mbar_expect_tx_cluster(bar, G_STAGE_BYTES);
                        tma_load_2d_pair(dst, ma, bar, m_col, w_row);
                        tma_load_2d_pair(dst + G_BOX_BYTES, ma, bar, m_col + 64, w_row);
                        tma_load_2d_pair(dst + 2 * G_BOX_BYTES, mb, bar, k, x_row);
                        if (leader) *prod_k = issued_k;
                    }
                    if (++stage == G_STAGES) { stage = 0; phase ^= 1u; }
                }
            }
            if (__any_sync(0xFFFFFFFFu, bad != 0u)) break;
        }
    } else if (warp == 1) {
        // ---- MMA issuer, leader CTA ----
        if (leader) {
            const uint32_t lead_lane = elect_one() ? 1u : 0u;
            int stage = 0;
            uint32_t phase = 0, bad = 0;
            for (int i = 0; take_item_warp(i, it); ++i) {
                const int acc = i & 1;
                bad = mbar_wait_conv(smem_u32(&hd.tempty[acc]), (((uint32_t)i >> 1) & 1u) ^ 1u, abort_addr, bad, lead_lane);
                tc_fence_after();
                const uint32_t d_tmem = tmem_base + (uint32_t)(acc * G_TILE);
                const uint32_t idesc = G_IDESC_BASE | (WEIGHTS ? G_IDESC_B_MN : 0u) | ((uint32_t)(columns_of(it) >> 3) << 17);
                if constexpr (WEIGHTS) {
                    uint32_t accumulate = 0;
                    for (int r = s_rep[it.e]; r < s_rep[it.e + 1]; ++r) {
                        const int hi = s_hi[r];
                        for (int k0 = s_lo[r]; k0 < hi; k0 += 64) {
                            const int slices = (min(64, hi - k0) + 15) >> 4;
                            const uint32_t src = ring + stage * G_STAGE_BYTES;
                            const uint64_t a_desc = smem_desc_mn(src), b_desc = smem_desc_mn(src + 2 * G_BOX_BYTES);
                            bad = mbar_wait_conv(smem_u32(&hd.full[stage]), phase, abort_addr, bad, lead_lane);
                            if (hi - k0 < 64) asm volatile("fence.acq_rel.cluster;" ::: "memory");   // the tail warps' zeros
                            tc_fence_after();
                            if (lead_lane && !bad) {
                                for (int k = 0; k < slices; ++k) {
                                    umma_pair_n(d_tmem, a_desc + 128u * k, b_desc + 128u * k, idesc, accumulate);
                                    accumulate = 1;
                                }
                                umma_commit_both(smem_u32(&hd.empty[stage]));
                            }
                            if (++stage == G_STAGES) { stage = 0; phase ^= 1u; }
                        }
                    }
                } else {
                    for (int kb = 0; kb < p.k_steps; ++kb) {
                        const uint32_t src = ring + stage * G_STAGE_BYTES;
                        const uint64_t a_desc = smem_desc_mn(src), b_desc = smem_desc(src + 2 * G_BOX_BYTES);
                        bad = mbar_wait_conv(smem_u32(&hd.full[stage]), phase, abort_addr, bad, lead_lane);
                        tc_fence_after();
                        if (lead_lane && !bad) {
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                umma_pair_n(d_tmem, a_desc + 128u * k, b_desc + 2u * k, idesc, (kb | k) != 0 ? 1u : 0u);
                            umma_commit_both(smem_u32(&hd.empty[stage]));
                        }
                        if (++stage == G_STAGES) { stage = 0; phase ^= 1u; }
                    }
                }
                if (__any_sync(0xFFFFFFFFu, bad != 0u)) break;
                if (lead_lane) umma_commit_both(smem_u32(&hd.tfull[acc]));
            }
        }
    } else if (warp == 2) {
        // ---- scheduler, leader CTA (see the forward kernel for why claims are held back to G_CLAIM_LEAD k-steps) ----
        if (lane == 0 && leader) {
            const int per_expert = p.m_blocks * p.n_blocks;            // weight gradients
            const int total = WEIGHTS ? E * per_expert : s_pre[E] * p.m_blocks;
            int e = 0, pub_k = 0;
            for (int i = 0;; ++i) {
                if (pub_k - *prod_k >= G_CLAIM_LEAD) {
                    const unsigned long long t0 = global_ns();
                    uint32_t n = 0;
                    bool give_up = false;
                    while (pub_k - *prod_k >= G_CLAIM_LEAD) {
                        __nanosleep(256);
                        if ((++n & 63u) == 0u && (*abort_flag || global_ns() - t0 > WAIT_LIMIT_NS)) { give_up = true; break; }
                    }
                    if (give_up) { *abort_flag = 1; break; }
                }
                const unsigned int c = atomicAdd(p.counter, 1u);
                const int w = c < (unsigned)total ? (int)c : total;
                const int q = i & (G_SLOTS - 1);
                if (!mbar_wait(smem_u32(&hd.sched_empty[q]), (((uint32_t)i / G_SLOTS) & 1u) ^ 1u, abort_flag)) break;
                int4 item = make_int4(0, 0, 0, 0);
                if (w < total) {
                    if constexpr (WEIGHTS) {
                        const int ex = s_order[w / per_expert], local = w % per_expert;
                        item = make_int4(local % p.m_blocks, 1, ex, local / p.m_blocks);
                        pub_k += s_steps[ex];
                    } else {
                        while (w >= s_pre[e + 1] * p.m_blocks) ++e;    // w only grows
                        const int nt = s_pre[e + 1] - s_pre[e], local = w - s_pre[e] * p.m_blocks;
                        const int wb = local / nt;                     // block by block, so that an expert's token tiles share it
                        int tile = local - wb * nt, r = s_rep[e];
                        for (;; ++r) {
                            const int n = (s_hi[r] - s_lo[r] + G_TILE - 1) / G_TILE;
                            if (tile < n) break;
                            tile -= n;
                        }
                        const int row0 = s_lo[r] + tile * G_TILE;
                        item = make_int4(row0, min(G_TILE, s_hi[r] - row0), e, wb);
                        pub_k += p.k_steps;
                    }
                }
                hd.item[q] = item;
                st_cluster_v4(map_to_cta(smem_u32(&hd.item[q]), 1), item);
                mbar_arrive(smem_u32(&hd.sched_full[q]));
                mbar_arrive_cluster_release(map_to_cta(smem_u32(&hd.sched_full[q]), 1));
                if (w >= total) break;
            }
        }
    } else if (warp == 3) {
        // ---- tail warp, both CTAs: zeroes the rows behind a segment's end inside the last MMA of a step ----
        if constexpr (WEIGHTS) {
            int stage = 0;
            uint32_t part_phase = 0, bad = 0;                          // one phase bit per stage
            for (int i = 0; take_item_warp(i, it); ++i) {
                const int boxes = 2 + (columns_of(it) >> 7);           // 64-column boxes of both operands in this CTA
                for (int r = s_rep[it.e]; r < s_rep[it.e + 1]; ++r) {
                    const int hi = s_hi[r];
                    for (int k0 = s_lo[r]; k0 < hi; k0 += 64) {
                        const int valid = hi - k0;
                        if (valid < 64 && (valid & 15) != 0) {
                            bad = mbar_wait_conv(smem_u32(&hd.part[stage]), (part_phase >> stage) & 1u, abort_addr, bad, 1u);
                            part_phase ^= 1u << stage;
                            if (!bad) {
                                const int zero = ((valid + 15) & ~15) - valid, vecs = zero * 8;    // whole rows: the swizzle stays inside one
                                uint8_t* const base = smem_raw + (ring - raw) + stage * G_STAGE_BYTES + valid * 128;
                                for (int v = lane; v < boxes * vecs; v += 32)
                                    *reinterpret_cast<uint4*>(base + (v / vecs) * G_BOX_BYTES + (v % vecs) * 16) = make_uint4(0u, 0u, 0u, 0u);
                                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");       // before the tensor core reads them
                            }
                            __syncwarp();
                            if (lane == 0 && !bad) mbar_arrive_cluster_release(map_to_cta(smem_u32(&hd.full[stage]), 0));
                        }
                        if (++stage == G_STAGES) stage = 0;
                    }
                }
                if (__any_sync(0xFFFFFFFFu, bad != 0u)) break;
            }
        }
    } else {
        // ---- epilogue, both CTAs: 32 rows of D per warp (its TMEM quadrant), every other 32 columns ----
        const int quad = warp & 3;
        const int c_first = 32 * ((warp - 4) >> 2);
        constexpr int CSTEP = 32 * (G_EPI_WARPS / 4);
        const int d_row = (int)rank * 128 + quad * 32 + lane;          // row of D inside the pair's 256
        for (int i = 0;; ++i) {
            if (!take_item(i, it)) break;
            __syncwarp();
            if (lane == 0) release_item(i);
            if (it.valid == 0) break;
            const int acc = i & 1;
            if (!mbar_wait(smem_u32(&hd.tfull[acc]), ((uint32_t)i >> 1) & 1u, abort_flag)) break;
            tc_fence_after();
            const uint32_t taddr = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)(acc * G_TILE);
            const int n = columns_of(it);
            if constexpr (KIND == GRAD_ACT) {
                const int f = it.b * 256 + d_row;
                const bool live = f < p.F;                             // the last block may be half a block (warp-uniform)
                const int blk = f / kCheckpointBlock;
#pragma unroll 1
                for (int c = c_first; c < n && live; c += CSTEP) {
                    uint32_t v[32];
                    tmem_ld32(taddr + c, v);
                    const int row = it.a + c, rem = it.valid - c;
                    // lane j: the exponents of row j for the warp's two blocks
                    uint32_t ex = 0;
                    if (lane < rem) {
                        const uint16_t* e0 = p.exps + (size_t)(blk - (lane >> 4)) * p.rows + row + lane;
                        ex = (uint32_t)__ldg(e0) | ((uint32_t)__ldg(e0 + p.rows) << 16);
                    }
                    const uint16_t* code = reinterpret_cast<const uint16_t*>(p.codes) + (size_t)row * p.F + f;
                    uint16_t *dg = p.out0 + (size_t)row * p.F + f, *du = p.out1 + (size_t)row * p.F + f, *act = p.out2 + (size_t)row * p.F + f;
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        const uint32_t pair = __shfl_sync(0xFFFFFFFFu, ex, j) >> (lane & 16);
                        if (j < rem) {
                            const uint32_t k = __ldg(code);
                            const float g = (float)(int8_t)k * checkpoint_scale(pair & 255u);
                            const float u = (float)(int8_t)(k >> 8) * checkpoint_scale((pair >> 8) & 255u);
                            const float da = __uint_as_float(v[j]);
                            const float s = __fdividef(1.0f, 1.0f + __expf(-g)), gs = g * s;
                            *dg = to_bf16(da * u * (s * (1.0f + g * (1.0f - s))));
                            *du = to_bf16(da * gs);
                            *act = to_bf16(gs * u);
                        }
                        code += p.F;
                        dg += p.F;
                        du += p.F;
                        act += p.F;
                    }
                }
            } else if constexpr (KIND == GRAD_DX) {
                uint16_t* const col = p.out0 + (size_t)it.a * p.H + it.b * 256 + d_row;
#pragma unroll 1
                for (int c = c_first; c < n; c += CSTEP) {
                    uint32_t v[32];
                    tmem_ld32(taddr + c, v);
                    tmem_ld_wait();
                    uint16_t* ptr = col + (size_t)c * p.H;
                    const int rem = it.valid - c;
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        if (j < rem) *ptr = to_bf16(__uint_as_float(v[j]));
                        ptr += p.H;
                    }
                }
            } else {
                const bool empty = s_steps[it.e] == 0;                 // nothing was accumulated: the gradient is zero
                const int h = it.a * 256 + d_row;
#pragma unroll 1
                for (int c = c_first; c < n; c += CSTEP) {
                    uint32_t v[32];
                    if (empty) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = 0u;
                    } else {
                        tmem_ld32(taddr + c, v);
                        tmem_ld_wait();
                    }
                    if constexpr (KIND == GRAD_GATEUP) {
                        // columns 0..127: dWg, 128..255: dWu; 32 lanes write 32 consecutive h of one feature
                        const int f = it.b * 128 + (c & 127);
                        uint16_t* ptr = (c < 128 ? p.out0 : p.out1) + ((size_t)it.e * p.F + f) * p.H + h;
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            *ptr = to_bf16(__uint_as_float(v[j]));
                            ptr += p.H;
                        }
                    } else {
                        // a lane writes 32 consecutive features of its h
                        uint4* ptr = reinterpret_cast<uint4*>(p.out0 + ((size_t)it.e * p.H + h) * p.F + it.b * 256 + c);
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            ptr[j] = make_uint4(pack_bf16(__uint_as_float(v[8 * j]), __uint_as_float(v[8 * j + 1])),
                                                pack_bf16(__uint_as_float(v[8 * j + 2]), __uint_as_float(v[8 * j + 3])),
                                                pack_bf16(__uint_as_float(v[8 * j + 4]), __uint_as_float(v[8 * j + 5])),
                                                pack_bf16(__uint_as_float(v[8 * j + 6]), __uint_as_float(v[8 * j + 7])));
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(map_to_cta(smem_u32(&hd.tempty[acc]), 0));
        }
    }

    // ---- teardown, as in the forward kernel: a role that gave up tells the peer CTA ----
    if (*abort_flag)
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_to_cta(abort_addr, 1u - rank)), "r"(1) : "memory");
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    if (tid == 0 && *abort_flag) director_set_status(p.status, DIRECTOR_ERR_TIMEOUT);
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
    }
}

template <int KIND>
int launch_grad(director_ctx* ctx, const char* name, const CUtensorMap& a0, const CUtensorMap& a1, const CUtensorMap& b0,
                const CUtensorMap& b1, const GradParams& p, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * ctx->pair_clusters));
    cfg.blockDim = dim3(G_THREADS);
    cfg.dynamicSmemBytes = (size_t)grad_smem_bytes(p.n_rep, p.E);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;    // see chain_prologue()
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = chain_allowed(st) ? 2 : 1;
    LaunchScope scope(ctx, st, name);
    return cuda_status(cudaLaunchKernelEx(&cfg, grouped_grad_kernel<KIND>, a0, a1, b0, b1, p));
}

// The four launches for one set of experts over one segment table.
int ffn_grad_pass(director_ctx* ctx, const FfnGrad& f, const int32_t* seg_offsets, int n_experts, int n_rep, int Fw, bool dense,
                  void* dgu, void* act, unsigned int* counters, cudaStream_t st) {
    const int H = ctx->shape.H;
    const uint64_t rows = (uint64_t)f.kept.rows;
    uint16_t* const dg = static_cast<uint16_t*>(dgu);
    uint16_t* const du = dg + rows * (uint64_t)Fw;
    CUtensorMap wd, wg, wu;                                   // left operands: boxes of 64 contraction rows
    CUtensorMap x_mn, dy_mn, dg_mn, du_mn, act_mn;            // operands of the weight gradients: the same boxes
    CUtensorMap dy_k, dg_k, du_k;                             // token rows, contraction along the row
    if (!map_2d(ctx, &wd, f.w_down, (uint64_t)n_experts * H, Fw, 64) || !map_2d(ctx, &wg, f.w_gate, (uint64_t)n_experts * Fw, H, 64) ||
        !map_2d(ctx, &wu, f.w_up, (uint64_t)n_experts * Fw, H, 64) || !map_2d(ctx, &x_mn, f.x, rows, H, 64) ||
        !map_2d(ctx, &dy_mn, f.dy, rows, H, 64) || !map_2d(ctx, &dg_mn, dg, rows, Fw, 64) || !map_2d(ctx, &du_mn, du, rows, Fw, 64) ||
        !map_2d(ctx, &act_mn, act, rows, Fw, 64) || !map_2d(ctx, &dy_k, f.dy, rows, H) || !map_2d(ctx, &dg_k, dg, rows, Fw) ||
        !map_2d(ctx, &du_k, du, rows, Fw))
        return DIRECTOR_ERR_CUDA;
    GradParams p{seg_offsets, ctx->d_rep_start, ctx->d_rep_slot, n_experts, n_rep, (int)rows, dense ? 1 : 0, H, Fw, 0, 0, 0,
                 f.kept.codes, f.kept.exps, nullptr, nullptr, nullptr, ctx->d_status, counters};
    p.m_blocks = (Fw + 255) / 256;
    p.k_steps = H / 64;
    p.out0 = dg;
    p.out1 = du;
    p.out2 = static_cast<uint16_t*>(act);
    int rc = launch_grad<GRAD_ACT>(ctx, "grouped_grad_act_kernel", wd, wd, dy_k, dy_k, p, st);
    if (rc != DIRECTOR_OK) return rc;
    p.m_blocks = H / 256;
    p.k_steps = 2 * (Fw / 64);
    p.out0 = static_cast<uint16_t*>(f.dx);
    p.counter = counters + 1;
    rc = launch_grad<GRAD_DX>(ctx, "grouped_grad_dx_kernel", wg, wu, dg_k, du_k, p, st);
    if (rc != DIRECTOR_OK) return rc;
    p.n_blocks = Fw / 128;
    p.out0 = static_cast<uint16_t*>(f.dw_gate);
    p.out1 = static_cast<uint16_t*>(f.dw_up);
    p.counter = counters + 2;
    rc = launch_grad<GRAD_GATEUP>(ctx, "grouped_grad_gateup_kernel", x_mn, x_mn, dg_mn, du_mn, p, st);
    if (rc != DIRECTOR_OK) return rc;
    p.n_blocks = (Fw + 255) / 256;
    p.out0 = static_cast<uint16_t*>(f.dw_down);
    p.counter = counters + 3;
    return launch_grad<GRAD_DOWN>(ctx, "grouped_grad_down_kernel", dy_mn, dy_mn, act_mn, act_mn, p, st);
}

template <int KIND>
bool grad_opt_in() {
    return cudaFuncSetAttribute(grouped_grad_kernel<KIND>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                grad_smem_bytes(kMaxG, kMaxE)) == cudaSuccess;
}

}  // namespace

int ffn_grad_init(director_ctx*) {
    return grad_opt_in<GRAD_ACT>() && grad_opt_in<GRAD_DX>() && grad_opt_in<GRAD_GATEUP>() && grad_opt_in<GRAD_DOWN>()
               ? DIRECTOR_OK : DIRECTOR_ERR_CUDA;
}

// routed: the permuted rows.  shared (x != nullptr): the S shared experts as one FFN of width S*F over the batch's own rows.
int launch_expert_ffn_backward(director_ctx* ctx, int T, const int32_t* seg_offsets, const FfnGrad& routed, const FfnGrad& shared,
                               cudaStream_t st) {
    StageScope stage(ctx, st, "stage_expert_ffn_backward");
    const director_shape& s = ctx->shape;
    if (cudaMemsetAsync(ctx->d_grad_sched, 0, 8 * sizeof(unsigned int), st) != cudaSuccess) return DIRECTOR_ERR_CUDA;
    const int rc = ffn_grad_pass(ctx, routed, seg_offsets, s.E, ctx->n_replicas, s.F, false, ctx->d_dgu, ctx->d_hidden,
                                 ctx->d_grad_sched, st);
    if (rc != DIRECTOR_OK || shared.x == nullptr) return rc;
    return ffn_grad_pass(ctx, shared, nullptr, 1, 1, s.S * s.F, true, ctx->d_dgu_shared, ctx->d_hidden_shared,
                         ctx->d_grad_sched + 4, st);
}

}  // namespace director
