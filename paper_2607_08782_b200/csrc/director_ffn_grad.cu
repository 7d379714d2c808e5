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
// Two launches: GRAD_ACT, and the other three kinds together - they need nothing of each other, and the many short work items
// of the weight gradients fill the idle end that the few long ones of GRAD_DX would leave.  The shared experts are one more
// expert with a width and row space of its own (problem 1), in the same launches.
//
// CTA pairs as in the forward kernel (tcgen05.mma cta_group::2, M = 256: 128 rows of D per CTA, accumulators of up to 256
// columns, two of them), operands by TMA through a ring of 32 KB stages.  What differs is the operands' direction: no matrix
// is transposed in memory.  An operand whose rows run along the contraction (Wd, Wg, Wu as the left operand; everything in
// the weight gradients) is loaded as boxes of 64 contraction rows x 64 columns and handed to the tensor core as an
// MN-major tile.
//   GRAD_ACT / GRAD_DX: D[feature, token], as in the forward: 256 weight columns x up to 256 tokens, the token count a runtime
//     operand in steps of 32, so a segment's ragged end costs little.
//   GRAD_GATEUP: D[f, h]: CTA 0 of the pair holds 128 features of dg, CTA 1 the same 128 of du, and both share 256 columns of
//     xp.   GRAD_DOWN: D[h, f]: 256 columns of dyp x up to 256 of act.
//     The contraction runs over the segments of all of an expert's replicas.  Where a segment ends inside a 64-row step the
//     rows behind it belong to another expert: the step issues only the MMAs it needs (16 rows each), and a warp of each CTA
//     zeroes the rows behind the end inside the last one, in both operands (a zero times another expert's infinity would be
//     NaN).  Experts are taken by descending length, so that the longest contractions do not end the launch.
//     A tile goes out through shared memory and TMA stores: a lane holds 32 consecutive columns of one row, which as plain
//     stores would touch 32 lines an instruction.  An expert without rows gets its zeros the same way.
// Work items are claimed from a global counter and handed to all roles through a small ring, as in the forward kernel.
// Every wait is bounded; an expired one raises DIRECTOR_ERR_TIMEOUT.
//
// What bounds it: long segments, the tensor pipe - a 64-deep step takes 508-520 cycles, the pipe's four MMAs 512 - at the clock the
// power cap leaves (8192 rows, eight experts, H = 4096, F = 14336: 0.73-0.85 and 3.65-4.0 ms for the two launches, 1.2-1.3
// PFLOP/s); few rows per expert, HBM (8168 rows, 128 experts, H = 2048, F = 768: 77-80 and 307 us, 5.3 TB/s of weights read and
// gradients written); a handful of rows, the launches' own latencies (8 us each).
#include "director_common.cuh"
#include "director_umma.cuh"

#include <cuda_bf16.h>

namespace director {

using namespace umma;

namespace {

enum GradKind { GRAD_ACT = 0, GRAD_DX = 1, GRAD_GATEUP = 2, GRAD_DOWN = 3 };

constexpr int G_STAGES = 6;
// GRAD_ACT with tiles of at most 64 tokens needs 20 KB a stage (one box of tokens): nine fit into the same ring.  Such a launch
// streams weights, and a stage comes back about 2500 cycles after it was asked for: what counts is how many are under way.
constexpr int G_FEW_STAGES = 9;
constexpr int G_BOX_BYTES = 64 * 128;                  // 64 rows of 64 bf16 columns
constexpr int G_STAGE_BYTES = 4 * G_BOX_BYTES;         // 16 KB of each operand
constexpr int G_FEW_STAGE_BYTES = 2 * G_BOX_BYTES + G_BOX_BYTES / 2;
static_assert(G_FEW_STAGES * G_FEW_STAGE_BYTES <= G_STAGES * G_STAGE_BYTES, "the deeper ring fits into the ordinary one");
// Epilogue warps, a multiple of the four TMEM lane quadrants; each takes every second or third chunk of 32 columns.  GRAD_ACT's epilogue (a
// sigmoid, two kept values in and three outputs an element) bounds contractions shorter than about 2048: at H = 1536, F = 640,
// 120 432 rows, the launch took 320 us with 8 warps, 291 with 12 and 293 with 16, at H = 4096 780, 754 and 766 us.
constexpr int grad_epi_warps(int phase) { return phase == 0 ? 12 : 8; }
constexpr int grad_threads(int phase) { return 128 + 32 * grad_epi_warps(phase); }   // producer, MMA, scheduler and tail warps + epilogue
constexpr int G_TILE = 256;                            // most tokens per tile; accumulators are this many columns apart
constexpr int G_SLOTS = 4;                             // ring of work items
constexpr int G_PACED_STEPS = 256;                     // contractions this long are paced
constexpr int G_CLAIM_LEAD = 32;                       // k-steps of claimed work ahead of the producer

constexpr int G_OUT_BYTES = 32 * 64;                   // per epilogue warp: 32 rows x 32 bf16 columns of a weight gradient

struct GradHeader {
    uint64_t full[G_FEW_STAGES], empty[G_FEW_STAGES];
    uint64_t part[G_STAGES];                           // this CTA's loads of a step that still has rows to be zeroed
    uint64_t tfull[2], tempty[2], sched_full[G_SLOTS], sched_empty[G_SLOTS];
    int4 item[G_SLOTS];
    uint32_t tmem;
    int abort;
    int prod_k;                                        // k-steps issued by the scheduler CTA's producer
    int warp_sum[2][20];
    int tile;                                          // tokens per full tile of this launch
};
// experts: all of them, the shared one among them; n_rep: their segments
constexpr int grad_out_bytes(int phase) { return phase == 1 ? grad_epi_warps(1) * G_OUT_BYTES : 0; }
constexpr int grad_smem_bytes(int phase, int n_rep, int experts) {
    return 1024 + G_STAGES * G_STAGE_BYTES + grad_out_bytes(phase) + (int)sizeof(GradHeader) + 8 * n_rep + 4 * (5 * experts + 3);
}
static_assert(grad_smem_bytes(1, kMaxG + 1, kMaxE + 1) <= 232448, "the ring does not fit with the largest tables");
static_assert(kMaxE + 1 <= grad_threads(1), "one thread per expert builds the tables");

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

// Problem 0: the routed experts over the segment table.  Problem 1: the shared experts, one FFN over all rows of the batch.
struct GradProblem {
    int F;
    int rows;                      // rows of the permuted operands
    const int8_t* codes;           // the checkpoint
    const uint16_t* exps;
    uint16_t *dg, *du, *act;       // written by GRAD_ACT, [rows, F]
    uint16_t* dx;                  // [rows, H]
};
// What a launch loads from and, for the weight gradients, stores to.  _K: boxes of 32 rows, contraction along the row (as many
// as a tile's tokens need); all others: boxes of 64 contraction rows; OUT_*: boxes of 32 rows x 32 columns.
enum GradMap { MAP_WD, MAP_WG, MAP_WU, MAP_DY_K, MAP_DG_K, MAP_DU_K, MAP_X, MAP_DG, MAP_DU, MAP_DY, MAP_ACT, MAP_OUT_G, MAP_OUT_U,
               MAP_OUT_D, GRAD_MAPS };
struct GradMaps {
    CUtensorMap m[2][GRAD_MAPS];
};
struct GradParams {
    const int32_t* seg_offsets;    // [G+1], clamped to [0, rows]
    const int32_t* rep_start;      // [E+1] replicas of expert e: rep_slot[rep_start[e] .. rep_start[e+1])
    const int32_t* rep_slot;
    int E;                         // routed experts
    int experts;                   // E, or E + 1 with the shared one behind them
    int n_rep;                     // segments: the routed experts' replicas, and the shared expert's one
    int H;
    GradProblem prob[2];
    int32_t* status;
    unsigned int* counter;         // next unclaimed work item of this launch (zero when the kernel starts)
    unsigned int* other_counter;   // the other launch's, cleared here for its next run
};

struct GradItem {
    int a, valid, e, b, kind;      // tokens: first row, rows (0: end), expert, block;   weights: h block, 1, expert, f block
    int later;                     // tokens: not the first tile of its segment
};

__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, uint32_t src, int x, int y) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];"
                 ::"l"(reinterpret_cast<uint64_t>(map)), "r"(src), "r"(x), "r"(y) : "memory");
}

// 1 / (1 + exp(-g)) from the two approximate units alone.  exp(-g) below 2^-126 counts as zero, above 2^127 as infinity, and so does the
// result: all it costs are sigmoids below 2^-126.
__device__ __forceinline__ float sigmoid(float g) {
    float e, s;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(g * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.0f + e));
    return s;
}
// a load that does not go through L1
__device__ __forceinline__ int ld_relaxed(const int32_t* p) {
    int v;
    asm volatile("ld.relaxed.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint64_t offset_by(const void* base, uint32_t bytes) {
    uint64_t r;
    asm("mad.wide.u32 %0, %1, 1, %2;" : "=l"(r) : "r"(bytes), "l"(reinterpret_cast<uint64_t>(base)));
    return r;
}
__device__ __forceinline__ void store_u32(uint64_t addr, uint32_t v) {
    asm volatile("st.global.b32 [%0], %1;" ::"l"(addr), "r"(v) : "memory");
}

// 16 bytes into the shared memory of a CTA of the cluster, counted on an mbarrier there when they have arrived
__device__ __forceinline__ void st_async_v4(uint32_t cluster_addr, int4 v, uint32_t cluster_bar) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];"
                 ::"r"(cluster_addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w), "r"(cluster_bar) : "memory");
}

// PHASE 0: GRAD_ACT.  PHASE 1: GRAD_DX, GRAD_GATEUP, GRAD_DOWN.
template <int PHASE>
__global__ void __launch_bounds__(grad_threads(PHASE), 1)
grouped_grad_kernel(const __grid_constant__ GradMaps maps, const __grid_constant__ GradParams p) {
    constexpr int G_THREADS = grad_threads(PHASE), G_EPI_WARPS = grad_epi_warps(PHASE);
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t ring = (raw + 1023u) & ~1023u;
    uint8_t* const out_buf = smem_raw + (ring - raw) + G_STAGES * G_STAGE_BYTES;      // phase 1: [G_EPI_WARPS][G_OUT_BYTES]
    GradHeader& hd = *reinterpret_cast<GradHeader*>(out_buf + grad_out_bytes(PHASE));
    const int experts = p.experts;
    int32_t* const s_rep = reinterpret_cast<int32_t*>(&hd + 1);        // [experts+1] first segment of every expert
    int32_t* const s_pre = s_rep + (experts + 1);                      // [experts+1] token work items before expert e
    int32_t* const s_wpre = s_pre + (experts + 1);                     // [experts+1] weight work items before s_order[i]
    int32_t* const s_steps = s_wpre + (experts + 1);                   // [experts] 64-row steps of expert e
    int32_t* const s_order = s_steps + experts;                        // [experts] experts, longest first
    int32_t* const s_lo = s_order + experts;                           // [n_rep] rows of every segment
    int32_t* const s_hi = s_lo + p.n_rep;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = cluster_ctarank();
    const bool leader = rank == 0;
    volatile int* const abort_flag = &hd.abort;
    volatile int* const prod_k = &hd.prod_k;
    const uint32_t abort_addr = smem_u32(&hd.abort);
    const int h_blocks = p.H / 256;
    auto problem_of = [&](int e) -> int { return e >= p.E ? 1 : 0; };

    // ---- set-up.  Under programmatic dependent launch this runs while the kernel before is still ending.  Phase 0 waits for that
    // kernel before it reads the segment table, and lets phase 1 start only after its wait: when a CTA of phase 1 runs, all that came
    // before phase 0 - the segment table's writer among it - has ended, so phase 1 builds its tables ahead of its own wait (2.5 us
    // of a small batch's time).  Without the launch attribute the instructions do nothing. ----
    if (tid == 0) {
        *abort_flag = 0;
        *prod_k = 0;
        for (int s = 0; s < G_FEW_STAGES; ++s) {
            mbar_init(smem_u32(&hd.full[s]), 2);
            mbar_init(smem_u32(&hd.empty[s]), 1);
        }
        for (int s = 0; s < G_STAGES; ++s) mbar_init(smem_u32(&hd.part[s]), 1);
        for (int a = 0; a < 2; ++a) {
            mbar_init(smem_u32(&hd.tfull[a]), 1);
            mbar_init(smem_u32(&hd.tempty[a]), 2 * G_EPI_WARPS);
        }
        // readers of an item: the MMA warp, both producers, all epilogue warps, in phase 1 both tail warps
        for (int q = 0; q < G_SLOTS; ++q) {
            mbar_init(smem_u32(&hd.sched_full[q]), 1);
            mbar_init(smem_u32(&hd.sched_empty[q]), 3 + 2 * G_EPI_WARPS + 2 * PHASE);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&hd.tmem)), "r"(TMEM_COLS)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    if (warp == 2)
        for (int i = lane; i < (p.experts > p.E ? 2 : 1) * GRAD_MAPS; i += 32)
            asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&maps.m[0][0] + i)) : "memory");
    if constexpr (PHASE == 0) {
        asm volatile("griddepcontrol.wait;" ::: "memory");
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    }

    // ---- tables ----
    for (int r = tid; r < p.n_rep; r += G_THREADS) {
        int lo = 0, hi = p.prob[1].rows;
        if (r < p.n_rep - (experts - p.E)) {
            const int g = ld_relaxed(p.rep_slot + r);
            lo = min(max(ld_relaxed(p.seg_offsets + g), 0), p.prob[0].rows);
            hi = min(max(ld_relaxed(p.seg_offsets + g + 1), lo), p.prob[0].rows);
        }
        s_lo[r] = lo;
        s_hi[r] = hi;
    }
    for (int e = tid; e <= experts; e += G_THREADS) s_rep[e] = e <= p.E ? ld_relaxed(p.rep_start + e) : p.n_rep;
    __syncthreads();
    {
        int steps = 0;                                  // 64-row steps of expert tid
        bool long_one = false;                          // a segment of more than 64 rows
        if (tid < experts) {
            for (int r = s_rep[tid]; r < s_rep[tid + 1]; ++r) {
                steps += (s_hi[r] - s_lo[r] + 63) / 64;
                long_one |= s_hi[r] - s_lo[r] > 64;
            }
            s_steps[tid] = steps;
        }
        // Token tiles are 256 rows; where that leaves fewer items than CTA pairs, 128 or 64: the same products on more SMs, each tile
        // with its own pass over the weights, which then come from L2 (1579 rows of three experts: 7 items of 256 rows on 74
        // pairs, 26 of 64).  Every CTA comes to the same tile.
        int tiles[3] = {0, 0, 0};                       // of 256, 128 and 64 rows
        int blocks = 0;
        if (tid < experts) {
            blocks = PHASE == 0 ? (p.prob[problem_of(tid)].F + 255) / 256 : h_blocks;
            for (int r = s_rep[tid]; r < s_rep[tid + 1]; ++r)
#pragma unroll
                for (int k = 0; k < 3; ++k) tiles[k] += (s_hi[r] - s_lo[r] + (G_TILE >> k) - 1) / (G_TILE >> k);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int in_warp = __reduce_add_sync(0xFFFFFFFFu, tiles[k] * blocks);
            if (lane == 0) hd.warp_sum[k][warp] = in_warp;
        }
        const bool any_long = __syncthreads_or(long_one ? 1 : 0) != 0;
        int total[2] = {0, 0};
        for (int w = 0; w < G_THREADS / 32; ++w) { total[0] += hd.warp_sum[0][w]; total[1] += hd.warp_sum[1][w]; }
        __syncthreads();
        const int pairs = (int)(gridDim.x >> 1), shift = !any_long ? 2 : total[0] >= pairs ? 0 : total[1] >= pairs ? 1 : 2;
        const int tile = G_TILE >> shift;
        int items = (shift == 0 ? tiles[0] : shift == 1 ? tiles[1] : tiles[2]) * blocks;
        if (tid == 0) hd.tile = tile;
        if (PHASE == 1 && tid < experts) {
            int before = 0;
            for (int e = 0; e < experts; ++e) before += s_steps[e] > steps || (s_steps[e] == steps && e < tid) ? 1 : 0;
            s_order[before] = tid;
        }
        __syncthreads();
        int w_items = 0;
        if (PHASE == 1 && tid < experts) {
            const int F = p.prob[problem_of(s_order[tid])].F;
            w_items = h_blocks * (F / 128 + (F + 255) / 256);
        }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xFFFFFFFFu, items, o), w = __shfl_up_sync(0xFFFFFFFFu, w_items, o);
            if (lane >= o) { items += v; w_items += w; }
        }
        if (lane == 31) { hd.warp_sum[0][warp] = items; hd.warp_sum[1][warp] = w_items; }
        __syncthreads();
        for (int w = 0; w < warp; ++w) { items += hd.warp_sum[0][w]; w_items += hd.warp_sum[1][w]; }
        if (tid < experts) { s_pre[tid + 1] = items; s_wpre[tid + 1] = w_items; }
        if (tid == 0) { s_pre[0] = 0; s_wpre[0] = 0; }
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    if constexpr (PHASE == 1) {
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
        asm volatile("griddepcontrol.wait;" ::: "memory");
    }
    if (tid == 0 && blockIdx.x == 0) *p.other_counter = 0u;   // its launch has ended (waited for above), or has not begun
    const uint32_t tmem_base = hd.tmem;
    const bool few = PHASE == 0 && hd.tile <= 64;
    const int n_stages = few ? G_FEW_STAGES : G_STAGES, stage_bytes = few ? G_FEW_STAGE_BYTES : G_STAGE_BYTES;

    // ---- work items: claimed by one thread of the leader CTA, read by every role of both ----
    auto take_item = [&](int i, GradItem& it) -> bool {
        const int q = i & (G_SLOTS - 1);
        const uint32_t par = ((uint32_t)i / G_SLOTS) & 1u, bar = smem_u32(&hd.sched_full[q]);
        const bool ok = mbar_wait(bar, par, abort_flag);
        if (ok) {
            const int4 v = hd.item[q];
            it = GradItem{v.x, v.y, v.z, v.w & 0x07FFFFFF, v.w >> 28, (v.w >> 27) & 1};
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
        it.kind = PHASE == 0 ? GRAD_ACT : __shfl_sync(0xFFFFFFFFu, it.kind, 0);
        it.later = __shfl_sync(0xFFFFFFFFu, it.later, 0);
        if (ok && lane == 0) release_item(i);
        return ok && it.valid != 0;
    };
    auto is_weights = [&](const GradItem& it) -> bool { return PHASE == 1 && it.kind != GRAD_DX; };
    auto columns_of = [&](const GradItem& it) -> int {            // N of the item's MMAs
        if (is_weights(it)) return it.kind == GRAD_GATEUP ? 256 : min(256, p.prob[problem_of(it.e)].F - it.b * 256);
        return (it.valid + 31) / 32 * 32;
    };
    auto token_steps = [&](int e) -> int { return PHASE == 0 ? p.H / 64 : 2 * (p.prob[problem_of(e)].F / 64); };

    GradItem it{};
    if (warp == 0) {
        // ---- operand producer, both CTAs ----
        const uint32_t lead_lane = elect_one() ? 1u : 0u;
        int stage = 0, issued_k = 0;
        uint32_t phase = 0, bad = 0;
        for (int i = 0; take_item_warp(i, it); ++i) {
            const int pr = problem_of(it.e);
            const CUtensorMap* const map = maps.m[pr];
            if (is_weights(it)) {
                const int half = columns_of(it) >> 1;             // columns of the right operand this CTA supplies: 128 or 64
                const CUtensorMap *ma, *mb;
                int m_col, n_col;
                if (it.kind == GRAD_GATEUP) {
                    ma = map + (rank ? MAP_DU : MAP_DG);
                    m_col = it.b * 128;
                    mb = map + MAP_X;
                    n_col = it.a * 256 + (int)rank * 128;
                } else {
                    ma = map + MAP_DY;
                    m_col = it.a * 256 + (int)rank * 128;
                    mb = map + MAP_ACT;
                    n_col = it.b * 256 + (int)rank * half;
                }
                const uint32_t tx = 2 * G_BOX_BYTES + half * 128;
                for (int r = s_rep[it.e]; r < s_rep[it.e + 1]; ++r) {
                    const int hi = s_hi[r];
                    for (int k0 = s_lo[r]; k0 < hi; k0 += 64) {
                        // a step whose last MMA reaches past the segment is reported to this CTA's tail warp first
                        const bool tail = hi - k0 < 64 && ((hi - k0) & 15) != 0;
                        const uint32_t dst = ring + stage * stage_bytes;
                        const uint32_t bar = tail ? map_to_cta(smem_u32(&hd.part[stage]), rank) : map_to_cta(smem_u32(&hd.full[stage]), 0);
                        bad = mbar_wait_conv(smem_u32(&hd.empty[stage]), phase ^ 1u, abort_addr, bad, lead_lane);
                        ++issued_k;
                        if (lead_lane && !bad) {
                            mbar_expect_tx_cluster(bar, tx);
                            tma_load_2d_pair(dst, ma, bar, m_col, k0);
                            tma_load_2d_pair(dst + G_BOX_BYTES, ma, bar, m_col + 64, k0);
                            tma_load_2d_pair(dst + 2 * G_BOX_BYTES, mb, bar, n_col, k0);
                            if (half > 64) tma_load_2d_pair(dst + 3 * G_BOX_BYTES, mb, bar, n_col + 64, k0);
                            if (leader) *prod_k = issued_k;
                        }
                        if (++stage == n_stages) { stage = 0; phase ^= 1u; }
                    }
                }
            } else {
                const int m_col = it.b * 256 + (int)rank * 128;
                const int half = columns_of(it) >> 1, x_row = it.a + (int)rank * half;      // tokens this CTA supplies
                const int boxes = (half + 31) >> 5;                       // of 32 tokens
                const uint32_t tx = 2 * G_BOX_BYTES + boxes * (G_BOX_BYTES / 2);
                const int k_steps = token_steps(it.e), e = pr ? 0 : it.e;
                for (int kb = 0; kb < k_steps; ++kb) {
                    const bool second = PHASE == 1 && kb >= k_steps / 2;
                    const int k = (second ? kb - k_steps / 2 : kb) * 64;
                    const int w_row = e * (PHASE == 0 ? p.H : p.prob[pr].F) + k;
                    const CUtensorMap* ma = map + (PHASE == 0 ? MAP_WD : second ? MAP_WU : MAP_WG);
                    const CUtensorMap* mb = map + (PHASE == 0 ? MAP_DY_K : second ? MAP_DU_K : MAP_DG_K);
                    const uint32_t dst = ring + stage * stage_bytes;
                    const uint32_t bar = map_to_cta(smem_u32(&hd.full[stage]), 0);
                    bad = mbar_wait_conv(smem_u32(&hd.empty[stage]), phase ^ 1u, abort_addr, bad, lead_lane);
                    ++issued_k;
                    if (lead_lane && !bad) {
                        mbar_expect_tx_cluster(bar, tx);
                        tma_load_2d_pair(dst, ma, bar, m_col, w_row);
                        tma_load_2d_pair(dst + G_BOX_BYTES, ma, bar, m_col + 64, w_row);
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            if (x < boxes) tma_load_2d_pair(dst + 2 * G_BOX_BYTES + x * (G_BOX_BYTES / 2), mb, bar, k, x_row + 32 * x);
                        if (leader) *prod_k = issued_k;
                    }
                    if (++stage == n_stages) { stage = 0; phase ^= 1u; }
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
                const uint32_t idesc = G_IDESC_BASE | (is_weights(it) ? G_IDESC_B_MN : 0u) | ((uint32_t)(columns_of(it) >> 3) << 17);
                if (is_weights(it)) {
                    bool first = true;
                    for (int r = s_rep[it.e]; r < s_rep[it.e + 1]; ++r) {
                        const int hi = s_hi[r];
                        for (int k0 = s_lo[r]; k0 < hi; k0 += 64) {
                            const int rows = hi - k0;                  // MMAs of 16 rows each, up to four
                            const uint32_t src = ring + stage * stage_bytes;
                            const uint64_t a_desc = smem_desc_mn(src), b_desc = smem_desc_mn(src + 2 * G_BOX_BYTES);
                            bad = mbar_wait_conv(smem_u32(&hd.full[stage]), phase, abort_addr, bad, lead_lane);
                            tc_fence_after();
                            if (lead_lane && !bad) {
#pragma unroll
                                for (int k = 0; k < 4; ++k)
                                    if (16 * k < rows)
                                        umma_pair_n(d_tmem, a_desc + 128u * k, b_desc + 128u * k, idesc, first && k == 0 ? 0u : 1u);
                                umma_commit_both(smem_u32(&hd.empty[stage]));
                            }
                            first = false;
                            if (++stage == n_stages) { stage = 0; phase ^= 1u; }
                        }
                    }
                } else {
                    const int k_steps = token_steps(it.e);
                    // The ragged end of a segment in a long contraction is held to a full tile's speed, as in the forward's down
                    // projection: pairs that run ahead stop meeting their neighbours' operands in L2.  A call on 4096 tokens, eight
                    // experts top-2, H = 4096, without and with: F = 4096 (128 steps) 1399 and 1402 us, 6144 2090 and 2098, 8192 (256)
                    // 2793 and 2768, 12288 4205 and 4138, 14336 4927 and 4829; 8192 tokens, F = 14336: 9721 and 9208.  Not where a
                    // segment has no full tile: few rows per expert stream weights and lose by waiting.
                    const bool paced = PHASE == 1 && k_steps >= G_PACED_STEPS && it.later && it.valid < G_TILE && hd.tile == G_TILE;
                    const uint32_t c_pace = (uint32_t)clock();
                    for (int kb = 0; kb < k_steps; ++kb) {
                        const uint32_t src = ring + stage * stage_bytes;
                        const uint64_t a_desc = smem_desc_mn(src), b_desc = smem_desc(src + 2 * G_BOX_BYTES);
                        bad = mbar_wait_conv(smem_u32(&hd.full[stage]), phase, abort_addr, bad, lead_lane);
                        tc_fence_after();
                        if (lead_lane && !bad) {
                            if (paced)
                                while ((uint32_t)clock() - c_pace < 512u * (uint32_t)kb) {}
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                umma_pair_n(d_tmem, a_desc + 128u * k, b_desc + 2u * k, idesc, (kb | k) != 0 ? 1u : 0u);
                            umma_commit_both(smem_u32(&hd.empty[stage]));
                        }
                        if (++stage == n_stages) { stage = 0; phase ^= 1u; }
                    }
                }
                if (__any_sync(0xFFFFFFFFu, bad != 0u)) break;
                if (lead_lane) umma_commit_both(smem_u32(&hd.tfull[acc]));
            }
        }
    } else if (warp == 2) {
        // ---- scheduler, leader CTA (see the forward kernel for why claims are held back to G_CLAIM_LEAD k-steps) ----
        if (lane == 0 && leader) {
            const int token_items = s_pre[experts], tile = hd.tile;
            const int total = token_items + (PHASE == 1 ? s_wpre[experts] : 0);
            int e = 0, ord = 0, pub_k = 0;
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
                // a pair's first item is the one of its number, the others come from the counter
                const unsigned int c = i == 0 ? blockIdx.x >> 1 : (gridDim.x >> 1) + atomicAdd(p.counter, 1u);
                const int w = c < (unsigned)total ? (int)c : total;
                const int q = i & (G_SLOTS - 1);
                if (!mbar_wait(smem_u32(&hd.sched_empty[q]), (((uint32_t)i / G_SLOTS) & 1u) ^ 1u, abort_flag)) break;
                int4 item = make_int4(0, 0, 0, 0);
                if (w < total) {
                    if (w < token_items) {
                        while (w >= s_pre[e + 1]) ++e;                 // w only grows
                        const int blocks = PHASE == 0 ? (p.prob[problem_of(e)].F + 255) / 256 : h_blocks;
                        const int nt = (s_pre[e + 1] - s_pre[e]) / blocks, local = w - s_pre[e];
                        const int wb = local / nt;                     // block by block, so that an expert's token tiles share it
                        int nth = local - wb * nt, r = s_rep[e];       // the expert's nth tile: in which segment?
                        for (;; ++r) {
                            const int n = (s_hi[r] - s_lo[r] + tile - 1) / tile;
                            if (nth < n) break;
                            nth -= n;
                        }
                        const int row0 = s_lo[r] + nth * tile;
                        item = make_int4(row0, min(tile, s_hi[r] - row0), e,
                                         wb | ((nth > 0 ? 1 : 0) << 27) | ((PHASE == 0 ? GRAD_ACT : GRAD_DX) << 28));
                        pub_k += token_steps(e);
                    } else if (PHASE == 1) {
                        const int v = w - token_items;
                        while (v >= s_wpre[ord + 1]) ++ord;
                        const int ex = s_order[ord], gateup = h_blocks * (p.prob[problem_of(ex)].F / 128);
                        int local = v - s_wpre[ord];
                        const int kind = local < gateup ? GRAD_GATEUP : GRAD_DOWN;
                        if (kind == GRAD_DOWN) local -= gateup;
                        item = make_int4(local % h_blocks, 1, ex, (local / h_blocks) | (kind << 28));
                        pub_k += s_steps[ex];
                    }
                }
                hd.item[q] = item;
                mbar_arrive(smem_u32(&hd.sched_full[q]));
                // the peer's copy carries its own signal: no release at cluster scope, which would cost as much as a short item
                const uint32_t peer_bar = map_to_cta(smem_u32(&hd.sched_full[q]), 1);
                mbar_expect_tx_cluster(peer_bar, 16);
                st_async_v4(map_to_cta(smem_u32(&hd.item[q]), 1), item, peer_bar);
                if (w >= total) break;
            }
        }
    } else if (warp == 3) {
        // ---- tail warp, both CTAs: zeroes the rows behind a segment's end inside the last MMA of a step ----
        if constexpr (PHASE == 1) {
            int stage = 0;
            uint32_t part_phase = 0, bad = 0;                          // one phase bit per stage
            for (int i = 0; take_item_warp(i, it); ++i) {
                if (!is_weights(it)) {
                    stage = (stage + token_steps(it.e)) % G_STAGES;
                    continue;
                }
                const int boxes = 2 + (columns_of(it) >> 7);           // 64-column boxes of both operands in this CTA
                for (int r = s_rep[it.e]; r < s_rep[it.e + 1]; ++r) {
                    const int hi = s_hi[r];
                    for (int k0 = s_lo[r]; k0 < hi; k0 += 64) {
                        const int valid = hi - k0;
                        if (valid < 64 && (valid & 15) != 0) {
                            bad = mbar_wait_conv(smem_u32(&hd.part[stage]), (part_phase >> stage) & 1u, abort_addr, bad, 1u);
                            part_phase ^= 1u << stage;
                            if (!bad) {
                                // whole rows of 128 bytes (the swizzle stays inside one): eight lanes a row, four rows at a time
                                const int last = (valid + 15) & ~15;
                                uint8_t* const base = smem_raw + (ring - raw) + stage * G_STAGE_BYTES + (lane & 7) * 16;
                                for (int row = valid + (lane >> 3); row < last; row += 4)
                                    for (int b = 0; b < boxes; ++b)
                                        *reinterpret_cast<uint4*>(base + b * G_BOX_BYTES + row * 128) = make_uint4(0u, 0u, 0u, 0u);
                                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");       // before the tensor core reads them
                            }
                            __syncwarp();
                            // The zeros lie in this CTA's own shared memory and are read by its own tensor core: the proxy fence has put
                            // them there, a plain arrive tells the leader (cluster-scope release and acquire cost 1700 cycles each).
                            if (lane == 0 && !bad) mbar_arrive_cluster(map_to_cta(smem_u32(&hd.full[stage]), 0));
                        }
                        if (++stage == G_STAGES) stage = 0;
                    }
                }
                if (__any_sync(0xFFFFFFFFu, bad != 0u)) break;
            }
        }
    } else {
        // ---- epilogue, both CTAs: 32 rows of D per warp (its TMEM quadrant), chunks of 32 columns ----
        const int quad = warp & 3;
        const int c_first = 32 * ((warp - 4) >> 2);
        constexpr int CSTEP = 32 * (G_EPI_WARPS / 4);
        const int d_row = (int)rank * 128 + quad * 32 + lane;          // row of D inside the pair's 256
        for (int i = 0;; ++i) {
            if (!take_item(i, it)) break;
            __syncwarp();
            if (lane == 0) release_item(i);
            if (it.valid == 0) break;
            const GradProblem& pr = p.prob[problem_of(it.e)];
            // D[feature, token] has a feature a lane.  Two lanes share their two features and split the tokens between them - the even
            // lane finishes the even tokens, the odd lane the odd ones, one shuffle per token pair - so that what is read and
            // written in global memory are pairs of features.
            const bool odd = (lane & 1) != 0;
            const int d_pair = d_row & ~1;                             // first of the lane pair's two features
            // GRAD_ACT: the kept values of 32 tokens from c on (code[m]: both features at token c + 2m + odd; ex of lane j: the
            // exponents of token c + j for the warp's two blocks).  The first chunk's are asked for while the products still run, the
            // others a chunk ahead - all before the chunk's arithmetic, among which a load would be waited for at the next use of any other.
            const bool live = it.b * 256 + d_row < pr.F;               // the last block may be half a block (warp-uniform)
            const size_t at0 = (size_t)(it.a + (odd ? 1 : 0)) * pr.F + it.b * 256 + d_pair;
            auto fetch = [&](int c, uint32_t (&code)[16], uint32_t& ex) {
                const uint16_t* const codes = reinterpret_cast<const uint16_t*>(pr.codes) + at0 + (size_t)c * pr.F;
                const int rem = live ? it.valid - c : 0;
#pragma unroll
                for (int m = 0; m < 16; ++m)
                    code[m] = 2 * m + (odd ? 1 : 0) < rem ? __ldg(reinterpret_cast<const uint32_t*>(codes + (size_t)(2 * m) * pr.F)) : 0u;
                if (lane < rem) {
                    const uint16_t* const e0 = pr.exps + (size_t)((it.b * 256 + d_row - lane) / kCheckpointBlock) * pr.rows + it.a + c + lane;
                    ex = (uint32_t)__ldg(e0) | ((uint32_t)__ldg(e0 + pr.rows) << 16);
                }
            };
            uint32_t code[16], ex = 0;
            if constexpr (PHASE == 0) fetch(c_first, code, ex);
            const int acc = i & 1;
            if (!mbar_wait(smem_u32(&hd.tfull[acc]), ((uint32_t)i >> 1) & 1u, abort_flag)) break;
            tc_fence_after();
            const uint32_t taddr = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)(acc * G_TILE);
            const int n = columns_of(it);
            if constexpr (PHASE == 0) {
                if (live) {
                    const uint16_t *dg = pr.dg + at0, *du = pr.du + at0, *act = pr.act + at0;
#pragma unroll 1
                    for (int c = c_first; c < n; c += CSTEP) {
                        uint32_t next[16], next_ex = 0, v[32];
                        fetch(c + CSTEP, next, next_ex);
                        tmem_ld32(taddr + c, v);
                        const int rem = it.valid - c - (odd ? 1 : 0);
                        uint32_t at = 2u * (uint32_t)c * (uint32_t)pr.F;              // bytes from the tile's first row: below 2^32
                        tmem_ld_wait();
#pragma unroll
                        for (int m = 0; m < 16; ++m) {
                            const float other = __uint_as_float(__shfl_xor_sync(0xFFFFFFFFu, odd ? v[2 * m] : v[2 * m + 1], 1));
                            const float mine = __uint_as_float(odd ? v[2 * m + 1] : v[2 * m]);
                            const uint32_t pair = __shfl_sync(0xFFFFFFFFu, ex, 2 * m + (odd ? 1 : 0)) >> (lane & 16);
                            // 2^(e - 127); e = 255 makes it infinity, and a code of zero times that NaN
                            const float sg = __uint_as_float((pair << 23) & 0x7F800000u), su = __uint_as_float((pair << 15) & 0x7F800000u);
                            const uint32_t biased = code[m] ^ 0x80808080u;
                            float dg2[2], du2[2], act2[2];
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                const float da = (k == 0) == odd ? other : mine;
                                const float g = checkpoint_value(biased, 2 * k, sg), u = checkpoint_value(biased, 2 * k + 1, su);
                                const float s = sigmoid(g), gs = g * s;
                                dg2[k] = da * u * fmaf(gs, 1.0f - s, s);
                                du2[k] = da * gs;
                                act2[k] = gs * u;
                            }
                            if (2 * m < rem) {
                                store_u32(offset_by(dg, at), pack_bf16(dg2[0], dg2[1]));
                                store_u32(offset_by(du, at), pack_bf16(du2[0], du2[1]));
                                store_u32(offset_by(act, at), pack_bf16(act2[0], act2[1]));
                            }
                            at += 4u * (uint32_t)pr.F;
                            code[m] = next[m];
                        }
                        ex = next_ex;
                    }
                }
            } else if (it.kind == GRAD_DX) {
                uint16_t* const col = pr.dx + (size_t)(it.a + (odd ? 1 : 0)) * p.H + it.b * 256 + d_pair;
#pragma unroll 1
                for (int c = c_first; c < n; c += CSTEP) {
                    uint32_t v[32];
                    tmem_ld32(taddr + c, v);
                    tmem_ld_wait();
                    uint16_t* ptr = col + (size_t)c * p.H;
                    const int rem = it.valid - c - (odd ? 1 : 0);
#pragma unroll
                    for (int m = 0; m < 16; ++m) {
                        const float other = __uint_as_float(__shfl_xor_sync(0xFFFFFFFFu, odd ? v[2 * m] : v[2 * m + 1], 1));
                        const float mine = __uint_as_float(odd ? v[2 * m + 1] : v[2 * m]);
                        if (2 * m < rem) *reinterpret_cast<uint32_t*>(ptr) = odd ? pack_bf16(other, mine) : pack_bf16(mine, other);
                        ptr += 2 * (size_t)p.H;
                    }
                }
            } else {
                const bool zero = s_steps[it.e] == 0;                  // nothing was accumulated: the gradient is zero
                const int e = problem_of(it.e) ? 0 : it.e;
                const CUtensorMap* mo;
                int row, col;                                          // of this warp's 32 rows in the gradient
                if (it.kind == GRAD_GATEUP) {
                    mo = maps.m[problem_of(it.e)] + (rank ? MAP_OUT_U : MAP_OUT_G);
                    row = e * pr.F + it.b * 128 + quad * 32;
                    col = it.a * 256;
                } else {
                    mo = maps.m[problem_of(it.e)] + MAP_OUT_D;
                    row = e * p.H + it.a * 256 + (int)rank * 128 + quad * 32;
                    col = it.b * 256;
                }
                // row r of the buffer: 64 bytes, its 16-byte pieces in the 64-byte swizzle's order
                uint8_t* const buf = out_buf + (warp - 4) * G_OUT_BYTES;
                uint4* const mine = reinterpret_cast<uint4*>(buf + lane * 64);
#pragma unroll 1
                for (int c = c_first; c < n; c += CSTEP) {
                    uint32_t v[32];
                    if (zero) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = 0u;
                    } else {
                        tmem_ld32(taddr + c, v);
                        tmem_ld_wait();
                    }
                    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");   // the buffer's last store has read it
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        mine[j ^ ((lane >> 1) & 3)] =
                            make_uint4(pack_bf16(__uint_as_float(v[8 * j]), __uint_as_float(v[8 * j + 1])),
                                       pack_bf16(__uint_as_float(v[8 * j + 2]), __uint_as_float(v[8 * j + 3])),
                                       pack_bf16(__uint_as_float(v[8 * j + 4]), __uint_as_float(v[8 * j + 5])),
                                       pack_bf16(__uint_as_float(v[8 * j + 6]), __uint_as_float(v[8 * j + 7])));
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_2d(mo, smem_u32(buf), col + c, row);
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(map_to_cta(smem_u32(&hd.tempty[acc]), 0));
        }
    }

    asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");          // a lane's own stores, none for most
    // ---- teardown, as in the forward kernel: a role that gave up tells the peer CTA; loads and products still under way then
    // get a millisecond to land before the shared and tensor memory they write to is given back ----
    if (*abort_flag) {
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_to_cta(abort_addr, 1u - rank)), "r"(1) : "memory");
        for (const unsigned long long t0 = global_ns(); global_ns() - t0 < 1000000ull;) __nanosleep(1000);
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    if (tid == 0 && *abort_flag) director_set_status(p.status, DIRECTOR_ERR_TIMEOUT);
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
    }
}

template <int PHASE>
int launch_grad(director_ctx* ctx, const char* name, const GradMaps& maps, const GradParams& p, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * ctx->pair_clusters));
    cfg.blockDim = dim3(grad_threads(PHASE));
    cfg.dynamicSmemBytes = (size_t)grad_smem_bytes(PHASE, p.n_rep, p.experts);
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
    return cuda_status(cudaLaunchKernelEx(&cfg, grouped_grad_kernel<PHASE>, maps, p));
}

// bf16 [rows, cols] row-major as the target of TMA stores: boxes of 32 rows x 32 columns, 64-byte swizzle
bool map_out(director_ctx* ctx, CUtensorMap* map, void* base, uint64_t rows, uint64_t cols) {
    const cuuint64_t dims[2] = {cols, rows};
    const cuuint64_t strides[1] = {cols * 2};
    const cuuint32_t box[2] = {32, 32};
    const cuuint32_t estr[2] = {1, 1};
    return reinterpret_cast<EncodeTiledFn>(ctx->encode_tiled)(
               map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// One problem's tensor maps and pointers.  dgu, act: the context's workspace.
bool describe(director_ctx* ctx, const FfnGrad& f, uint64_t n_experts, int F, void* dgu, void* act, CUtensorMap* m, GradProblem& pr) {
    const uint64_t H = (uint64_t)ctx->shape.H, rows = (uint64_t)f.kept.rows;
    uint16_t* const dg = static_cast<uint16_t*>(dgu);
    uint16_t* const du = dg + rows * (uint64_t)F;
    pr = GradProblem{F, (int)rows, f.kept.codes, f.kept.exps, dg, du, static_cast<uint16_t*>(act), static_cast<uint16_t*>(f.dx)};
    return map_2d(ctx, m + MAP_WD, f.w_down, n_experts * H, F, 64) && map_2d(ctx, m + MAP_DY_K, f.dy, rows, H, 32) &&
           map_2d(ctx, m + MAP_WG, f.w_gate, n_experts * F, H, 64) && map_2d(ctx, m + MAP_WU, f.w_up, n_experts * F, H, 64) &&
           map_2d(ctx, m + MAP_DG_K, dg, rows, F, 32) && map_2d(ctx, m + MAP_DU_K, du, rows, F, 32) &&
           map_2d(ctx, m + MAP_X, f.x, rows, H, 64) && map_2d(ctx, m + MAP_DG, dg, rows, F, 64) &&
           map_2d(ctx, m + MAP_DU, du, rows, F, 64) && map_2d(ctx, m + MAP_DY, f.dy, rows, H, 64) &&
           map_2d(ctx, m + MAP_ACT, act, rows, F, 64) && map_out(ctx, m + MAP_OUT_G, f.dw_gate, n_experts * F, H) &&
           map_out(ctx, m + MAP_OUT_U, f.dw_up, n_experts * F, H) && map_out(ctx, m + MAP_OUT_D, f.dw_down, n_experts * H, F);
}

template <int PHASE>
bool grad_opt_in() {
    return cudaFuncSetAttribute(grouped_grad_kernel<PHASE>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                grad_smem_bytes(PHASE, kMaxG + 1, kMaxE + 1)) == cudaSuccess;
}

}  // namespace

int ffn_grad_init(director_ctx*) { return grad_opt_in<0>() && grad_opt_in<1>() ? DIRECTOR_OK : DIRECTOR_ERR_CUDA; }

// routed: the permuted rows.  shared (x != nullptr): the S shared experts as one FFN of width S*F over the batch's own rows.
int launch_expert_ffn_backward(director_ctx* ctx, const int32_t* seg_offsets, const FfnGrad& routed, const FfnGrad& shared,
                               cudaStream_t st) {
    StageScope stage(ctx, st, "stage_expert_ffn_backward");
    const director_shape& s = ctx->shape;
    const int extra = shared.x != nullptr ? 1 : 0;
    GradMaps maps;
    GradParams p{seg_offsets, ctx->d_rep_start, ctx->d_rep_slot, s.E, s.E + extra, ctx->n_replicas + extra, s.H, {}, ctx->d_status,
                 ctx->d_grad_sched, ctx->d_grad_sched + 1};
    if (!describe(ctx, routed, s.E, s.F, ctx->d_dgu, ctx->d_hidden, maps.m[0], p.prob[0])) return DIRECTOR_ERR_CUDA;
    if (extra) {
        if (!describe(ctx, shared, 1, s.S * s.F, ctx->d_dgu_shared, ctx->d_hidden_shared, maps.m[1], p.prob[1])) return DIRECTOR_ERR_CUDA;
    } else {
        memcpy(maps.m[1], maps.m[0], sizeof(maps.m[0]));      // never used
        p.prob[1] = p.prob[0];
    }
    const int rc = launch_grad<0>(ctx, "grouped_grad_act_kernel", maps, p, st);
    if (rc != DIRECTOR_OK) return rc;
    p.counter = ctx->d_grad_sched + 1;
    p.other_counter = ctx->d_grad_sched;
    const int rc2 = launch_grad<1>(ctx, "grouped_grad_weights_kernel", maps, p, st);
    // it would have cleared the first launch's counter, at whose end the next call would find its items claimed
    if (rc2 != DIRECTOR_OK) cudaMemsetAsync(ctx->d_grad_sched, 0, 2 * sizeof(unsigned int), st);
    return rc2;
}

}  // namespace director
