// Fused LM-head variant: the logits z = hidden W^T are formed tile by tile on the tensor cores
// (tcgen05.mma, operands staged in shared memory by TMA, accumulators in tensor memory) and consumed
// by the softmax / loss epilogue straight from tensor memory, so they never reach HBM.
//
// One warp-specialised kernel template serves three contractions (all bf16 x bf16 -> fp32):
//   LSE   z tile = H W^T, epilogue keeps a running (max, sum exp) per token      -> log-sum-exp;
//         for rows that take part in the backward it also stores e = exp(z - rho_t) as bf16, rho_t a
//         per-row reference known before the sweep (or exp(z - tile max) on the fallback path)
//   GH    grad_hidden = f_t (e W)      (A = e K-major, B = W vocabulary-major rows: N-major operand;
//                                       f_t = c_t exp(rho_t - lse_t) applied in the epilogue)
//   GW    grad_W     += e^T (f_t H)    (both operands token-major rows: M-/N-major operands)
// CTA = 192 threads: warp 0 issues TMA loads into a multi-stage ring, warp 1 issues the MMAs (one
// thread), warps 2..5 drain the accumulator with tcgen05.ld (one token row per thread).  The sweeps
// use a double-buffered 128 x 256 fp32 accumulator (all 512 TMEM columns), so the drain of a tile
// overlaps the multiplies of the next; the gradient contractions use both halves as two
// accumulators that share every B slab.  Every mbarrier wait is bounded; a wait that runs out raises
// a CTA-wide abort flag, all roles leave their loops, tensor memory is released and RLF_DEV_TIMEOUT
// is set.  The persistent workers of a launch meet on a global counter before each of their units
// (pacing), which keeps the operand slabs they share in L2.
//
// Forward + backward: the tokens are partitioned into unmasked rows and the others (only the first
// carry gradient).  Unmasked rows go by chunks: LSE with the exponentials stored in a [chunk, V] bf16
// scratch, per-row factors once the rows' log-sum-exp is known, then GH and GW read the scratch:
// three contractions per unmasked row, one per masked row, no recomputation and no pass over the
// scratch in between.  The logits themselves are never stored; the bf16 scratch is (stated in the
// entry point's contract).
//
// The supervised objective (rlf_fused_lmhead_cross_entropy, last section) uses the same template with
// CE set in its gradient contractions: a bf16 grad_W that leaves by TMA stores, rank-one terms added in
// the epilogues, and grad_hidden's long axis cut into pieces when a batch has few rows.
#include <cuda.h>

#include <atomic>
#include <mutex>

#include "common.cuh"

namespace rlf {
namespace lm {

constexpr int BM = 128, BN = 256, BK = 64;
// Single-CTA form: each CTA multiplies a 128 x 256 tile (A 16 KB + B 32 KB per stage, 4 stages).
// Pair form (cta_group::2): two CTAs of a cluster multiply a 256 x 256 tile; each stages its own 128
// rows of A and HALF of B (16 KB + 16 KB per stage, 6 stages), the leader CTA issues the MMAs, and
// each CTA's tensor memory receives its own 128 rows of the accumulator.  Per flop the pair form
// moves two thirds of the shared-memory bytes of the single form.
constexpr int kABytes = BM * BK * 2;
constexpr int kDrainPitch = 36;              // floats per row of a drain staging tile (32 + 4 of padding)
// Two-accumulator pair form (ACC2, the two gradient contractions): a pair works on TWO 256-row tiles
// against the same 256 columns, each CTA staging two A tiles beside its half of B (48 KB per stage, 4
// stages), so every B slab that crosses L2 -> shared memory is used for 512 rows: three quarters of
// the shared-memory fill bytes per flop of the plain pair form, and half the passes over the B
// matrix.  The two accumulators take all 512 TMEM columns, so the drain of a unit does not overlap the
// next unit's multiplies; with K running over the whole vocabulary or a whole chunk of tokens the
// drain is a per cent or two of a unit.
// The cross-entropy form's gradient contractions (CE) keep two bf16 output tiles of 32 rows x 64 columns per drain warp
// instead of the fp32 staging tile: grad_W leaves them by TMA stores.
template <bool PAIR, bool ACC2 = false, bool CE = false> struct Cfg {
    static_assert(PAIR || !ACC2, "two accumulators per CTA exist in pair form only");
    static constexpr int kAcc = ACC2 ? 2 : 1;
    static constexpr int kStages = ACC2 ? 4 : (PAIR ? 6 : 4);
    static constexpr int kBRows = PAIR ? BN / 2 : BN;
    static constexpr int kBBytes = kBRows * BK * 2;
    static constexpr int kStageBytes = kAcc * kABytes + kBBytes;
    // + alignment slack, the barriers, and (two-accumulator form) a 32 x 32 fp32 staging tile per drain warp
    static constexpr int kDrainBytes = CE ? 4 * 2 * 4096 : ACC2 ? 4 * 32 * kDrainPitch * 4 : 0;
    static constexpr int kSmemBytes = kStages * kStageBytes + 1024 + 256 + kDrainBytes;
};
constexpr int kMaxStages = 6;
constexpr int kThreads = 192;
constexpr int kTmemCols = 512;
constexpr int kSlabBytes = 64 * BK * 2;      // one 64-wide slab of an MN-major operand: 64 k-rows of 128 B

enum Mode { kLse = 0, kGradHidden = 2, kGradW = 3 };

// The [rows, V] scratch that carries a chunk's exponentials, then its dZ, is stored in blocks of
// 128 token rows x 64 vocabulary columns (16 KB, rows of 128 bytes), blocks of one token tile side by
// side: element (row, col) sits at ((row / 128 * nc + col / 64) * 128 + row % 128) * 64 + col % 64,
// nc = 4 x the number of 256-column tiles.  Every operand box the two gradient contractions fetch
// (128 or 64 rows of 128 bytes) is then one contiguous piece of memory, and so is what a warp of the
// sweep's epilogue stores; with plain rows of 2 V bytes each of those touched 64 - 128 DRAM pages for
// 128 bytes apiece.
constexpr int kDzBlockRows = 128, kDzBlockCols = 64;
__host__ __device__ __forceinline__ long long dz_offset(long long row, int col, int nc) {
    return (((row >> 7) * nc + (col >> 6)) * kDzBlockRows + (row & 127)) * kDzBlockCols + (col & 63);
}

struct GemmParams {
    int mode;
    int M, N;                 // extent of the output tile grid in rows / columns (valid elements)
    int m_tiles, n_tiles, k_slabs;
    int nsplit, n_tiles_per_split;
    int m_block;              // kLse: row units per scheduling block
    float2* part;             // kLse: [M][nsplit] (max, sum exp)
    float* part_u;            // kLse (optional): [M][nsplit] sum of 2^x x, x the base-2 exponent against that max
    __nv_bfloat16* dz;        // kLse (optional) out, blocked scratch (see dz_offset): exp(z - tile max) as bf16
    float* tmax;              // kLse with dz: [M][n_tiles] the tile maxima those exponentials refer to
    int dz_nc;                // 64-column blocks per token tile of the blocked scratch; also set for the
                              // gradient contractions, whose A operand is that scratch
    __nv_bfloat16* out_bf16;  // kGradHidden out [M][out_stride]
    float* out_f32;           // kGradW out [M][out_stride]
    long long out_stride;
    int accumulate;
    int32_t* dev_status;
    // Token extent known only on the device (launches over the gathered unmasked / masked rows):
    // when live_count is set, the token extent of this launch is
    // clamp(*live_count - live_off, 0, M or K as built on the host).
    const int* live_count;
    int live_off;
    const int32_t* row_index; // kGradHidden: output row of compact row r is row_index[live_off + r]
    const float* ref;         // kLse with dz (optional): per-row reference of the stored exponentials (see below)
    // kLse (optional): {., target column} of compact row r.  Its logit goes to target_logit[r] and stays out of the row's sums (and,
    // as a zero, of the scratch)
    const int2* target;
    float* target_logit;
    const float* row_scale;   // kGradHidden (optional): fp32 factor of compact row r applied to its output row
    const int* run_flag;      // optional: the launch does nothing unless *run_flag == run_want
    int run_want;
    // Pacing (optional): a counter, zero at launch, on which the load-issuing threads of all workers meet
    // before each of their units but the first.  Workers that share operand slabs through L2 then
    // request them within a short time of each other; left alone they drift apart over a launch until
    // each fetches its slabs from HBM on its own.  Waits are bounded and only delay loads: a worker
    // that gives up runs on unpaced.
    int* pace;
    int pace_is_zero;         // the counter has been zeroed already (else the launch does it)
    // Sweep over device-counted rows (optional): with at most auto_units row units the number of vocabulary splits is chosen
    // on the device (auto_split); with more it is fixed_split, and only block_workers workers take part (the host's L2
    // blocking).  nsplit is then the most splits there may be, and the partials' stride.
    int auto_units, fixed_split, block_workers;
    // Cross-entropy form (CE, the gradient contractions).  Label smoothing adds a rank-one term to either gradient:
    const float* col_vec;     // kGradHidden (optional): out += row_add[r] * col_vec[col];  kGradW (optional): out += col_vec[col]
    const float* row_add;     // kGradHidden with col_vec: factor of compact row r
    int store_w16;            // kGradW: the result goes to map_c's matrix as bf16 instead of to out_f32 (last chunk of a call)
    const float* add_f32;     // kGradW with store_w16 (optional): earlier chunks' fp32 sum, [M][out_stride], added before rounding
    // kGradHidden: with few row units the vocabulary (the long axis) is cut into up to k_split_max pieces (hidden_splits), whose
    // raw sums go to k_part, [piece][live rows of the chunk][out_stride] fp32, for ce_join_hidden_kernel
    int k_split_max;
    float* k_part;
    long long k_part_floats;  // what k_part holds: there are never more pieces than fit
};

// ---- PTX wrappers ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
constexpr int kWaitPolls = 1 << 22;
constexpr int kPacePolls = 1 << 14;          // a pacing wait gives up after about 10 ms and is not taken again
// wait (bounded) until the pacing counter has reached `want`; `seen` is a value read earlier
__device__ __forceinline__ void pace_settle(const int* counter, int seen, long long want, bool& keep_waiting) {
    int polls = 0;
    while ((long long)seen < want) {
        if (++polls > kPacePolls) { keep_waiting = false; return; }
        __nanosleep(64);
        asm volatile("ld.relaxed.gpu.global.s32 %0, [%1];" : "=r"(seen) : "l"(counter) : "memory");
    }
}
// bounded wait; on failure (or if another role already gave up) returns false
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
    for (int i = 0; i < kWaitPolls; ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((i & 1023) == 1023 && *abort_flag) return false;
    }
    *abort_flag = 1;
    return false;
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 :: "r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
}
__device__ __forceinline__ void tc_mma(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 :: "r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(acc) : "memory");
}
// cta_group::2 forms: the MMA spans both CTAs of the pair; its commit arrives on the same barrier
// offset in both CTAs; TMA loads of either CTA credit a barrier in the leader CTA.
__device__ __forceinline__ void tc_mma2(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 :: "r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(acc) : "memory");
}
// The multicast here is that of a BARRIER SIGNAL: the commit arrives on the mbarrier at the same offset in
// both CTAs of the pair (mask 0b11).  No load in this file is multicast -- every cp.async.bulk.tensor
// below is a plain per-CTA copy -- and every tensor map covers this GPU's own memory.
__device__ __forceinline__ void tc_commit2(uint32_t bar) {
    const unsigned short both = 3;
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 :: "r"(bar), "h"(both) : "memory");
}
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* map, uint32_t leader_bar, int x, int y) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 :: "r"(dst), "l"(map), "r"(leader_bar), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ uint32_t map_to_cta(uint32_t local_addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(local_addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" :: "r"(cluster_addr) : "memory");
}
__device__ __forceinline__ uint32_t pair_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void pair_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// 32 consecutive fp32 columns of this thread's TMEM lane
__device__ __forceinline__ void tc_ld32(uint32_t taddr, uint32_t (&v)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
                   "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
                   "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
                   "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
                 : "r"(taddr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// the same load without its wait, and the wait: the registers pass through the wait as in/out operands
// so that no use of them can be scheduled ahead of it
__device__ __forceinline__ void tc_ld32_issue(uint32_t taddr, uint32_t (&v)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
                   "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
                   "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
                   "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tc_ld_wait(uint32_t (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                   "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]),
                   "+r"(v[16]), "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]),
                   "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])
                 :: "memory");
}

// Shared-memory operand descriptor, 128-byte swizzle, descriptor version 1.
//   K-major tile  (rows of 64 bf16 = 128 B, 8-row groups 1024 B apart): LBO 1, SBO 1024 B.
//   MN-major tile (64-wide slabs, each 64 k-rows of 128 B): LBO = slab pitch 8192 B, SBO 1024 B.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, bool mn_major) {
    const uint64_t lbo = mn_major ? (uint64_t)(kSlabBytes >> 4) : 1ull;
    return (uint64_t)((addr & 0x3FFFF) >> 4) | (lbo << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) |
           (2ull << 61);
}
// Instruction descriptor: D fp32, A and B bf16, M = 128, N = 256, majorness per operand.
__host__ __device__ constexpr uint32_t instr_desc(bool a_mn, bool b_mn, int m) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) |
           ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

struct SmemCtl {
    unsigned long long full[kMaxStages];
    unsigned long long empty[kMaxStages];
    unsigned long long tmem_full[2];
    unsigned long long tmem_empty[2];
    uint32_t tmem_base;
    volatile int abort_flag;
};

static_assert(sizeof(SmemCtl) <= 256, "the barriers share a 256-byte slot behind the stage ring");

// Vocabulary splits of a sweep whose token tiles all stay in L2: the persistent workers take the m_units x s units
// round-robin, so the launch lasts about ceil(m_units s / workers) rounds of ceil(n_tiles / s) tiles (and a little per unit); the
// best such s.  (593 column tiles, 74 pairs: one row unit 74 splits of 8 or 9 tiles instead of 60 of 9 or 10; six row units of
// 125 tiles 12 splits, one round of 11, instead of 16, two rounds of 8.)  Every lane of a full warp calls it.
__device__ __forceinline__ int auto_split(int m_units, int n_tiles, int workers, int most) {
    const int lane = threadIdx.x & 31;
    unsigned best = 0xffffffffu;
    for (int s = lane + 1; s <= most && s <= n_tiles; s += 32) {
        const unsigned rounds = (unsigned)((m_units * s + workers - 1) / workers), tiles = (unsigned)((n_tiles + s - 1) / s);
        const unsigned cost = (rounds * (8 * tiles + 1)) << 7 | (unsigned)s;
        best = best < cost ? best : cost;
    }
    return (int)(__reduce_min_sync(0xffffffffu, best) & 127u);
}
// Pieces that the vocabulary is cut into in grad_hidden, `units` output tiles of k_slabs each on the workers: rounds of a
// piece's slabs (six more for its drain), and a quarter of a slab's time per unit and piece to write and join its raw sums.
// (10 row units x 16 column tiles on 74 pairs: three rounds uncut, 2.33 in three pieces.)
constexpr int kSlabsPerPiece = 16;          // a piece holds at least so many k-slabs
__host__ __device__ constexpr unsigned hidden_cost(int units, int k_slabs, int workers, int k) {
    const unsigned rounds = (unsigned)((units * k + workers - 1) / workers), slabs = (unsigned)((k_slabs + k - 1) / k);
    return (rounds * (slabs + 6) + (k > 1 ? (unsigned)(units * k + 3) / 4 : 0)) << 7 | (unsigned)k;
}
// room: floats that the pieces may take, `rows` rows of D each.  Every lane of a full warp calls it.
__device__ __forceinline__ int hidden_splits(int units, int k_slabs, int workers, int most, long long room, int rows, int D) {
    const int lane = threadIdx.x & 31;
    const long long fit = room / ((long long)max(rows, 1) * D);
    if (fit < most) most = fit < 1 ? 1 : (int)fit;
    unsigned best = 0xffffffffu;
    for (int k = lane + 1; k <= most && (k == 1 || k_slabs >= kSlabsPerPiece * k); k += 32) best = min(best, hidden_cost(units, k_slabs, workers, k));
    return (int)(__reduce_min_sync(0xffffffffu, best) & 127u);
}

// ---- the kernel -----------------------------------------------------------------------------
template <bool PAIR, bool ACC2, bool CE = false>
__global__ void __launch_bounds__(kThreads, 1)
umma_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                 const __grid_constant__ CUtensorMap map_c, const GemmParams p) {
    using C = Cfg<PAIR, ACC2, CE>;
    constexpr int NACC = C::kAcc;
    extern __shared__ unsigned char smem_raw[];
    // a launch that is conditional on a device-side flag (uniform over the grid): leave before
    // anything is set up
    if (p.run_flag && *p.run_flag != p.run_want) return;
    // operand stages must sit on 1024-byte boundaries (swizzle atom)
    const uint32_t raw = smem_addr(smem_raw);
    const uint32_t tiles = (raw + 1023u) & ~1023u;
    float* drain_stage = reinterpret_cast<float*>(smem_raw + (tiles - raw) + C::kStages * C::kStageBytes);   // 1 KB aligned
    SmemCtl* ctl = reinterpret_cast<SmemCtl*>(smem_raw + (tiles - raw) + C::kStages * C::kStageBytes + C::kDrainBytes);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool a_mn = p.mode == kGradW;
    const bool b_mn = p.mode == kGradHidden || p.mode == kGradW;
    const bool sweep = p.mode == kLse;                      // a unit sweeps several vocabulary tiles
    // in pair form the scheduling unit covers two token tiles: this CTA takes tile 2 * mp + rank
    const int rank = PAIR ? (int)pair_rank() : 0;
    int M = p.M, m_tiles = p.m_tiles, k_slabs = p.k_slabs;
    if (p.live_count) {
        const int host_extent = p.mode == kGradW ? p.k_slabs * BK : p.M;
        const int live = max(0, min(*p.live_count - p.live_off, host_extent));
        if (p.mode == kGradW) k_slabs = (live + BK - 1) / BK;
        else { M = live; m_tiles = (live + BM - 1) / BM; }
    }
    // no tokens under a grad_W tile: nothing to add; without accumulate the tile is still written (zeros)
    const bool no_k = k_slabs == 0;
    // token (or vocabulary) tiles per scheduling unit: 1, 2 in pair form, 4 with two accumulators; this
    // CTA's tile for accumulator a of unit m is kTilesPerUnit * m + 2 * a + rank
    constexpr int kTilesPerUnit = (PAIR ? 2 : 1) * NACC;
    const int m_units = (m_tiles + kTilesPerUnit - 1) / kTilesPerUnit;
    const int worker = PAIR ? blockIdx.x >> 1 : blockIdx.x;
    int workers = PAIR ? gridDim.x >> 1 : gridDim.x;
    int nsplit = p.nsplit, m_block = p.m_block;
    if (sweep && p.auto_units > 0) {
        if (m_units <= p.auto_units) {
            nsplit = auto_split(m_units, p.n_tiles, workers, p.nsplit);
            m_block = p.auto_units;
        } else {
            nsplit = p.fixed_split;
            workers = min(workers, p.block_workers);
        }
    }
    const int k_split = (CE && p.mode == kGradHidden)
                            ? hidden_splits(m_units * p.n_tiles, k_slabs, workers, p.k_split_max, p.k_part_floats, M, (int)p.out_stride) : 1;
    const int all_units = (no_k && p.accumulate) ? 0 : sweep ? m_units * nsplit : m_units * p.n_tiles * k_split;
    const int units = worker < workers ? all_units : 0;      // (a worker beyond those that take part has nothing to do)

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::kStages; ++s) {
            mbar_init(smem_addr(&ctl->full[s]), 1);
            mbar_init(smem_addr(&ctl->empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_addr(&ctl->tmem_full[b]), 1);
            mbar_init(smem_addr(&ctl->tmem_empty[b]), PAIR ? 8 : 4);
        }
        ctl->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        if (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                         :: "r"(smem_addr(&ctl->tmem_base)), "r"((uint32_t)kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                         :: "r"(smem_addr(&ctl->tmem_base)), "r"((uint32_t)kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) pair_sync();        // both CTAs' barriers exist before either signals the other
    tc_fence_after();
    const uint32_t tmem_base = ctl->tmem_base;

    // unit -> (m unit, first n tile, one-past-last n tile)
    const int split_base = sweep ? p.n_tiles / nsplit : 0, split_rem = sweep ? p.n_tiles % nsplit : 0;
    auto unit_range = [&](int u, int& m, int& n0, int& n1) {
        if (sweep) {
            // blocks of m_block row units; inside a block, units run over its row units first, then
            // over the splits: the CTAs running at one time share both the rows of the head they
            // sweep and a set of token tiles small enough to stay in L2
            const int per_block = m_block * nsplit;
            const int blk = u / per_block, within = u - blk * per_block;
            const int rows_here = min(m_block, m_units - blk * m_block);
            const int sp = within / rows_here;
            m = blk * m_block + (within - sp * rows_here);
            // column tiles dealt evenly: the first split_rem splits hold one tile more than the others
            n0 = sp * split_base + min(sp, split_rem);
            n1 = n0 + split_base + (sp < split_rem ? 1 : 0);
        } else {
            // column tiles fastest: the CTAs running at the same time share their A slabs (the dZ
            // rows or columns) in L2 instead of each streaming the whole scratch from HBM
            n0 = u % p.n_tiles;
            m = u / p.n_tiles;
            if (CE) m %= m_units;            // (pieces of the long axis slowest)
            n1 = n0 + 1;
        }
    };
    // unit -> its k-slabs
    auto unit_k = [&](int u, int& k0, int& k1) {
        k0 = 0;
        k1 = k_slabs;
        if (CE && k_split > 1) {
            const int piece = u / (m_units * p.n_tiles);
            k0 = (int)((long long)k_slabs * piece / k_split);
            k1 = (int)((long long)k_slabs * (piece + 1) / k_split);
        }
    };

    if (warp == 0) {
        // ---------------- TMA producer (one per CTA) ----------------
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            long long pace_due = 0;       // arrivals expected on the counter before this worker goes on
            bool pace_wait = p.pace != nullptr, pace_pending = false;
            int pace_seen = 0;
            int iter = 0;
            for (int u = worker; u < units && ok && !no_k; u += workers, ++iter) {
                int m, n0, n1;
                unit_range(u, m, n0, n1);
                const int with_me = min(workers, all_units - iter * workers);     // workers that have a unit number `iter`
                int k0, k1;
                unit_k(u, k0, k1);
                long long pos = 0;
                for (int n = n0; n < n1 && ok; ++n) {
                    const int b_row0 = n * BN + rank * C::kBRows;      // this CTA's rows of the B tile
                    for (int kb = k0; kb < k1; ++kb, ++pos) {
                        // the meeting point before a unit: announce the arrival and read the counter; the value
                        // is looked at two k-slabs later, so its round trip to L2 overlaps the issue of those
                        // slabs' loads instead of draining the ring
                        if (p.pace && iter > 0 && pos == 0) {
                            pace_due += with_me;
                            if (rank == 0) asm volatile("red.relaxed.gpu.global.add.s32 [%0], 1;" :: "l"(p.pace) : "memory");
                            if (pace_wait) {
                                asm volatile("ld.relaxed.gpu.global.s32 %0, [%1];" : "=r"(pace_seen) : "l"(p.pace) : "memory");
                                pace_pending = true;
                            }
                        }
                        if (pace_pending && pos >= 2) {
                            pace_settle(p.pace, pace_seen, pace_due, pace_wait);
                            pace_pending = false;
                        }
                        if (!mbar_wait(smem_addr(&ctl->empty[stage]), phase ^ 1u, &ctl->abort_flag)) { ok = false; break; }
                        const uint32_t own_bar = smem_addr(&ctl->full[stage]);
                        const uint32_t bar = PAIR ? map_to_cta(own_bar, 0) : own_bar;   // the leader's barrier
                        const uint32_t sa0 = tiles + stage * C::kStageBytes;
                        const uint32_t sb = sa0 + NACC * kABytes;
                        if (!PAIR) mbar_expect_tx(own_bar, C::kStageBytes);
                        else if (rank == 0) mbar_expect_tx(own_bar, 2 * C::kStageBytes);
                        auto load = [&](uint32_t dst, const CUtensorMap* map, int x, int y) {
                            if (PAIR) tma_load_2d_pair(dst, map, bar, x, y);
                            else tma_load_2d(dst, map, bar, x, y);
                        };
#pragma unroll
                        for (int a = 0; a < NACC; ++a) {
                            const int my_m = kTilesPerUnit * m + 2 * a + rank;
                            const uint32_t sa = sa0 + a * kABytes;
                            if (p.mode == kGradHidden) {
                                // dZ block (token tile my_m, vocabulary block kb): 128 rows of 128 bytes
                                load(sa, &map_a, 0, (my_m * p.dz_nc + kb) * kDzBlockRows);
                            } else if (p.mode == kGradW) {
                                // dZ^T: vocabulary blocks 2 my_m + j, the 64 token rows of k-slab kb
                                for (int j = 0; j < BM / 64; ++j)
                                    load(sa + j * kSlabBytes, &map_a, 0,
                                         ((kb >> 1) * p.dz_nc + (my_m * 2 + j)) * kDzBlockRows + (kb & 1) * 64);
                            } else {
                                load(sa, &map_a, kb * BK, my_m * BM);
                            }
                        }
                        if (!b_mn) {
                            load(sb, &map_b, kb * BK, b_row0);
                        } else {
                            for (int j = 0; j < C::kBRows / 64; ++j) load(sb + j * kSlabBytes, &map_b, b_row0 + j * 64, kb * BK);
                        }
                        if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
                    }
                }
            }
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer (in pair form: the leader CTA only) ----------------
        if (lane == 0 && rank == 0) {
            const uint32_t idesc = instr_desc(a_mn, b_mn, PAIR ? 2 * BM : BM);
            const uint32_t a_kstep = a_mn ? (16 * 128) >> 4 : 32 >> 4;   // 16 k per instruction, in 16-byte units
            const uint32_t b_kstep = b_mn ? (16 * 128) >> 4 : 32 >> 4;
            int stage = 0;
            uint32_t phase = 0;
            int buf = 0;
            uint32_t tphase[2] = {0, 0};
            bool ok = true;
            for (int u = worker; u < units && ok && !no_k; u += workers) {
                int m, n0, n1, k0, k1;
                unit_range(u, m, n0, n1);
                unit_k(u, k0, k1);
                for (int n = n0; n < n1 && ok; ++n) {
                    if (!mbar_wait(smem_addr(&ctl->tmem_empty[buf]), tphase[buf] ^ 1u, &ctl->abort_flag)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t d_tmem = tmem_base + (uint32_t)buf * BN;
                    for (int kb = k0; kb < k1; ++kb) {
                        if (!mbar_wait(smem_addr(&ctl->full[stage]), phase, &ctl->abort_flag)) { ok = false; break; }
                        tc_fence_after();
                        const uint32_t sa = tiles + stage * C::kStageBytes;
                        const uint64_t adesc = smem_desc(sa, a_mn);
                        const uint64_t bdesc = smem_desc(sa + NACC * kABytes, b_mn);
#pragma unroll
                        for (int k = 0; k < BK / 16; ++k) {
                            if (ACC2) {
                                // accumulator a (TMEM columns a * 256 ..) takes A tile a; both share the B slab
#pragma unroll
                                for (int a = 0; a < NACC; ++a)
                                    tc_mma2(tmem_base + (uint32_t)(a * BN),
                                            adesc + (uint64_t)(a * (kABytes >> 4)) + (uint64_t)(k * a_kstep),
                                            bdesc + (uint64_t)(k * b_kstep), idesc, ((kb - k0) | k) ? 1u : 0u);
                            } else if (PAIR) tc_mma2(d_tmem, adesc + (uint64_t)(k * a_kstep), bdesc + (uint64_t)(k * b_kstep), idesc,
                                                     ((kb - k0) | k) ? 1u : 0u);
                            else tc_mma(d_tmem, adesc + (uint64_t)(k * a_kstep), bdesc + (uint64_t)(k * b_kstep), idesc,
                                        ((kb - k0) | k) ? 1u : 0u);
                        }
                        // frees the stage (in both CTAs) when these MMAs retire
                        if (PAIR) tc_commit2(smem_addr(&ctl->empty[stage]));
                        else tc_commit(smem_addr(&ctl->empty[stage]));
                        if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
                    }
                    if (!ok) break;
                    // accumulator complete (in both CTAs)
                    if (PAIR) tc_commit2(smem_addr(&ctl->tmem_full[buf]));
                    else tc_commit(smem_addr(&ctl->tmem_full[buf]));
                    tphase[buf] ^= 1u;
                    if (!ACC2) buf ^= 1;              // with two accumulators per unit there is one "buffer": both
                }
            }
        }
    } else {
        // ---------------- epilogue: warps 2..5, one accumulator row per thread ----------------
        const int quarter = warp & 3;                    // TMEM lane quarter this warp may read
        const int row_in_tile = quarter * 32 + lane;
        int buf = 0;
        int out_tile = 0;                                // CE: which of this warp's two output tiles is filled next
        (void)out_tile;
        uint32_t tphase[2] = {0, 0};
        bool ok = true;
        for (int u = worker; u < units && ok; u += workers) {
            int m, n0, n1;
            unit_range(u, m, n0, n1);
            const int row = (kTilesPerUnit * m + rank) * BM + row_in_tile;     // accumulator 0's row
            const bool row_ok = row < M;
            float run_m = -INFINITY, run_s = 0.0f;       // kLse
            float run_u = 0.0f;                          // kLse with entropy: sum of 2^x x against run_m
            const int piece = (CE && k_split > 1) ? u / (m_units * p.n_tiles) : 0;
            (void)piece;
            const int target = (!CE && sweep && p.target && row_ok) ? p.target[row].y : -1;
            for (int n = n0; n < n1 && ok; ++n) {
                if (!no_k) {
                    // one lane polls for the warp (128 polling threads would only burn issue slots and
                    // power while the tile is being multiplied); the shuffle hands its result to the others
                    int got = 0;
                    if (lane == 0) got = mbar_wait(smem_addr(&ctl->tmem_full[buf]), tphase[buf], &ctl->abort_flag) ? 1 : 0;
                    got = __shfl_sync(0xffffffffu, got, 0);
                    if (!got) { ok = false; break; }
                    tc_fence_after();
                }
                const uint32_t t_row = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)buf * BN;
                const int col0 = n * BN;
                // takes the target's logit out of the 32 columns from cb on (a vote per tile, and per 32 columns of a tile that holds
                // a target of the warp's rows, keeps the selection out of the others)
                const bool target_here = !CE && sweep && __any_sync(0xffffffffu, (unsigned)(target - col0) < (unsigned)BN);
                auto take_target = [&](int cb, uint32_t (&v)[32]) {
                    const int at = target - cb;
                    if (!target_here || !__any_sync(0xffffffffu, (unsigned)at < 32u)) return;
                    uint32_t z = 0u;
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        z = i == at ? v[i] : z;
                        v[i] = i == at ? 0xff800000u : v[i];
                    }
                    if ((unsigned)at < 32u) p.target_logit[row] = __uint_as_float(z);
                };
                if (p.mode == kLse && p.dz && p.ref) {
                    // Forward sweep that keeps the tile for the backward, exponentials taken against a
                    // reference rho known BEFORE the sweep (one per row): e = exp(z - rho) is summed for
                    // the log-sum-exp and stored as bf16 in one pass over the accumulator.  bf16 has
                    // fp32's exponent range, so any rho within some tens of the row's log-sum-exp
                    // keeps every entry that matters a normal number at full relative precision, and
                    // dZ = (c_t exp(rho - lse)) e needs only a per-row factor afterwards.  A row whose
                    // reference turns out too far off shows in its sum (inf, or far from one) and
                    // sends its chunk through the per-tile-maximum path instead.
                    const float off = row_ok ? -p.ref[row] * kLog2e : 0.0f;
                    float ts0 = 0.0f, ts1 = 0.0f;
#pragma unroll 1
                    for (int c = 0; c < BN / 32; ++c) {
                        const int cb = col0 + c * 32;
                        const int nvalid = max(0, min(32, p.N - cb));
                        uint32_t o[16];
                        if (nvalid > 0) {                  // warp-uniform: the tensor-memory load is a warp-wide instruction
                            uint32_t v[32];
                            tc_ld32(t_row + (uint32_t)(c * 32), v);
                            take_target(cb, v);
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                float e0 = ex2_approx(fmaf(__uint_as_float(v[2 * i]), kLog2e, off));
                                float e1 = ex2_approx(fmaf(__uint_as_float(v[2 * i + 1]), kLog2e, off));
                                if (2 * i >= nvalid) e0 = 0.0f;
                                if (2 * i + 1 >= nvalid) e1 = 0.0f;
                                ts0 += e0;
                                ts1 += e1;
                                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[i]) : "f"(e1), "f"(e0));
                            }
                        }
                        if (nvalid <= 0 || !row_ok) {
                            // columns past the vocabulary and rows past the live extent (up to the end of
                            // this pair of token tiles) read as zeros in the gradient contractions
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = 0u;
                        }
                        uint4* d4 = reinterpret_cast<uint4*>(p.dz + dz_offset(row, cb, p.dz_nc));
                        d4[0] = make_uint4(o[0], o[1], o[2], o[3]);
                        d4[1] = make_uint4(o[4], o[5], o[6], o[7]);
                        d4[2] = make_uint4(o[8], o[9], o[10], o[11]);
                        d4[3] = make_uint4(o[12], o[13], o[14], o[15]);
                    }
                    run_s += ts0 + ts1;
                    if (row_ok) run_m = p.ref[row];
                } else if (p.mode == kLse && p.dz) {
                    // Forward sweep that keeps the tile for the backward.  Pass 1 over the accumulator:
                    // the row's maximum inside this tile; pass 2: e = exp(z - that maximum), summed for
                    // the log-sum-exp and stored as bf16 (e <= 1: no overflow whatever the logits are;
                    // the relative rounding error is that of a bf16 gradient entry).
                    float tm = -INFINITY;
#pragma unroll 1
                    for (int c = 0; c < BN / 32; ++c) {
                        const int cb = col0 + c * 32;
                        if (cb >= p.N) break;
                        uint32_t v[32];
                        tc_ld32(t_row + (uint32_t)(c * 32), v);
                        take_target(cb, v);
                        const int nvalid = min(32, p.N - cb);
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (i < nvalid) tm = fmaxf(tm, __uint_as_float(v[i]));
                    }
                    const float tms = (tm == -INFINITY) ? 0.0f : tm;
                    if (tm > run_m) {
                        run_s *= ex2_approx((run_m - tm) * kLog2e);
                        run_m = tm;
                    }
                    const float off = -tms * kLog2e;
                    float ts0 = 0.0f, ts1 = 0.0f;
#pragma unroll 1
                    for (int c = 0; c < BN / 32; ++c) {
                        // every column block of the tile is written: the scratch covers whole tiles and
                        // the columns past the vocabulary must read as zeros (warp-uniform conditions)
                        const int cb = col0 + c * 32;
                        const int nvalid = max(0, min(32, p.N - cb));
                        uint32_t o[16];
                        if (nvalid > 0) {
                            uint32_t v[32];
                            tc_ld32(t_row + (uint32_t)(c * 32), v);
                            take_target(cb, v);
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                float e0 = ex2_approx(fmaf(__uint_as_float(v[2 * i]), kLog2e, off));
                                float e1 = ex2_approx(fmaf(__uint_as_float(v[2 * i + 1]), kLog2e, off));
                                if (2 * i >= nvalid) e0 = 0.0f;
                                if (2 * i + 1 >= nvalid) e1 = 0.0f;
                                ts0 += e0;
                                ts1 += e1;
                                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[i]) : "f"(e1), "f"(e0));
                            }
                        } else {
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = 0u;
                        }
                        if (row_ok) {
                            uint4* d4 = reinterpret_cast<uint4*>(p.dz + dz_offset(row, cb, p.dz_nc));
                            d4[0] = make_uint4(o[0], o[1], o[2], o[3]);
                            d4[1] = make_uint4(o[4], o[5], o[6], o[7]);
                            d4[2] = make_uint4(o[8], o[9], o[10], o[11]);
                            d4[3] = make_uint4(o[12], o[13], o[14], o[15]);
                        }
                    }
                    // (a tile of -inf has the sum 0; one of -inf and NaN has the same maximum and the sum NaN, which must stay)
                    run_s += tm == -INFINITY ? ts0 + ts1 : (ts0 + ts1) * ex2_approx((tm - run_m) * kLog2e);
                    if (row_ok) p.tmax[(long long)row * p.n_tiles + n] = tms;
                } else {
                // 32-column chunks of the accumulator(s), software-pipelined: the tensor-memory load of
                // chunk ac + 1 is in flight while chunk ac is consumed (with two accumulators the drain is
                // not hidden behind the next unit's multiplies, so its latency chain matters)
                // (CE, grad_W) one thread's 32 columns of its row: the smoothing term is added; then, for a bf16 result, the
                // earlier chunks' sum, and the piece goes into this warp's 32 x 64 output tile (128-byte rows, swizzled
                // like every TMA box here), which lane 0 stores once its second half is in.  nvalid is 32 (the hidden size
                // is a multiple of 64).
                auto drain_w = [&](int row_r, int cb, uint32_t (&v)[32]) {
                    if (p.col_vec) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float4 g = reinterpret_cast<const float4*>(p.col_vec + cb)[i];
                            v[4 * i] = __float_as_uint(__uint_as_float(v[4 * i]) + g.x);
                            v[4 * i + 1] = __float_as_uint(__uint_as_float(v[4 * i + 1]) + g.y);
                            v[4 * i + 2] = __float_as_uint(__uint_as_float(v[4 * i + 2]) + g.z);
                            v[4 * i + 3] = __float_as_uint(__uint_as_float(v[4 * i + 3]) + g.w);
                        }
                    }
                    if (!p.store_w16) {
                        if (row_r < M) {
                            float4* d4 = reinterpret_cast<float4*>(p.out_f32 + (long long)row_r * p.out_stride + cb);
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                if (p.accumulate)
                                    asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};"
                                                 :: "l"(d4 + i), "r"(v[4 * i]), "r"(v[4 * i + 1]), "r"(v[4 * i + 2]),
                                                    "r"(v[4 * i + 3]) : "memory");
                                else
                                    d4[i] = make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]),
                                                        __uint_as_float(v[4 * i + 2]), __uint_as_float(v[4 * i + 3]));
                            }
                        }
                        return;
                    }
                    if (p.add_f32 && row_r < M) {
                        const float4* a4 = reinterpret_cast<const float4*>(p.add_f32 + (long long)row_r * p.out_stride + cb);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float4 g = a4[i];
                            v[4 * i] = __float_as_uint(__uint_as_float(v[4 * i]) + g.x);
                            v[4 * i + 1] = __float_as_uint(__uint_as_float(v[4 * i + 1]) + g.y);
                            v[4 * i + 2] = __float_as_uint(__uint_as_float(v[4 * i + 2]) + g.z);
                            v[4 * i + 3] = __float_as_uint(__uint_as_float(v[4 * i + 3]) + g.w);
                        }
                    }
                    const int half = (cb >> 5) & 1;
                    const uint32_t tile = smem_addr(drain_stage) + (uint32_t)((warp - 2) * 8192 + out_tile * 4096);
                    if (half == 0) {                     // the store that read this tile last has read it
                        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
                        __syncwarp();
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t q[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(q[j])
                                : "f"(__uint_as_float(v[8 * i + 2 * j + 1])), "f"(__uint_as_float(v[8 * i + 2 * j])));
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};"
                                     :: "r"(tile + (uint32_t)(lane * 128 + (((4 * half + i) ^ (lane & 7)) << 4))),
                                        "r"(q[0]), "r"(q[1]), "r"(q[2]), "r"(q[3]) : "memory");
                    }
                    if (half == 1) {
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) {
                            // (rows past the vocabulary's end are clipped by the tensor map)
                            if (row_r - lane < M)
                                asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];"
                                             :: "l"(&map_c), "r"(tile), "r"(cb - 32), "r"(row_r) : "memory");
                            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                        }
                        out_tile ^= 1;
                    }
                };
                (void)drain_w;
                auto consume = [&](int ac, uint32_t (&v)[32]) {
                    // accumulator a of this unit: the token (vocabulary) tile 2 a further on, TMEM columns a * 256 ..
                    const int a = ac / (BN / 32), c = ac - a * (BN / 32);
                    const int row_a = row + a * 2 * BM;
                    const bool row_ok_a = row_a < M;
                    const int cb = col0 + c * 32;
                    if (cb >= p.N) return;               // whole chunk beyond the valid columns (warp-uniform)
                    if (no_k) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = 0u;
                    }
                    const int nvalid = min(32, p.N - cb);
                    if (CE && p.mode == kGradW) {
                        drain_w(row_a, cb, v);
                        return;
                    }
                    if (p.mode == kLse) {
                        take_target(cb, v);
                        float cm = -INFINITY;
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (i < nvalid) cm = fmaxf(cm, __uint_as_float(v[i]));
                        if (cm > run_m) {
                            // a larger maximum shifts every exponent so far by dx <= 0:
                            // s -> 2^dx s,  u -> 2^dx (u + dx s)
                            const float dx = (run_m - cm) * kLog2e;       // -inf on the first chunk
                            const float f = ex2_approx(dx);               // exp2(-inf) = 0 on the first chunk
                            if (p.part_u) run_u = (run_m == -INFINITY) ? 0.0f : f * fmaf(dx, run_s, run_u);
                            run_s *= f;
                            run_m = cm;
                        }
                        // (nothing but -inf so far, log-prob only: they add zero; against a maximum of -inf they would add NaN)
                        const float off = (run_m == -INFINITY && !p.part_u) ? 0.0f : -run_m * kLog2e;
                        float s0 = 0.0f, s1 = 0.0f;
                        if (p.part_u) {
                            float u0 = 0.0f, u1 = 0.0f;
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                if (i < nvalid) {
                                    const float x = fmaf(__uint_as_float(v[i]), kLog2e, off), e = ex2_approx(x);
                                    s0 += e;
                                    u0 = fmaf(e, x, u0);
                                }
                                if (i + 1 < nvalid) {
                                    const float x = fmaf(__uint_as_float(v[i + 1]), kLog2e, off), e = ex2_approx(x);
                                    s1 += e;
                                    u1 = fmaf(e, x, u1);
                                }
                            }
                            run_u += u0 + u1;
                        } else {
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                if (i < nvalid) s0 += ex2_approx(fmaf(__uint_as_float(v[i]), kLog2e, off));
                                if (i + 1 < nvalid) s1 += ex2_approx(fmaf(__uint_as_float(v[i + 1]), kLog2e, off));
                            }
                        }
                        run_s += s0 + s1;
                    } else if (p.mode == kGradHidden) {
                        if (row_ok_a) {
                            const long long orow = p.row_index ? (long long)p.row_index[p.live_off + row_a] : (long long)row_a;
                            __nv_bfloat16* dst = p.out_bf16 + orow * p.out_stride + cb;
                            const float sc = p.row_scale ? p.row_scale[row_a] : 1.0f;
                            float so = sc;
                            if (CE && k_split > 1) {
                                // a piece's raw sums (nvalid is a multiple of 4)
                                float4* d4 = reinterpret_cast<float4*>(p.k_part + ((long long)piece * M + row_a) * p.out_stride + cb);
#pragma unroll
                                for (int i = 0; i < 8; ++i)
                                    if (4 * i < nvalid)
                                        d4[i] = make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]),
                                                            __uint_as_float(v[4 * i + 2]), __uint_as_float(v[4 * i + 3]));
                                return;
                            }
                            if (CE && sc == 0.0f) {
                                // a row that was taken out: zeros, whatever its zero entries met in W
#pragma unroll
                                for (int i = 0; i < 32; ++i) v[i] = 0u;
                            } else if (CE && p.col_vec) {
                                const float ra = p.row_add[row_a];
#pragma unroll
                                for (int i = 0; i < 32; ++i)
                                    if (i < nvalid) v[i] = __float_as_uint(fmaf(__uint_as_float(v[i]), sc, ra * p.col_vec[cb + i]));
                                so = 1.0f;
                            }
                            if (nvalid == 32) {
                                uint32_t o[16];
#pragma unroll
                                for (int i = 0; i < 16; ++i)
                                    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[i])
                                        : "f"(__uint_as_float(v[2 * i + 1]) * so), "f"(__uint_as_float(v[2 * i]) * so));
                                uint4* d4 = reinterpret_cast<uint4*>(dst);
                                d4[0] = make_uint4(o[0], o[1], o[2], o[3]);
                                d4[1] = make_uint4(o[4], o[5], o[6], o[7]);
                                d4[2] = make_uint4(o[8], o[9], o[10], o[11]);
                                d4[3] = make_uint4(o[12], o[13], o[14], o[15]);
                            } else {
#pragma unroll
                                for (int i = 0; i < 32; ++i)
                                    if (i < nvalid) dst[i] = __float2bfloat16_rn(__uint_as_float(v[i]) * so);
                            }
                        }
                    } else if (ACC2 && nvalid == 32) {   // kGradW, two-accumulator form: the drain is not hidden
                        // One accumulator row per thread means a warp's store touches 32 rows for 16 bytes
                        // each.  The 32 x 32 chunk goes through a padded staging tile in shared memory
                        // instead (rows of 144 bytes: conflict-free both ways), and comes back with eight
                        // lanes along each row, so that a warp's store covers 4 rows x 128 contiguous bytes.
                        float* stg = drain_stage + (warp - 2) * (32 * kDrainPitch);
                        float4* w4 = reinterpret_cast<float4*>(stg + lane * kDrainPitch);
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            w4[i] = make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]),
                                                __uint_as_float(v[4 * i + 2]), __uint_as_float(v[4 * i + 3]));
                        __syncwarp();
                        const int piece8 = lane & 7, rq = lane >> 3;
                        const int row_w0 = row_a - lane;                 // first row of this warp's 32
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const int r = rq + 4 * j;
                            const float4 val = *reinterpret_cast<const float4*>(stg + r * kDrainPitch + piece8 * 4);
                            if (row_w0 + r < M) {
                                float4* d4 = reinterpret_cast<float4*>(p.out_f32 + (long long)(row_w0 + r) * p.out_stride + cb) + piece8;
                                // accumulation is a fire-and-forget vector reduction at the memory side (no
                                // read round trip in the drain); each element gets exactly one addend per
                                // launch, so the result does not depend on timing
                                if (p.accumulate)
                                    asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};"
                                                 :: "l"(d4), "f"(val.x), "f"(val.y), "f"(val.z), "f"(val.w) : "memory");
                                else
                                    *d4 = val;
                            }
                        }
                        __syncwarp();                                    // the tile is free for the next chunk
                    } else {   // kGradW
                        if (row_ok_a) {
                            float* dst = p.out_f32 + (long long)row_a * p.out_stride + cb;
                            if (nvalid == 32) {
                                float4* d4 = reinterpret_cast<float4*>(dst);
#pragma unroll
                                for (int i = 0; i < 8; ++i) {
                                    if (p.accumulate)
                                        asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};"
                                                     :: "l"(d4 + i), "r"(v[4 * i]), "r"(v[4 * i + 1]), "r"(v[4 * i + 2]),
                                                        "r"(v[4 * i + 3]) : "memory");
                                    else
                                        d4[i] = make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]),
                                                            __uint_as_float(v[4 * i + 2]), __uint_as_float(v[4 * i + 3]));
                                }
                            } else {
#pragma unroll
                                for (int i = 0; i < 32; ++i)
                                    if (i < nvalid) dst[i] = __uint_as_float(v[i]) + (p.accumulate ? dst[i] : 0.0f);
                            }
                        }
                    }
                };
                constexpr int kChunks = NACC * (BN / 32);
                const uint32_t t_buf = t_row;
                uint32_t va[32], vb[32];
                if (!no_k) tc_ld32_issue(t_buf, va);
#pragma unroll 1
                for (int ac = 0; ac < kChunks; ac += 2) {
                    if (!no_k) {
                        tc_ld_wait(va);
                        tc_ld32_issue(t_buf + (uint32_t)((ac + 1) * 32), vb);      // kChunks is even
                    }
                    consume(ac, va);
                    if (!no_k) {
                        tc_ld_wait(vb);
                        if (ac + 2 < kChunks) tc_ld32_issue(t_buf + (uint32_t)((ac + 2) * 32), va);
                    }
                    consume(ac + 1, vb);
                }
                }
                // hand the accumulator buffer back to the MMA warp
                tc_fence_before();
                __syncwarp();
                if (lane == 0 && !no_k) {
                    if (PAIR) mbar_arrive_cluster(map_to_cta(smem_addr(&ctl->tmem_empty[buf]), 0));
                    else mbar_arrive(smem_addr(&ctl->tmem_empty[buf]));
                }
                tphase[buf] ^= 1u;
                if (!ACC2) buf ^= 1;
            }
            if (p.mode == kLse && row_ok && ok) {
                // inverse of unit_range's n0(sp)
                const int big = split_rem * (split_base + 1);
                const int sp = n0 < big ? n0 / (split_base + 1) : split_rem + (n0 - big) / max(split_base, 1);
                p.part[(long long)row * p.nsplit + sp] = make_float2(run_m, run_s);
                if (p.part_u) p.part_u[(long long)row * p.nsplit + sp] = run_u;
            }
        }
        // (CE) the last output tiles have been written before their shared memory goes
        if (CE && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }

    // ---------------- teardown ----------------
    tc_fence_before();
    __syncthreads();
    if (ctl->abort_flag) {
        // copies or MMAs may still be in flight: give them time before the memory is released
        if (threadIdx.x == 0 && p.dev_status) atomicOr(p.dev_status, RLF_DEV_TIMEOUT);
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    }
    if (PAIR) pair_sync();        // the peer may still be signalling this CTA's barriers until here
    if (warp == 0) {
        tc_fence_after();
        if (PAIR)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(tmem_base), "r"((uint32_t)kTmemCols) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem_base), "r"((uint32_t)kTmemCols) : "memory");
    }
}

// ---- small kernels around it ----------------------------------------------------------------
// <h, w> over D bf16 elements by one warp, fp32 accumulation (every lane gets the sum)
__device__ __forceinline__ float warp_dot_bf16(const uint4* __restrict__ h, const uint4* __restrict__ w, int D, int lane) {
    float acc = 0.0f;
    for (int i = lane; i < D / 8; i += 32) {
        const uint4 a = h[i], b = w[i];
        const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, bw[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            acc = fmaf(__uint_as_float(aw[k] << 16), __uint_as_float(bw[k] << 16), acc);
            acc = fmaf(__uint_as_float(aw[k] & 0xffff0000u), __uint_as_float(bw[k] & 0xffff0000u), acc);
        }
    }
    return warp_sum(acc);
}

// z_target[t] = <hidden[t, :], W[ids[t], :]> in fp32: one warp per token
__global__ void __launch_bounds__(256)
target_logit_kernel(const __nv_bfloat16* __restrict__ hidden, const __nv_bfloat16* __restrict__ W,
                    const float4* __restrict__ rec, int64_t T, int32_t D, float* __restrict__ zy) {
    const int64_t t = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (t >= T) return;
    const int lane = threadIdx.x & 31;
    const int y = __float_as_int(rec[t].w) & 0x7fffffff;
    const uint4* h = reinterpret_cast<const uint4*>(hidden + t * (int64_t)D);
    const uint4* w = reinterpret_cast<const uint4*>(W + (int64_t)y * D);
    const float acc = warp_dot_bf16(h, w, D, lane);
    if (lane == 0) zy[t] = acc;
}

// One token's row statistics from its per-split (max, sum exp) partials, and its gradient coefficient
// c_t = -(w_t) (dpg/dlogp + beta (1 - exp(ref - logp))), w_t = the token's loss weight.
struct TokenStats {
    float lse, logp, coef;
    bool finite;
};
__device__ __forceinline__ TokenStats token_stats(const float2* __restrict__ parts, int nsplit, float zy, const float4 rec,
                                                  const float* __restrict__ wtok, int64_t t,
                                                  const long long* __restrict__ denom, float eps_clip, float eps_hi,
                                                  float beta) {
    float M = -INFINITY;
    for (int j = 0; j < nsplit; ++j) M = fmaxf(M, parts[j].x);
    float S = 0.0f;
    for (int j = 0; j < nsplit; ++j) {
        const float2 ms = parts[j];
        S += ms.x == -INFINITY ? ms.y : ms.y * expf(ms.x - M);      // (0 for a split of -inf, NaN where it held a NaN)
    }
    TokenStats o;
    o.lse = M + logf(S);
    o.logp = (zy - M) - logf(S);
    o.finite = (M > -INFINITY) && (M < INFINITY) && (S > 0.0f) && (S < INFINITY) && (fabsf(o.logp) < INFINITY);
    o.coef = 0.0f;
    if ((__float_as_int(rec.w) < 0) && o.finite) {
        const long long N = *denom;
        const float inv_n = wtok ? wtok[t] : 1.0f / (float)(N > 1 ? N : 1);
        const float A = rec.z;
        const float rho = expf(o.logp - rec.x);
        const bool clipped = ((A > 0.0f) && (rho > 1.0f + eps_hi)) || ((A < 0.0f) && (rho < 1.0f - eps_clip));
        const float dpg = clipped ? 0.0f : -A * rho;
        o.coef = -inv_n * fmaf(beta, -expm1f(rec.y - o.logp), dpg);
    }
    return o;
}

// merge the per-split (max, sum exp) pairs of every token into lse, logp and the gradient coefficient
__global__ void __launch_bounds__(256)
combine_kernel(const float2* __restrict__ part, int nsplit, const float* __restrict__ zy,
               const float4* __restrict__ rec, int64_t T, const long long* __restrict__ denom, float eps_clip,
               float eps_hi, const float* __restrict__ wtok, float beta, float* __restrict__ logp_out,
               float* __restrict__ lse_out, float* __restrict__ coef_out, int32_t* __restrict__ dev_status) {
    const int64_t t = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (t >= T) return;
    const TokenStats ts = token_stats(part + t * nsplit, nsplit, zy[t], rec[t], wtok, t, denom, eps_clip, eps_hi, beta);
    logp_out[t] = ts.finite ? ts.logp : __int_as_float(0x7fc00000);
    lse_out[t] = ts.finite ? ts.lse : 0.0f;
    coef_out[t] = ts.coef;
    if (!ts.finite && dev_status) atomicOr(dev_status, RLF_DEV_NONFINITE);
}

// forward-only pass from target ids alone: z_target per token (NaN and a status bit for an id outside
// the vocabulary), one warp per token
__global__ void __launch_bounds__(256)
target_logit_ids_kernel(const __nv_bfloat16* __restrict__ hidden, const __nv_bfloat16* __restrict__ W,
                        const int32_t* __restrict__ ids, int64_t T, int32_t D, int32_t V, float* __restrict__ zy,
                        int32_t* __restrict__ dev_status) {
    const int64_t t = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (t >= T) return;
    const int lane = threadIdx.x & 31;
    const int y = ids[t];
    if (y < 0 || y >= V) {
        if (lane == 0) {
            zy[t] = __int_as_float(0x7fc00000);
            if (dev_status) atomicOr(dev_status, RLF_DEV_BAD_TARGET);
        }
        return;
    }
    const uint4* h = reinterpret_cast<const uint4*>(hidden + t * (int64_t)D);
    const uint4* w = reinterpret_cast<const uint4*>(W + (int64_t)y * D);
    const float acc = warp_dot_bf16(h, w, D, lane);
    if (lane == 0) zy[t] = acc;
}

// merge the per-split (max, s, u) triples of every token: logp = z_y - lse, H = ln S - ln2 U / S with
// S = sum_k s_k 2^dx_k, U = sum_k 2^dx_k (u_k + s_k dx_k), dx_k the split's base against the row maximum
__global__ void __launch_bounds__(256)
combine_logp_entropy_kernel(const float2* __restrict__ part, const float* __restrict__ part_u, int nsplit,
                            const float* __restrict__ zy, int64_t T, float* __restrict__ logp_out,
                            float* __restrict__ entropy_out, int32_t* __restrict__ dev_status) {
    const int64_t t = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (t >= T) return;
    float M = -INFINITY;
    for (int j = 0; j < nsplit; ++j) M = fmaxf(M, part[t * nsplit + j].x);
    float S = 0.0f, U = 0.0f;
    for (int j = 0; j < nsplit; ++j) {
        const float2 ms = part[t * nsplit + j];
        if (ms.x == -INFINITY) {
            S += ms.y;                           // 0, or NaN where there was one
            continue;
        }
        const float dx = (ms.x - M) * kLog2e;
        const float f = exp2f(dx);
        S += ms.y * f;
        if (part_u && f > 0.0f) U += f * fmaf(ms.y, dx, part_u[t * nsplit + j]);
    }
    const float lnS = logf(S);
    const float logp = (zy[t] - M) - lnS;
    const bool finite = (M > -INFINITY) && (M < INFINITY) && (S > 0.0f) && (S < INFINITY);
    const float nan = __int_as_float(0x7fc00000);
    logp_out[t] = (finite && fabsf(logp) < INFINITY) ? logp : nan;      // NaN z_y (bad target id) stays NaN
    if (entropy_out) entropy_out[t] = finite ? lnS - kLn2 * U / S : nan;
    if (!finite && dev_status) atomicOr(dev_status, RLF_DEV_NONFINITE);
}

// Masked rows contribute nothing to either gradient, so the backward (and the part of the forward
// that keeps logits for it) runs over the unmasked rows only.  Stable partition of the tokens by
// the live bit of their record (token order is kept inside each part, so results do not depend on
// timing): one CTA scans the T flags.  counts[0] = live rows, counts[1] = the others.
__global__ void __launch_bounds__(1024)
partition_rows_kernel(const float4* __restrict__ rec, int T, int32_t* __restrict__ idx_live,
                      int32_t* __restrict__ idx_dead, int* __restrict__ counts) {
    __shared__ int warp_tot[32];
    __shared__ int base_s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) base_s = 0;
    __syncthreads();
    for (int t0 = 0; t0 < T; t0 += 1024) {
        const int t = t0 + tid;
        const bool live = t < T && __float_as_int(rec[t].w) < 0;
        const unsigned bal = __ballot_sync(0xffffffffu, live);
        if (lane == 0) warp_tot[warp] = __popc(bal);
        __syncthreads();
        int before = 0, total = 0;
        for (int w = 0; w < 32; ++w) {
            const int c = warp_tot[w];
            if (w < warp) before += c;
            total += c;
        }
        const int base = base_s;
        const int live_before = base + before + __popc(bal & ((1u << lane) - 1u));
        if (live) idx_live[live_before] = t;
        else if (t < T) idx_dead[t - live_before] = t;
        __syncthreads();
        if (tid == 0) base_s = base + total;
    }
    __syncthreads();
    if (tid == 0) { counts[0] = base_s; counts[1] = T - base_s; }
}

// out row r <- hidden row idx[r] for r < *count; rows up to the next multiple of 256 are zero-filled
// (the contractions read whole tiles)
// ref_out (optional): the reference of row r's stored exponentials, its target logit plus kRefShift
constexpr float kRefShift = 32.0f;
__global__ void __launch_bounds__(128)
gather_rows_kernel(const __nv_bfloat16* __restrict__ hidden, int D, const int32_t* __restrict__ idx,
                   const int* __restrict__ count, __nv_bfloat16* __restrict__ out, const float* __restrict__ zy,
                   float* __restrict__ ref_out) {
    const int n = *count;
    const int r = blockIdx.x;
    if (r >= ((n + 255) & ~255)) return;
    if (ref_out && threadIdx.x == 0) ref_out[r] = r < n ? zy[idx[r]] + kRefShift : 0.0f;
    uint4* dst = reinterpret_cast<uint4*>(out + (long long)r * D);
    const int nv = D / 8;
    if (r < n) {
        const uint4* src = reinterpret_cast<const uint4*>(hidden + (long long)idx[r] * D);
        for (int i = threadIdx.x; i < nv; i += blockDim.x) dst[i] = src[i];
    } else {
        for (int i = threadIdx.x; i < nv; i += blockDim.x) dst[i] = make_uint4(0u, 0u, 0u, 0u);
    }
}

// skip-masked form: the rows without loss weight are not multiplied at all; their log-prob reads NaN
__global__ void __launch_bounds__(256)
fill_nan_rows_kernel(const int32_t* __restrict__ idx, const int* __restrict__ count, float* __restrict__ logp_out) {
    const int r = blockIdx.x * blockDim.x + threadIdx.x;
    if (r < *count) logp_out[idx[r]] = __int_as_float(0x7fc00000);
}

// combine_kernel for a launch over gathered rows: row r of the launch (partials part[r][.]) is token
// idx[off + r]; logp goes to the token's place, lse / coefficient / target id to the gathered place.
//
// With ref_g (the sweep stored e = exp(z - rho_r), rho_r = ref_g[off + r]) the kernel also finishes the
// row for the gradient contractions: scale_g = c_t exp(rho - lse), the per-row factor that turns the
// stored exponentials into dZ, and the target column of the scratch is overwritten with
// (p_y - 1) exp(lse - rho) (formed in fp32 from the fp32 target logit), so that factor x entry is
// c_t (p_y - 1) to bf16 rounding even when p_y is close to one.  The reference is usable while the
// factor and the entries stay normal numbers: a row with a non-finite sum or lse - rho above
// kRefWindow raises *fallback instead of a status bit, and the chunk is redone with per-tile maxima.
// Without ref_g, scale_g (if given) is set to one: the scratch will hold dZ itself.
constexpr float kRefWindow = 46.0f;
__global__ void __launch_bounds__(256)
combine_rows_kernel(const float2* __restrict__ part, int nsplit, int rows_max, const int32_t* __restrict__ idx,
                    const int* __restrict__ count, int off, const float* __restrict__ zy,
                    const float4* __restrict__ rec, const long long* __restrict__ denom, float eps_clip, float eps_hi,
                    const float* __restrict__ wtok, float beta, float* __restrict__ logp_out, float* __restrict__ lse_g,
                    float* __restrict__ coef_g, int32_t* __restrict__ y_g, int32_t* __restrict__ dev_status,
                    const float* __restrict__ ref_g, float* __restrict__ scale_g, __nv_bfloat16* __restrict__ dz,
                    int dz_nc, int V, int* __restrict__ fallback, const int* __restrict__ run_flag, int run_want) {
    if (run_flag && *run_flag != run_want) return;
    const int r = blockIdx.x * blockDim.x + threadIdx.x;
    const int n = max(0, min(*count - off, rows_max));
    if (r >= n) return;
    const int t = idx[off + r];
    const float4 rc = rec[t];
    const TokenStats ts = token_stats(part + (long long)r * nsplit, nsplit, zy[t], rc, wtok, t, denom, eps_clip, eps_hi,
                                      beta);
    logp_out[t] = ts.finite ? ts.logp : __int_as_float(0x7fc00000);
    const int y = __float_as_int(rc.w) & 0x7fffffff;
    if (lse_g) {
        lse_g[off + r] = ts.finite ? ts.lse : 0.0f;
        coef_g[off + r] = ts.coef;
        y_g[off + r] = y;
    }
    if (ref_g) {
        const float rho = ref_g[off + r];
        const bool usable = ts.finite && (ts.lse - rho <= kRefWindow);
        if (!usable) {
            atomicOr(fallback, 1);
            scale_g[off + r] = 0.0f;
            return;
        }
        scale_g[off + r] = ts.coef * expf(rho - ts.lse);
        if (ts.coef != 0.0f && y < V) dz[dz_offset(r, y, dz_nc)] = __float2bfloat16_rn(expm1f(ts.logp) * expf(ts.lse - rho));
        return;
    }
    if (scale_g) scale_g[off + r] = 1.0f;
    if (!ts.finite && dev_status) atomicOr(dev_status, RLF_DEV_NONFINITE);
}

// Hs[r, :] = bf16(scale[off + r] * Hl[r, :]) for the rows of one chunk: the token-side operand of
// grad_W = e^T (scale H) when the scratch holds exponentials against a per-row reference.  Rows from
// the live extent up to the next multiple of 256 become zeros.
__global__ void __launch_bounds__(128)
scale_rows_kernel(const __nv_bfloat16* __restrict__ Hl, int D, int rows_max, const int* __restrict__ count, int off,
                  const float* __restrict__ scale_g, __nv_bfloat16* __restrict__ Hs) {
    const int n = max(0, min(*count - off, rows_max));
    const int r = blockIdx.x;
    if (r >= ((n + 255) & ~255)) return;
    uint4* dst = reinterpret_cast<uint4*>(Hs + (long long)r * D);
    const int nv = D / 8;
    if (r >= n) {
        for (int i = threadIdx.x; i < nv; i += blockDim.x) dst[i] = make_uint4(0u, 0u, 0u, 0u);
        return;
    }
    const float f = scale_g[off + r];
    const uint4* src = reinterpret_cast<const uint4*>(Hl + (long long)r * D);
    for (int i = threadIdx.x; i < nv; i += blockDim.x) {
        const uint4 z = src[i];
        const uint32_t w[4] = {z.x, z.y, z.z, z.w};
        uint32_t o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[k])
                : "f"(__uint_as_float(w[k] & 0xffff0000u) * f), "f"(__uint_as_float(w[k] << 16) * f));
        dst[i] = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

// in place over one chunk of stored exponentials e = exp(z - tile max): dZ = coef (e exp(tile max - lse)
// - [v == y]) as bf16; the target column takes the fp32 target logit.  Rows from the live extent up
// to the next multiple of 256 become zeros.  A work item is one (token tile, 256-column tile): four adjacent
// blocks of the scratch, 64 KB of contiguous memory; the CTAs stride over the items (the launch is
// usually one that a device flag turns into a no-op, which a small grid makes cheap).
// CE (cross-entropy form): the row's target entry comes ready-made in tgt_g, y_g is negative for a row
// without a gradient, and zy / idx are not used.
template <bool CE>
__global__ void __launch_bounds__(256)
dz_from_e_kernel(__nv_bfloat16* __restrict__ ebuf, int V, int n_tiles, const float* __restrict__ tmax, int rows_max,
                 const int* __restrict__ count, int off, const float* __restrict__ lse_g,
                 const float* __restrict__ coef_g, const int32_t* __restrict__ y_g, const int32_t* __restrict__ idx,
                 const float* __restrict__ zy, const float* __restrict__ tgt_g, const int* __restrict__ run_flag,
                 int run_want) {
    __shared__ float f_s[kDzBlockRows];          // signed scale of each row for this column tile
    if (run_flag && *run_flag != run_want) return;
    __shared__ int live_s[kDzBlockRows];
    const int n = max(0, min(*count - off, rows_max));
    const int nc = 4 * n_tiles;
    const long long items = (long long)(((n + 255) & ~255) / kDzBlockRows) * n_tiles;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
    const int tt = (int)(item / n_tiles), jt = (int)(item - (long long)tt * n_tiles);
    __syncthreads();                             // the previous item's readers of f_s / live_s are done
    if (threadIdx.x < kDzBlockRows) {
        const int r = tt * kDzBlockRows + threadIdx.x;
        const float coef = r < n ? coef_g[off + r] : 0.0f;
        float f = 0.0f;
        if (coef != 0.0f) {
            const float c2 = lg2_approx(fabsf(coef)) - lse_g[off + r] * kLog2e;
            f = copysignf(ex2_approx(fmaf(tmax[(long long)r * n_tiles + jt], kLog2e, c2)), coef);
        }
        f_s[threadIdx.x] = f;
        live_s[threadIdx.x] = CE ? (r < n && y_g[off + r] >= 0) : (coef != 0.0f);
    }
    __syncthreads();
    uint4* base = reinterpret_cast<uint4*>(ebuf + dz_offset((long long)tt * kDzBlockRows, jt * BN, nc));
    // 4 blocks x 128 rows x 8 vectors of 16 bytes
    for (int i = threadIdx.x; i < 4 * kDzBlockRows * 8; i += 256) {
        const int rr = (i >> 3) & (kDzBlockRows - 1);
        if (!live_s[rr]) {
            base[i] = make_uint4(0u, 0u, 0u, 0u);
            continue;
        }
        const float f = f_s[rr];
        const uint4 z = base[i];
        const uint32_t w[4] = {z.x, z.y, z.z, z.w};
        uint32_t o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[k])
                : "f"(__uint_as_float(w[k] & 0xffff0000u) * f), "f"(__uint_as_float(w[k] << 16) * f));
        base[i] = make_uint4(o[0], o[1], o[2], o[3]);
    }
    __syncthreads();
    if (threadIdx.x < kDzBlockRows && live_s[threadIdx.x]) {
        const int r = tt * kDzBlockRows + threadIdx.x;
        const int y = y_g[off + r];
        if (y >= jt * BN && y < jt * BN + BN && y < V) {
            if (CE) {
                ebuf[dz_offset(r, y, nc)] = __float2bfloat16_rn(tgt_g[off + r]);
                continue;
            }
            const float coef = coef_g[off + r];
            const float py = ex2_approx((zy[idx[off + r]] - lse_g[off + r]) * kLog2e);
            ebuf[dz_offset(r, y, nc)] = __float2bfloat16_rn(fmaf(coef, py, -coef));
        }
    }
    }
}

// ---- host side ------------------------------------------------------------------------------
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeTiledFn encode_fn() {
    static std::mutex mu;
    static EncodeTiledFn fn = nullptr;
    std::lock_guard<std::mutex> lock(mu);
    if (!fn) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(p);
    }
    return fn;
}

// bf16 row-major matrix [rows][cols] (cols contiguous); box = box_cols x box_rows, 128-byte swizzle
static bool make_map(CUtensorMap* map, const void* base, uint64_t rows, uint64_t cols, uint64_t row_stride_elems,
                     uint32_t box_cols, uint32_t box_rows) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {cols, rows};
    const cuuint64_t strides[1] = {row_stride_elems * 2};
    const cuuint32_t box[2] = {box_cols, box_rows};
    const cuuint32_t estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static int sm_count_lm() {
    int dev = 0, v = 0;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev);
    return v > 0 ? v : 148;
}

static std::atomic<int> g_pair{1};       // 1: cta_group::2 pair form, 0: single-CTA form
static std::atomic<int> g_m_block{0};    // row units per scheduling block of the sweep; 0: automatic
static std::atomic<int> g_max_workers{0};   // persistent CTAs (or pairs) per launch; 0: one per SM (pair of SMs)
static std::atomic<int> g_chunk_tiles{0};   // token tiles per backward chunk; 0: the most the workspace holds
static std::atomic<int> g_pace{1};          // pacing of the workers' loads (see GemmParams::pace): 1 on, 0 off
static std::atomic<int> g_row_ref{1};       // backward scratch: 1 exponentials against a per-row reference, 0 per-tile maxima

// what a launch settled that the kernels after it have to know
struct Sched { int workers, auto_units; };

template <bool PAIR, bool ACC2, bool CE = false>
static rlf_status launch_gemm_t(const CUtensorMap& ma, const CUtensorMap& mb, const CUtensorMap& mc, const GemmParams& p,
                                cudaStream_t s, Sched* sched) {
    static std::mutex mu;
    static bool opted[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    {
        std::lock_guard<std::mutex> lock(mu);
        if (dev >= 0 && dev < 64 && !opted[dev]) {
            if (cudaFuncSetAttribute((const void*)umma_gemm_kernel<PAIR, ACC2, CE>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                     Cfg<PAIR, ACC2, CE>::kSmemBytes) != cudaSuccess) {
                cudaGetLastError();
                return RLF_ERR_CUDA;
            }
            opted[dev] = true;
        }
    }
    const bool sweep = p.mode == kLse;
    constexpr int kTilesPerUnit = (PAIR ? 2 : 1) * (ACC2 ? 2 : 1);
    const int m_units = (p.m_tiles + kTilesPerUnit - 1) / kTilesPerUnit;
    const int units = sweep ? m_units * p.nsplit : m_units * p.n_tiles * (p.k_split_max > 1 ? p.k_split_max : 1);
    if (units <= 0) return RLF_OK;
    int workers = PAIR ? sm_count_lm() / 2 : sm_count_lm();
    // Sweep schedule: the CTAs (or pairs) running at one time cover m_block row units x (workers / m_block)
    // splits, in lockstep.  Their token tiles (256 x D bf16 per pair: 1.3 MB at D = 2560, 2 MB at 4096)
    // are re-read for every column tile and must stay in L2 next to the streaming head: with all 74 pairs
    // on different row units (97 MB at D = 2560) they did not, and the same launch drew its 1 kW at
    // 1.06 GHz instead of 1.39 GHz.  So m_block is what keeps about 48 MB of token tiles live, at most half
    // the workers, and a divisor of the worker count (blocks that leave the splits misaligned cost
    // 4 - 10 %): when no nearby divisor exists a few workers are left out instead (D = 4096: 24 row
    // units on 72 of the 74 pairs measured 5 % faster than 37 on 74; D = 2560 keeps 37 on 74).
    if (g_max_workers.load() > 0 && g_max_workers.load() < workers) workers = g_max_workers.load();
    GemmParams q = p;
    q.m_block = workers / 2 > 0 ? workers / 2 : 1;
    if (sweep && g_m_block.load() == 0 && g_max_workers.load() == 0) {
        const double unit_bytes = (double)(PAIR ? 2 : 1) * BM * (double)p.k_slabs * BK * 2.0;
        const double target = 48.0 * 1024 * 1024 / unit_bytes;
        int hi = (int)(target * 1.05);
        if (hi > workers / 2) hi = workers / 2;
        if (hi < 1) hi = 1;
        int lo = (int)(target * 0.6);
        if (lo < 1) lo = 1;
        int best_mb = hi, best_w = workers / hi * hi;
        for (int mb = hi - 1; mb >= lo; --mb) {
            const int w = workers / mb * mb;
            if (w > best_w) { best_w = w; best_mb = mb; }
        }
        q.m_block = best_mb;
        // a sweep that may size itself on the device launches every worker; the blocked form leaves some of them out there
        q.block_workers = best_w;
        if (p.auto_units > 0) q.auto_units = hi < 64 ? hi : 64;
        else workers = best_w;
    } else {
        q.block_workers = workers;
        if (p.auto_units > 0) q.auto_units = 1;
    }
    if (g_m_block.load() > 0) q.m_block = g_m_block.load();
    if (workers > units) workers = units;
    if (sched) {
        sched->workers = workers;
        sched->auto_units = q.auto_units;
    }
    // Pacing, measured at full size with one-pass ncu counts: grad_hidden 32 -> 10 GB of HBM reads and
    // 9.6 -> 8.5 ms per launch, grad_W 35 -> 11 GB and 10.3 -> 9.1 ms (D = 2560); the sweep at D = 4096
    // 71 -> 61 ms.  Meeting points inside a unit were tried too and cost more than they return.
    if (q.pace && g_pace.load() != 0) {
        if (!q.pace_is_zero && cudaMemsetAsync(q.pace, 0, sizeof(int), s) != cudaSuccess) return RLF_ERR_CUDA;
    } else {
        q.pace = nullptr;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(PAIR ? 2 * workers : workers);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Cfg<PAIR, ACC2, CE>::kSmemBytes;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = PAIR ? 2 : 1;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, umma_gemm_kernel<PAIR, ACC2, CE>, ma, mb, mc, q) != cudaSuccess) {
        cudaGetLastError();
        return RLF_ERR_CUDA;
    }
    count_launch();
    return RLF_OK;
}

static std::atomic<int> g_acc2{1};          // gradient contractions in pair form: 1 two accumulators per CTA, 0 one
static rlf_status launch_gemm(const CUtensorMap& ma, const CUtensorMap& mb, const GemmParams& p, bool pair,
                              cudaStream_t s, Sched* sched = nullptr) {
    if (!pair) return launch_gemm_t<false, false>(ma, mb, ma, p, s, sched);
    if (p.mode != kLse && g_acc2.load() != 0) return launch_gemm_t<true, true>(ma, mb, ma, p, s, sched);
    return launch_gemm_t<true, false>(ma, mb, ma, p, s, sched);
}
// gradient contractions of the cross-entropy form; mc: the bf16 grad_W that they store to, if any
static rlf_status launch_gemm_ce(const CUtensorMap& ma, const CUtensorMap& mb, const CUtensorMap& mc, const GemmParams& p,
                                 bool pair, bool acc2, cudaStream_t s, Sched* sched = nullptr) {
    if (!pair) return launch_gemm_t<false, false, true>(ma, mb, mc, p, s, sched);
    if (acc2) return launch_gemm_t<true, true, true>(ma, mb, mc, p, s, sched);
    return launch_gemm_t<true, false, true>(ma, mb, mc, p, s, sched);
}

// Rows of dZ held in scratch at a time: up to 148 token tiles = 37 units of the two-accumulator
// gradient contractions (37 x D/256 = 370 units at D = 2560: five whole waves on 74 CTA pairs) = two
// scheduling blocks of the sweep; 5.8 GB at V = 151936.  Larger chunks mean fewer passes over the head
// in grad_hidden and fewer accumulations into grad_W.
constexpr int kChunkTokens = 148 * BM;
constexpr int kMaxSplit = 64;               // most vocabulary splits a sweep may use (sizes the partials)

// Number of vocabulary splits of a sweep.  A work unit is (pair of token tiles, split); the units are
// dealt round-robin to the persistent CTAs, which keep their load / multiply / drain pipelines
// running across units, so small units cost nothing, while large ones leave a ragged last wave
// (the number of rows that take part is only known on the device).  Splits of at least 8 column
// tiles, at most kMaxSplit of them; concurrently running CTAs still work on the same few splits, so
// the head's rows are shared in L2.
static int pick_split(int n_tiles) {
    int per = (n_tiles + kMaxSplit - 1) / kMaxSplit;
    if (per < 8) per = 8;
    return (n_tiles + per - 1) / per;
}

struct LmWs {
    size_t n_count, partial, rec, zy, lse, coef, wtok, seqcnt, part, idx_live, idx_dead, lse_g, coef_g, y_g, ref_g, scale_g,
        hidden_g, hidden_s, tmax, dz, total;
};
static size_t up1k(size_t x) { return (x + 1023) & ~(size_t)1023; }
static LmWs lm_workspace(int64_t T, int32_t V, int32_t D) {
    LmWs w;
    size_t o = 0;
    const size_t Tn = (size_t)(T > 0 ? T : 0);
    const size_t Tp = (Tn + 255) & ~(size_t)255;     // compact arrays are padded to whole tile pairs
    w.n_count = o; o += 1024;                        // [0] mask count, [64] live / other row counts, [128] chunk flag, [256] pacing counter
    w.partial = o; o += up1k(token_loss_partial_bytes());
    w.rec = o;     o += up1k(16 * Tn);
    w.zy = o;      o += up1k(4 * Tn);
    w.lse = o;     o += up1k(4 * Tn);
    w.coef = o;    o += up1k(4 * Tn);
    w.wtok = o;    o += up1k(4 * Tn);                // sequence-mean aggregation: per-token weights
    w.seqcnt = o;  o += up1k(4 * (Tn + 1));          //   and unmasked tokens per response (B <= T + 1)
    w.part = o;    o += up1k(8 * Tn * kMaxSplit);
    w.idx_live = o; o += up1k(4 * Tp);
    w.idx_dead = o; o += up1k(4 * Tp);
    w.lse_g = o;   o += up1k(4 * Tp);
    w.coef_g = o;  o += up1k(4 * Tp);
    w.y_g = o;     o += up1k(4 * Tp);
    w.ref_g = o;   o += up1k(4 * Tp);                // per-row reference of the stored exponentials
    w.scale_g = o; o += up1k(4 * Tp);                // per-row factor exponentials -> dZ
    w.hidden_g = o; o += 2 * up1k(Tp * (size_t)(D > 0 ? D : 0) * 2);   // live rows, then the others
    const size_t chunk = Tp < (size_t)kChunkTokens ? Tp : (size_t)kChunkTokens;
    w.hidden_s = o; o += up1k(chunk * (size_t)(D > 0 ? D : 0) * 2);    // one chunk of live rows times their factors
    w.tmax = o;    o += up1k(4 * chunk * (size_t)((V + BN - 1) / BN));
    w.dz = o;
    o += up1k(chunk * (size_t)((V + BN - 1) / BN) * BN * 2);     // blocked: whole 256-column tiles
    w.total = o + 1024;
    return w;
}

}  // namespace lm

size_t lmhead_logp_workspace_bytes(int64_t T) {
    const size_t Tn = (size_t)(T > 0 ? T : 0);
    return 1024 + lm::up1k(4 * Tn) + lm::up1k(8 * Tn * lm::kMaxSplit) + lm::up1k(4 * Tn * lm::kMaxSplit) + 1024;
}

size_t lmhead_workspace_bytes(int64_t T, int32_t V, int32_t D) {
    if (V < 1 || D < 1) return 0;
    return lm::lm_workspace(T, V, D).total;
}

}  // namespace rlf

namespace rlf {
namespace lm {

// eps_clip is the lower clip width, eps_hi the upper one; aggregation 0 = token mean (denom counts
// tokens), 1 = sequence mean (denom counts responses); skip_masked: rows without loss weight are not
// multiplied at all and their log-prob reads NaN
static rlf_status fused_lmhead_impl(const void* hidden, const void* W, int64_t T, int32_t D, int32_t V,
                                    const int32_t* ids, const int32_t* seq_id, const float* adv, int32_t B,
                                    const float* old_logp, const float* ref_logp, const uint8_t* mask,
                                    float eps_clip, float eps_hi, float beta_kl, int aggregation, int skip_masked,
                                    const int64_t* denom, float* logp_out,
                                    double* loss_out, void* grad_hidden, float* grad_W,
                                    int accumulate_grad_W, void* workspace, size_t workspace_bytes,
                                    int32_t* dev_status, rlf_stream_t stream) {
    if (T < 0 || V < 1 || D < 1 || B < 0) return RLF_ERR_SHAPE;
    if (aggregation != 0 && aggregation != 1) return RLF_ERR_SHAPE;
    if (aggregation == 1 && (int64_t)B > T + 1) return RLF_ERR_SHAPE;
    if (D % 64 != 0 || V % 8 != 0) return RLF_ERR_SHAPE;
    if (T >= (1ll << 30)) return RLF_ERR_UNSUPPORTED;
    if (!loss_out) return RLF_ERR_NULL;
    if (T > 0 && (!hidden || !W || !ids || !seq_id || !adv || !old_logp || !ref_logp || !mask || !logp_out))
        return RLF_ERR_NULL;
    if (T > 0 && B == 0) return RLF_ERR_SHAPE;
    if (!aligned(hidden, 16) || !aligned(W, 16) || !aligned(grad_hidden, 16) || !aligned(grad_W, 16))
        return RLF_ERR_ALIGN;
    const LmWs w = lm_workspace(T, V, D);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < w.total) return RLF_ERR_WORKSPACE;
    rlf_status st = check_arch();
    if (st != RLF_OK) return st;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);

    // 1 KB alignment of the scratch pieces that TMA reads
    char* ws = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(workspace) + 1023) & ~(uintptr_t)1023);
    long long* n_count = reinterpret_cast<long long*>(ws + w.n_count);
    double* partial = reinterpret_cast<double*>(ws + w.partial);
    float4* rec = reinterpret_cast<float4*>(ws + w.rec);
    float* zy = reinterpret_cast<float*>(ws + w.zy);
    float* lse = reinterpret_cast<float*>(ws + w.lse);
    float* coef = reinterpret_cast<float*>(ws + w.coef);
    float2* part = reinterpret_cast<float2*>(ws + w.part);
    __nv_bfloat16* dz = reinterpret_cast<__nv_bfloat16*>(ws + w.dz);
    const __nv_bfloat16* H = static_cast<const __nv_bfloat16*>(hidden);
    const __nv_bfloat16* Wm = static_cast<const __nv_bfloat16*>(W);

    // token mean: dn is the token count (given, or counted by the record kernel); sequence mean: the
    // per-token weights carry the whole normalisation and dn is only a valid address to read
    const long long* dn = aggregation == 0 ? reinterpret_cast<const long long*>(denom) : nullptr;
    const bool count_here = dn == nullptr;
    if (count_here) {
        if (cudaMemsetAsync(n_count, 0, sizeof(long long), s) != cudaSuccess) return RLF_ERR_CUDA;
        dn = n_count;
    }
    float* wtok = nullptr;
    auto token_loss = [&](int64_t rows) {
        return launch_token_loss_w(logp_out, rec, rows, eps_clip, eps_hi, beta_kl, wtok, partial, dn, loss_out, s);
    };
    if (T == 0) return token_loss(0);

    st = launch_token_prep(ids, seq_id, adv, old_logp, ref_logp, mask, T, V, B, rec, count_here ? n_count : nullptr,
                           dev_status, s);
    if (st != RLF_OK) return st;
    if (aggregation == 1) {
        wtok = reinterpret_cast<float*>(ws + w.wtok);
        st = launch_seq_weights(rec, seq_id, T, B, reinterpret_cast<const long long*>(denom),
                                reinterpret_cast<int*>(ws + w.seqcnt), n_count + 4, wtok, s);
        if (st != RLF_OK) return st;
    }
    target_logit_kernel<<<(unsigned)((T + 7) / 8), 256, 0, s>>>(H, Wm, rec, T, D, zy);
    count_launch();
    if (cudaGetLastError() != cudaSuccess) return RLF_ERR_CUDA;

    const bool pair = g_pair.load() != 0;
    const uint32_t b_rows = pair ? BN / 2 : BN;       // rows of a K-major B tile that one CTA stages
    CUtensorMap mapW;
    if (!make_map(&mapW, Wm, (uint64_t)V, (uint64_t)D, (uint64_t)D, BK, b_rows)) return RLF_ERR_CUDA;
    GemmParams g = {};
    g.mode = kLse;
    g.N = V;
    g.n_tiles = (V + BN - 1) / BN;
    g.k_slabs = D / BK;
    g.part = part;
    g.dev_status = dev_status;
    g.pace = reinterpret_cast<int*>(ws + w.n_count + 256);
    auto set_rows = [&](GemmParams& q, int64_t rows) {
        q.M = (int)rows;
        q.m_tiles = (int)((rows + BM - 1) / BM);
        q.nsplit = pick_split(q.n_tiles);
        q.n_tiles_per_split = (q.n_tiles + q.nsplit - 1) / q.nsplit;
    };

    if (!grad_hidden && !grad_W && !skip_masked) {
        // forward only: one sweep over all rows, running (max, sum exp) per token and vocabulary split
        CUtensorMap mapH;
        if (!make_map(&mapH, H, (uint64_t)T, (uint64_t)D, (uint64_t)D, BK, BM)) return RLF_ERR_CUDA;
        set_rows(g, T);
        st = launch_gemm(mapH, mapW, g, pair, s);
        if (st != RLF_OK) return st;
        combine_kernel<<<(unsigned)((T + 255) / 256), 256, 0, s>>>(part, g.nsplit, zy, rec, T, dn, eps_clip, eps_hi, wtok,
                                                                    beta_kl, logp_out, lse, coef, dev_status);
        count_launch();
        if (cudaGetLastError() != cudaSuccess) return RLF_ERR_CUDA;
        return token_loss(T);
    }

    // forward + backward.  The tokens are partitioned (stably) into unmasked rows and the others;
    // their numbers stay on the device (no host sync), so every chunk is launched and the kernels
    // size themselves.  Unmasked rows, by chunks: forward sweep that also keeps the chunk's
    // exponentials (relative to tile maxima) as bf16 -> lse, logp, coefficient -> dZ in place -> grad_hidden rows, grad_W += chunk's part.
    // The other rows only need their log-prob: one forward sweep.
    int* counts = reinterpret_cast<int*>(ws + w.n_count + 64);
    int32_t* idx_live = reinterpret_cast<int32_t*>(ws + w.idx_live);
    int32_t* idx_dead = reinterpret_cast<int32_t*>(ws + w.idx_dead);
    float* lse_g = reinterpret_cast<float*>(ws + w.lse_g);
    float* coef_g = reinterpret_cast<float*>(ws + w.coef_g);
    int32_t* y_g = reinterpret_cast<int32_t*>(ws + w.y_g);
    const int64_t Tp = (T + 255) & ~(int64_t)255;
    __nv_bfloat16* Hl = reinterpret_cast<__nv_bfloat16*>(ws + w.hidden_g);
    __nv_bfloat16* Hd = reinterpret_cast<__nv_bfloat16*>(ws + w.hidden_g + up1k((size_t)Tp * D * 2));
    const bool bwd = grad_hidden || grad_W;
    // backward scratch: exponentials against a per-row reference (no rescaling pass; the per-tile-maximum
    // path stays queued behind a device flag for chunks whose reference turns out unusable), or the
    // per-tile-maximum path alone
    const bool row_ref = bwd && g_row_ref.load() != 0;
    float* ref_g = reinterpret_cast<float*>(ws + w.ref_g);
    float* scale_g = reinterpret_cast<float*>(ws + w.scale_g);
    __nv_bfloat16* Hs = reinterpret_cast<__nv_bfloat16*>(ws + w.hidden_s);
    int* chunk_flag = reinterpret_cast<int*>(ws + w.n_count + 128);
    partition_rows_kernel<<<1, 1024, 0, s>>>(rec, (int)T, idx_live, idx_dead, counts);
    gather_rows_kernel<<<(unsigned)Tp, 128, 0, s>>>(H, D, idx_live, counts, Hl, zy, row_ref ? ref_g : nullptr);
    if (!skip_masked) gather_rows_kernel<<<(unsigned)Tp, 128, 0, s>>>(H, D, idx_dead, counts + 1, Hd, nullptr, nullptr);
    count_launch(skip_masked ? 2 : 3);
    if (cudaGetLastError() != cudaSuccess) return RLF_ERR_CUDA;
    if (grad_hidden && cudaMemsetAsync(grad_hidden, 0, (size_t)T * D * 2, s) != cudaSuccess) return RLF_ERR_CUDA;

    const int tuned_tiles = g_chunk_tiles.load();
    const int64_t chunk_tokens = (tuned_tiles > 0 && tuned_tiles * BM < kChunkTokens) ? tuned_tiles * BM : kChunkTokens;
    for (int64_t t0 = 0; t0 < T; t0 += chunk_tokens) {
        const int64_t tc = (T - t0) < chunk_tokens ? (T - t0) : chunk_tokens;
        CUtensorMap mapHc;
        if (!make_map(&mapHc, Hl + t0 * D, (uint64_t)tc, (uint64_t)D, (uint64_t)D, BK, BM)) return RLF_ERR_CUDA;
        GemmParams z = g;
        set_rows(z, tc);
        if (bwd) {
            z.dz = dz;
            z.dz_nc = 4 * z.n_tiles;
            z.tmax = reinterpret_cast<float*>(ws + w.tmax);
        }
        z.live_count = counts;
        z.live_off = (int)t0;
        auto combine = [&](bool with_ref, const int* run_flag) {
            combine_rows_kernel<<<(unsigned)((tc + 255) / 256), 256, 0, s>>>(
                part, z.nsplit, (int)tc, idx_live, counts, (int)t0, zy, rec, dn, eps_clip, eps_hi, wtok, beta_kl, logp_out,
                lse_g, coef_g, y_g, dev_status, with_ref ? ref_g : nullptr, row_ref ? scale_g : nullptr, dz, z.dz_nc, V,
                chunk_flag, run_flag, 1);
            count_launch();
        };
        const int64_t tcp = (tc + 255) & ~(int64_t)255;
        auto dz_pass = [&](const int* run_flag) {
            const long long dz_items = (tcp / kDzBlockRows) * (long long)z.n_tiles;
            dz_from_e_kernel<false><<<(unsigned)(dz_items < 148 * 8 ? dz_items : 148 * 8), 256, 0, s>>>(
                dz, V, z.n_tiles, z.tmax, (int)tc, counts, (int)t0, lse_g, coef_g, y_g, idx_live, zy, nullptr, run_flag, 1);
            count_launch();
        };
        if (row_ref) {
            if (cudaMemsetAsync(chunk_flag, 0, sizeof(int), s) != cudaSuccess) return RLF_ERR_CUDA;
            z.ref = ref_g + t0;
            st = launch_gemm(mapHc, mapW, z, pair, s);
            if (st != RLF_OK) return st;
            combine(true, nullptr);
            // queued always, run only if some row of the chunk raised the flag: the chunk again with
            // per-tile maxima, rescaled in place into dZ (every row's factor becomes one)
            GemmParams zf = z;
            zf.ref = nullptr;
            zf.run_flag = chunk_flag;
            zf.run_want = 1;
            st = launch_gemm(mapHc, mapW, zf, pair, s);
            if (st != RLF_OK) return st;
            combine(false, chunk_flag);
            dz_pass(chunk_flag);
            scale_rows_kernel<<<(unsigned)tcp, 128, 0, s>>>(Hl + t0 * D, D, (int)tc, counts, (int)t0, scale_g, Hs);
            count_launch();
        } else {
            st = launch_gemm(mapHc, mapW, z, pair, s);
            if (st != RLF_OK) return st;
            combine(false, nullptr);
            if (!bwd) continue;
            dz_pass(nullptr);
        }
        // the scratch as the contractions see it: rows of 64 columns, 128 rows per block
        const uint64_t dz_rows = (uint64_t)(tcp / kDzBlockRows) * (uint64_t)(4 * z.n_tiles) * kDzBlockRows;
        if (cudaGetLastError() != cudaSuccess) return RLF_ERR_CUDA;
        if (grad_hidden) {
            // grad_hidden[token of gathered row] = (row factor) dZ[chunk, V] W[V, D]
            CUtensorMap mapDzK, mapWn;
            if (!make_map(&mapDzK, dz, dz_rows, kDzBlockCols, kDzBlockCols, BK, BM)) return RLF_ERR_CUDA;
            if (!make_map(&mapWn, Wm, (uint64_t)V, (uint64_t)D, (uint64_t)D, 64, BK)) return RLF_ERR_CUDA;
            GemmParams h = {};
            h.mode = kGradHidden;
            h.M = (int)tc;
            h.N = D;
            h.m_tiles = (int)((tc + BM - 1) / BM);
            h.n_tiles = (D + BN - 1) / BN;
            h.k_slabs = 4 * z.n_tiles;                     // every block of the scratch (zeros past the vocabulary)
            h.dz_nc = 4 * z.n_tiles;
            h.out_bf16 = static_cast<__nv_bfloat16*>(grad_hidden);
            h.out_stride = D;
            h.dev_status = dev_status;
            h.live_count = counts;
            h.live_off = (int)t0;
            h.row_index = idx_live;
            h.row_scale = row_ref ? scale_g + t0 : nullptr;
            h.pace = g.pace;
            st = launch_gemm(mapDzK, mapWn, h, pair, s);
            if (st != RLF_OK) return st;
        }
        if (grad_W) {
            // grad_W[V, D] (+)= dZ[chunk, V]^T hidden[chunk, D]  (hidden rows times their factors)
            CUtensorMap mapDzM, mapHn;
            if (!make_map(&mapDzM, dz, dz_rows, kDzBlockCols, kDzBlockCols, 64, BK)) return RLF_ERR_CUDA;
            if (!make_map(&mapHn, row_ref ? Hs : Hl + t0 * D, (uint64_t)tc, (uint64_t)D, (uint64_t)D, 64, BK))
                return RLF_ERR_CUDA;
            GemmParams q = {};
            q.mode = kGradW;
            q.M = V;
            q.N = D;
            q.m_tiles = (V + BM - 1) / BM;
            q.n_tiles = (D + BN - 1) / BN;
            q.k_slabs = (int)((tc + BK - 1) / BK);
            q.dz_nc = 4 * z.n_tiles;
            q.out_f32 = grad_W;
            q.out_stride = D;
            q.accumulate = (accumulate_grad_W || t0 > 0) ? 1 : 0;
            q.dev_status = dev_status;
            q.live_count = counts;
            q.live_off = (int)t0;
            q.pace = g.pace;
            st = launch_gemm(mapDzM, mapHn, q, pair, s);
            if (st != RLF_OK) return st;
        }
    }

    // the masked rows: log-prob only
    if (skip_masked) {
        fill_nan_rows_kernel<<<(unsigned)((T + 255) / 256), 256, 0, s>>>(idx_dead, counts + 1, logp_out);
        count_launch();
        if (cudaGetLastError() != cudaSuccess) return RLF_ERR_CUDA;
    } else {
        CUtensorMap mapHd;
        if (!make_map(&mapHd, Hd, (uint64_t)T, (uint64_t)D, (uint64_t)D, BK, BM)) return RLF_ERR_CUDA;
        GemmParams d = g;
        set_rows(d, T);
        d.live_count = counts + 1;
        d.live_off = 0;
        st = launch_gemm(mapHd, mapW, d, pair, s);
        if (st != RLF_OK) return st;
        combine_rows_kernel<<<(unsigned)((T + 255) / 256), 256, 0, s>>>(part, d.nsplit, (int)T, idx_dead, counts + 1, 0, zy,
                                                                         rec, dn, eps_clip, eps_hi, wtok, beta_kl, logp_out,
                                                                         nullptr, nullptr, nullptr, dev_status, nullptr,
                                                                         nullptr, nullptr, 0, V, nullptr, nullptr, 0);
        count_launch();
        if (cudaGetLastError() != cudaSuccess) return RLF_ERR_CUDA;
    }
    return token_loss(T);
}

}  // namespace lm
}  // namespace rlf

extern "C" rlf_status rlf_fused_lmhead_grpo(const void* hidden, const void* W, int64_t T, int32_t D, int32_t V,
                                            const int32_t* ids, const int32_t* seq_id, const float* adv, int32_t B,
                                            const float* old_logp, const float* ref_logp, const uint8_t* mask,
                                            float eps_clip, float beta_kl, const int64_t* denom, float* logp_out,
                                            double* loss_out, void* grad_hidden, float* grad_W,
                                            int accumulate_grad_W, void* workspace, size_t workspace_bytes,
                                            int32_t* dev_status, rlf_stream_t stream) {
    return rlf::lm::fused_lmhead_impl(hidden, W, T, D, V, ids, seq_id, adv, B, old_logp, ref_logp, mask, eps_clip,
                                      eps_clip, beta_kl, 0, 0, denom, logp_out, loss_out, grad_hidden, grad_W,
                                      accumulate_grad_W, workspace, workspace_bytes, dev_status, stream);
}

extern "C" rlf_status rlf_fused_lmhead_grpo_obj(const void* hidden, const void* W, int64_t T, int32_t D, int32_t V,
                                                const int32_t* ids, const int32_t* seq_id, const float* adv, int32_t B,
                                                const float* old_logp, const float* ref_logp, const uint8_t* mask,
                                                float eps_clip_low, float eps_clip_high, float beta_kl, int aggregation,
                                                int skip_masked, const int64_t* denom, float* logp_out,
                                                double* loss_out, void* grad_hidden, float* grad_W,
                                                int accumulate_grad_W, void* workspace, size_t workspace_bytes,
                                                int32_t* dev_status, rlf_stream_t stream) {
    if (skip_masked != 0 && skip_masked != 1) return RLF_ERR_SHAPE;
    return rlf::lm::fused_lmhead_impl(hidden, W, T, D, V, ids, seq_id, adv, B, old_logp, ref_logp, mask, eps_clip_low,
                                      eps_clip_high, beta_kl, aggregation, skip_masked, denom, logp_out, loss_out,
                                      grad_hidden, grad_W, accumulate_grad_W, workspace, workspace_bytes, dev_status,
                                      stream);
}


extern "C" rlf_status rlf_fused_lmhead_logp_entropy(const void* hidden, const void* W, int64_t T, int32_t D, int32_t V,
                                                    const int32_t* ids, float* logp_out, float* entropy_out,
                                                    void* workspace, size_t workspace_bytes, int32_t* dev_status,
                                                    rlf_stream_t stream) {
    using namespace rlf;
    using namespace rlf::lm;
    if (T < 0 || V < 1 || D < 1) return RLF_ERR_SHAPE;
    if (D % 64 != 0 || V % 8 != 0) return RLF_ERR_SHAPE;
    if (T >= (1ll << 30)) return RLF_ERR_UNSUPPORTED;
    if (T == 0) return RLF_OK;
    if (!hidden || !W || !ids || !logp_out) return RLF_ERR_NULL;
    if (!aligned(hidden, 16) || !aligned(W, 16)) return RLF_ERR_ALIGN;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < lmhead_logp_workspace_bytes(T))
        return RLF_ERR_WORKSPACE;
    rlf_status st = check_arch();
    if (st != RLF_OK) return st;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    char* ws = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(workspace) + 1023) & ~(uintptr_t)1023);
    float* zy = reinterpret_cast<float*>(ws);
    float2* part = reinterpret_cast<float2*>(ws + up1k(4 * (size_t)T));
    float* part_u = reinterpret_cast<float*>(ws + up1k(4 * (size_t)T) + up1k(8 * (size_t)T * kMaxSplit));
    const __nv_bfloat16* H = static_cast<const __nv_bfloat16*>(hidden);
    const __nv_bfloat16* Wm = static_cast<const __nv_bfloat16*>(W);
    target_logit_ids_kernel<<<(unsigned)((T + 7) / 8), 256, 0, s>>>(H, Wm, ids, T, D, V, zy, dev_status);
    count_launch();
    if (cudaGetLastError() != cudaSuccess) return RLF_ERR_CUDA;
    const bool pair = g_pair.load() != 0;
    CUtensorMap mapH, mapW;
    if (!make_map(&mapH, H, (uint64_t)T, (uint64_t)D, (uint64_t)D, BK, BM)) return RLF_ERR_CUDA;
    if (!make_map(&mapW, Wm, (uint64_t)V, (uint64_t)D, (uint64_t)D, BK, pair ? BN / 2 : BN)) return RLF_ERR_CUDA;
    GemmParams g = {};
    g.mode = kLse;
    g.M = (int)T;
    g.N = V;
    g.m_tiles = (int)((T + BM - 1) / BM);
    g.n_tiles = (V + BN - 1) / BN;
    g.k_slabs = D / BK;
    g.nsplit = pick_split(g.n_tiles);
    g.n_tiles_per_split = (g.n_tiles + g.nsplit - 1) / g.nsplit;
    g.part = part;
    g.part_u = entropy_out ? part_u : nullptr;
    g.dev_status = dev_status;
    // the pacing counter sits in the kilobyte that closes the workspace
    g.pace = reinterpret_cast<int*>(ws + up1k(4 * (size_t)T) + up1k(8 * (size_t)T * kMaxSplit) + up1k(4 * (size_t)T * kMaxSplit));
    st = launch_gemm(mapH, mapW, g, pair, s);
    if (st != RLF_OK) return st;
    combine_logp_entropy_kernel<<<(unsigned)((T + 255) / 256), 256, 0, s>>>(part, g.part_u, g.nsplit, zy, T, logp_out,
                                                                             entropy_out, dev_status);
    count_launch();
    return cuda_ok(cudaGetLastError());
}

// ---------------------------------------------------------------------------------------------
// Cross entropy through the fused head (the objective of rlf_cross_entropy_fwd_bwd).  Same sweeps and
// gradient contractions as above over the rows that carry loss, with, per row,
//   A_t = 1 + 2 zeta lse_t,   dZ_t = c A_t p_t - c eps / V - c (1 - eps) e_y,   c = 1 / N:
// the scratch holds e = exp(z - rho_t) with the target column overwritten, factor f_t = c A_t exp(rho_t - lse_t),
// and the uniform part -c eps / V never enters it: it is rank one, so with u = sum_v W_v
//   grad_hidden_t += a_t u,   grad_W_v += sum_t a_t h_t,   a_t = -c eps / V,
// two fp32 vectors of length D added in the contractions' epilogues; the mean logit is h_t . u / V.
//
// What bounds it, at the measured 1662 (burst) and 1399 TFLOP/s (under the power cap) and 6.56 TB/s:
//   8192 x 4096 x 151936, 4768 live rows: the tensor pipe; 3 x 2 T V D = 17.8 TFLOP in 12.4 ms at full clocks (1.44 PFLOP/s),
//     13.4 - 14.0 ms back to back (1.27 - 1.33);
//   2047 x 2048 x 32000, 1433 live rows: 614 - 680 us, 619 of them = 180 + 188 + 183 us of contractions at 1.0 PFLOP/s: six row tiles of 256 (93 %
//     filled) by 125 column tiles are 10.1 rounds of 74 pairs, so an eleventh round runs nearly empty, and each of the launches
//     fills and drains once; 65 us of small kernels, 32 of them the sum of W's rows for the smoothing;
//   64 x 2560 x 151936: 617 - 655 us.  Sweep 162 us (reads W at 4.8 TB/s, and writes 64 MB of exponentials for a tile of 256 rows),
//     grad_hidden 157 us (W again, and those), a bf16 grad_W 263 us: 714 MB at 2.7 TB/s, K is one slab, so that a unit is its drain and
//     a drain warp has two 4 KB tiles under way; 50 us of small kernels.  An fp32 grad_W leaves row by row from the registers,
//     1.5 GB in 830 us (1.8 TB/s): 1.2 ms in all.
namespace rlf {
namespace lm {

// Entry r of the work list.  A live row (r < n): its hidden row goes to compact row r, with its target logit, its mean logit
// (with u), the reference of its stored exponentials and its place in the output; the compact rows up to the next multiple of
// 256 are zero-filled.  A row without loss (n <= r < T): NaN statistics, no loss term, a zero row of grad_hidden.
__global__ void __launch_bounds__(128)
ce_gather_rows_kernel(const __nv_bfloat16* __restrict__ hidden, const __nv_bfloat16* __restrict__ W, int T, int D,
                      const int2* __restrict__ list, const int* __restrict__ count, const float* __restrict__ u,
                      float inv_v, __nv_bfloat16* __restrict__ out, int32_t* __restrict__ idx, float* __restrict__ zy_g,
                      float* __restrict__ mean_g, float* __restrict__ ref_g, float* __restrict__ logp_out,
                      float* __restrict__ lse_out, float4* __restrict__ terms, __nv_bfloat16* __restrict__ grad_hidden) {
    __shared__ float red[2][4];
    const int n = *count;
    const int r = blockIdx.x;
    const int nv = D / 8;
    if (r >= n) {
        const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
        if (r < ((n + 255) & ~255)) {
            for (int i = threadIdx.x; i < nv; i += 128) reinterpret_cast<uint4*>(out + (long long)r * D)[i] = zero;
            if (threadIdx.x == 0) ref_g[r] = 0.0f;
        }
        if (r >= T) return;
        const int t = list[r].x;
        if (threadIdx.x == 0) {
            const float nan = __int_as_float(0x7fc00000);
            logp_out[t] = nan;
            if (lse_out) lse_out[t] = nan;
            terms[t] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
        if (grad_hidden)
            for (int i = threadIdx.x; i < nv; i += 128) reinterpret_cast<uint4*>(grad_hidden + (long long)t * D)[i] = zero;
        return;
    }
    uint4* dst = reinterpret_cast<uint4*>(out + (long long)r * D);
    const int2 job = list[r];
    const uint4* src = reinterpret_cast<const uint4*>(hidden + (long long)job.x * D);
    const uint4* w = reinterpret_cast<const uint4*>(W + (long long)job.y * D);
    float a = 0.0f, b = 0.0f;
    for (int i = threadIdx.x; i < nv; i += 128) {
        const uint4 h = src[i], ww = w[i];
        dst[i] = h;
        const uint32_t hw[4] = {h.x, h.y, h.z, h.w}, wv[4] = {ww.x, ww.y, ww.z, ww.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float h0 = __uint_as_float(hw[k] << 16), h1 = __uint_as_float(hw[k] & 0xffff0000u);
            a = fmaf(h0, __uint_as_float(wv[k] << 16), a);
            a = fmaf(h1, __uint_as_float(wv[k] & 0xffff0000u), a);
            if (u) {
                b = fmaf(h0, u[8 * i + 2 * k], b);
                b = fmaf(h1, u[8 * i + 2 * k + 1], b);
            }
        }
    }
    a = warp_sum(a);
    b = warp_sum(b);
    if ((threadIdx.x & 31) == 0) {
        red[0][threadIdx.x >> 5] = a;
        red[1][threadIdx.x >> 5] = b;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        const float zy = (red[0][0] + red[0][1]) + (red[0][2] + red[0][3]);
        idx[r] = job.x;                    // (the gradient contraction's epilogue looks its output rows up here)
        zy_g[r] = zy;                      // (the sweep puts its own there)
        mean_g[r] = ((red[1][0] + red[1][1]) + (red[1][2] + red[1][3])) * inv_v;
        ref_g[r] = zy + kRefShift;
    }
}

constexpr int kCeSplit = 80;                // most vocabulary splits of a sweep (sizes the partials): one row unit on 74 pairs

struct CeCombine {
    const float2* part;
    int nsplit, rows_max;       // the partials' stride; the number of splits itself is found as the sweep found it:
    int n_tiles, fixed_split, rows_per_unit;
    Sched sched;
    const int2* list;
    const int* count;
    int off;
    const float* zy_g;          // target logit as the sweep has it
    const float* mean_g;
    const long long* denom;
    float eps, zeta, inv_v;
    float* logp_out;
    float* lse_out;
    float4* terms;
    int32_t* dev_status;
    // backward only
    float* lse_g;
    float* coef_g;              // c A_t
    float* tgt_g;               // dZ at the target column
    int32_t* ok_y;              // target id, -1 for a row without a gradient
    float* add_g;               // a_t
    float* scale_g;
    const float* ref_g;         // per-row references, or NULL: the scratch will hold dZ itself
    __nv_bfloat16* dz;
    int dz_nc;
    int* fallback;
    const int* run_flag;
    // grad_W wanted: the chunk's rows Hl times their factors go to Hs (zeros for a row that was taken out, whose hidden
    // state may hold anything, and up to the next multiple of 256 rows).  bf16, as the tensor cores take it: one rounding of grad_W's
    // terms besides the stored exponential's.  The factor is known only after the sweep, so that it could not go into the
    // exponentials without another pass over the scratch, which would round them once more all the same.
    const __nv_bfloat16* Hl;
    __nv_bfloat16* Hs;
    int D;
};
__device__ __forceinline__ void scale_row(const CeCombine& p, int r, float f, int lane) {
    if (!p.Hs) return;
    const uint4* src = reinterpret_cast<const uint4*>(p.Hl + (long long)r * p.D);
    uint4* dst = reinterpret_cast<uint4*>(p.Hs + (long long)r * p.D);
    for (int i = lane; i < p.D / 8; i += 32) {
        uint4 o = make_uint4(0u, 0u, 0u, 0u);
        if (f != 0.0f) {
            const uint4 z = src[i];
            const uint32_t w[4] = {z.x, z.y, z.z, z.w};
            uint32_t* q = reinterpret_cast<uint32_t*>(&o);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(q[k])
                    : "f"(__uint_as_float(w[k] & 0xffff0000u) * f), "f"(__uint_as_float(w[k] << 16) * f));
        }
        dst[i] = o;
    }
}
// As combine_rows_kernel: statistics, outputs and gradient factors of one chunk's rows.  Target logit and sums come from the
// same tensor-core products, whose errors (they round toward zero: a logit of 20 loses up to 1e-4 at D = 4096) then leave log p
// and 1 - p alone as p goes to one; with the target's logit from another sum, log p of such tokens came out above zero.  The target
// entry is formed as (expm1(logp) + 2 zeta lse p_y + eps) / A_t, which keeps its digits as p_y -> 1;
// with |A_t| below a half (a log-sum-exp near -1 / (2 zeta)) that quotient is not formed, the chunk is
// redone with dZ itself in the scratch.
// One warp per row, its lanes along the splits.
__global__ void __launch_bounds__(256)
ce_combine_rows_kernel(const CeCombine p) {
    if (p.run_flag && *p.run_flag != 1) return;
    const int r = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int n = max(0, min(*p.count - p.off, p.rows_max));
    if (r >= n) {
        if (r < ((n + 255) & ~255)) scale_row(p, r, 0.0f, lane);
        return;
    }
    const int m_units = (n + p.rows_per_unit - 1) / p.rows_per_unit;
    const int nsplit = m_units <= p.sched.auto_units ? auto_split(m_units, p.n_tiles, p.sched.workers, p.nsplit) : p.fixed_split;
    const int g = p.off + r;
    const int2 job = p.list[g];
    const int t = job.x;
    const float2* parts = p.part + (long long)r * p.nsplit;
    constexpr int kPer = (kCeSplit + 31) / 32;
    float2 q[kPer];
    float M = -INFINITY;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int k = lane + 32 * j;
        q[j] = k < nsplit ? parts[k] : make_float2(-INFINITY, 0.0f);
        M = fmaxf(M, q[j].x);
    }
    const float zy = p.zy_g[g];
    M = fmaxf(warp_max(M), zy);
    float others = 0.0f;                       // the sum over the other columns
#pragma unroll
    for (int j = 0; j < kPer; ++j)
        others += q[j].x == -INFINITY ? q[j].y : q[j].y * expf(q[j].x - M);      // (0 for a split of -inf, NaN where it held a NaN)
    others = warp_sum(others);
    if (p.ref_g) others = fmaf(others, offset_error(M), others);     // (M is the reference, below which the target lies)
    const float e_y = expf(zy - M), S = others + e_y, odds = others / e_y;
    // log p = -log(1 + odds) keeps its digits as p goes to one, where z_y - lse has none left
    const bool near = odds < 1e30f;
    const float logp = near ? -log1pf(odds) : (zy - M) - logf(S), lse = near ? zy - logp : M + logf(S);
    const float smooth = p.eps > 0.0f ? lse - p.mean_g[g] : 0.0f;
    const bool ok = (M > -INFINITY) && (M < INFINITY) && (S > 0.0f) && (S < INFINITY) && (fabsf(lse) < INFINITY) &&
                    (fabsf(logp) < INFINITY) && (fabsf(smooth) < INFINITY);
    const float A = 1.0f + 2.0f * p.zeta * lse;
    const long long N = *p.denom;
    const float c = 1.0f / (float)(N > 1 ? N : 1);
    const float rho = p.ref_g ? p.ref_g[g] : 0.0f;
    if (p.ref_g && !(ok && (lse - rho <= kRefWindow) && fabsf(A) >= 0.5f)) {
        if (lane == 0) atomicOr(p.fallback, 1);
        return;
    }
    // the row's factor (uniform over the warp)
    const float f = p.ref_g ? c * A * expf(rho - lse) : ok ? 1.0f : 0.0f;
    scale_row(p, r, f, lane);
    if (lane != 0) return;
    const float nan = __int_as_float(0x7fc00000);
    p.logp_out[t] = ok ? logp : nan;
    if (p.lse_out) p.lse_out[t] = ok ? lse : nan;
    p.terms[t] = ok ? make_float4(-logp, smooth, lse, 1.0f) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (!ok && p.dev_status) atomicOr(p.dev_status, RLF_DEV_NONFINITE);
    if (!p.scale_g) return;
    const float tgt = expm1f(logp) + fmaf(2.0f * p.zeta * lse, expf(logp), p.eps);
    p.add_g[g] = ok ? -c * p.eps * p.inv_v : 0.0f;
    p.scale_g[g] = f;
    if (p.ref_g) {
        p.dz[dz_offset(r, job.y, p.dz_nc)] = __float2bfloat16_rn(tgt / A * expf(lse - rho));
        return;
    }
    p.lse_g[g] = ok ? lse : 0.0f;
    p.coef_g[g] = ok ? c * A : 0.0f;
    p.tgt_g[g] = c * tgt;
    p.ok_y[g] = ok ? job.y : -1;
}

// joins the pieces of grad_hidden's long axis: row r (of *count - off) of the output, factors applied as in the contraction's
// epilogue.  Nothing to do where hidden_splits made one piece.
__global__ void __launch_bounds__(256)
ce_join_hidden_kernel(const float* __restrict__ part, long long part_floats, int D, const int* __restrict__ count, int off,
                      int rows_max, const int32_t* __restrict__ row_index, const float* __restrict__ row_scale,
                      const float* __restrict__ col_vec, const float* __restrict__ row_add, int rows_per_unit, int k_slabs,
                      int workers, int k_split_max, __nv_bfloat16* __restrict__ out) {
    const int n = max(0, min(*count - off, rows_max));
    const int r = blockIdx.x;
    const int units = (n + rows_per_unit - 1) / rows_per_unit * ((D + BN - 1) / BN);
    const int pieces = hidden_splits(units, k_slabs, workers, k_split_max, part_floats, n, D);
    if (r >= n || pieces == 1) return;
    const float sc = row_scale[r], ra = col_vec ? row_add[r] : 0.0f;
    __nv_bfloat16* o = out + (long long)row_index[off + r] * D;
    for (int c = 4 * threadIdx.x; c < D; c += 4 * blockDim.x) {
        float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
        for (int k = 0; sc != 0.0f && k < pieces; ++k) {       // (sc = 0: zeros, as in the epilogue)
            const float4 q = *reinterpret_cast<const float4*>(part + ((long long)k * n + r) * D + c);
            a.x += q.x; a.y += q.y; a.z += q.z; a.w += q.w;
        }
        a.x *= sc; a.y *= sc; a.z *= sc; a.w *= sc;
        if (col_vec && sc != 0.0f) {
            const float4 u = *reinterpret_cast<const float4*>(col_vec + c);
            a.x = fmaf(ra, u.x, a.x); a.y = fmaf(ra, u.y, a.y); a.z = fmaf(ra, u.z, a.z); a.w = fmaf(ra, u.w, a.w);
        }
        uint2 q;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(q.x) : "f"(a.y), "f"(a.x));
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(q.y) : "f"(a.w), "f"(a.z));
        *reinterpret_cast<uint2*>(o + c) = q;
    }
}

// out[d] = sum_r weight[r] M[r, d] (weight NULL: 1) over the rows r < rows (or *count - off, if given and less):
// CTA (x, y) covers 256 columns of slice y and leaves partial row y; rows of weight 0 are not looked at.
__global__ void __launch_bounds__(256)
colsum_kernel(const __nv_bfloat16* __restrict__ M, long long rows, int D, const float* __restrict__ weight,
              const int* __restrict__ count, int off, float* __restrict__ part) {
    __shared__ float red[8][256];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (count) rows = min(rows, (long long)max(0, *count - off));
    const int col = blockIdx.x * 256 + lane * 8;
    float acc[8] = {};
    if (col < D) {
        const long long step = (long long)gridDim.y * 8;
        auto add = [&](const uint4& v, float w) {
            const uint32_t q[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                acc[2 * k] = fmaf(w, __uint_as_float(q[k] << 16), acc[2 * k]);
                acc[2 * k + 1] = fmaf(w, __uint_as_float(q[k] & 0xffff0000u), acc[2 * k + 1]);
            }
        };
        long long r = (long long)blockIdx.y * 8 + warp;
        for (; r + 3 * step < rows; r += 4 * step) {       // four loads in flight
            uint4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = *reinterpret_cast<const uint4*>(M + (r + k * step) * D + col);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float w = weight ? weight[r + k * step] : 1.0f;
                if (w != 0.0f) add(v[k], w);
            }
        }
        for (; r < rows; r += step) {
            const float w = weight ? weight[r] : 1.0f;
            if (w != 0.0f) add(*reinterpret_cast<const uint4*>(M + r * D + col), w);
        }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) red[warp][lane * 8 + k] = acc[k];
    __syncthreads();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c < D) {
        float s = 0.0f;
        for (int w = 0; w < 8; ++w) s += red[w][threadIdx.x];
        part[(long long)blockIdx.y * D + c] = s;
    }
}
__global__ void __launch_bounds__(256)
colsum_reduce_kernel(const float* __restrict__ part, int parts, int D, float* __restrict__ out) {
    __shared__ float acc[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (col < D)
        for (int k = warp; k < parts; k += 8) s += part[(long long)k * D + col];
    acc[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && col < D) {
        for (int w = 1; w < 8; ++w) s += acc[w][lane];
        out[col] = s;
    }
}
constexpr int kColsumParts = 128;
static rlf_status launch_colsum(const __nv_bfloat16* M, int64_t rows, int32_t D, const float* weight, const int* count,
                                int off, float* part, float* out, cudaStream_t s) {
    const int64_t want = (rows + 63) / 64;
    const int parts = (int)(want < kColsumParts ? (want > 0 ? want : 1) : kColsumParts);
    colsum_kernel<<<dim3((unsigned)((D + 255) / 256), (unsigned)parts), 256, 0, s>>>(M, rows, D, weight, count, off, part);
    colsum_reduce_kernel<<<(unsigned)((D + 31) / 32), 256, 0, s>>>(part, parts, D, out);
    count_launch(2);
    return cuda_ok(cudaGetLastError());
}

// Most pieces of grad_hidden's long axis: what it has slabs for, and a gigabyte of fp32 rows holds.
static int hidden_pieces(int64_t T, int32_t V, int32_t D) {
    int64_t rows = ((T > 0 ? T : 1) + 255) & ~(int64_t)255;
    if (rows > kChunkTokens) rows = kChunkTokens;
    int64_t k = (256ll << 20) / (rows * D);
    const int64_t slabs = 4ll * ((V + BN - 1) / BN);
    if (k > slabs / kSlabsPerPiece) k = slabs / kSlabsPerPiece;
    return (int)(k < 1 ? 1 : k > 64 ? 64 : k);
}
// Floats that their raw sums take at most: over every number of live rows, the pieces that hidden_splits would make of them in
// any form of the contraction (units of 512 or 256 rows on pairs of SMs, of 128 on single ones).
static size_t hidden_part_floats(int64_t T, int32_t V, int32_t D) {
    const int most = hidden_pieces(T, V, D);
    if (most < 2) return 0;
    const int64_t rows = T < kChunkTokens ? T : kChunkTokens;
    const int slabs = 4 * ((V + BN - 1) / BN), n_tiles = (D + BN - 1) / BN, sms = sm_count_lm();
    size_t need = 0;
    for (int unit_rows = 128; unit_rows <= 512; unit_rows *= 2) {
        const int64_t m_units = (rows + unit_rows - 1) / unit_rows;
        const int64_t all = m_units * n_tiles * most;
        int workers = unit_rows == 128 ? sms : sms / 2;
        if (workers > all) workers = (int)all;
        for (int64_t m = 1; m <= m_units; ++m) {
            unsigned best = 0xffffffffu;
            for (int k = 1; k <= most; ++k) {
                const unsigned cost = hidden_cost((int)(m * n_tiles), slabs, workers, k);
                best = best < cost ? best : cost;
            }
            const int64_t live = m * unit_rows < rows ? m * unit_rows : rows;
            const size_t floats = (best & 127u) > 1 ? (size_t)(best & 127u) * (size_t)live * (size_t)D : 0;
            need = need > floats ? need : floats;
        }
    }
    return need;
}
struct CeWs {
    size_t head, terms, list, zy, mean, part, idx_live, ok_y, lse_g, coef_g, tgt_g, add_g, ref_g, scale_g, ucol,
        gcol, col_part, hidden_g, hidden_s, tmax, gw_acc, k_part, dz, total;
};
// grads: false for a forward-only call, which keeps no scratch
static CeWs ce_workspace(int64_t T, int32_t V, int32_t D, bool w16, bool grads) {
    CeWs w = {};
    size_t o = 0;
    const size_t Tn = (size_t)(T > 0 ? T : 0), Tp = (Tn + 255) & ~(size_t)255, Dn = (size_t)D;
    const size_t chunk = Tp < (size_t)kChunkTokens ? Tp : (size_t)kChunkTokens;
    const size_t tiles = (size_t)((V + BN - 1) / BN);
    auto take = [&](size_t bytes) { const size_t at = o; o += up1k(bytes); return at; };
    w.head = take(1024);             // [0] mask count, [64] live rows, [128] chunk flag and pacing counters
    w.terms = take(16 * Tn);
    w.list = take(8 * Tn);
    w.zy = take(4 * Tp);
    w.mean = take(4 * Tp);
    w.part = take(8 * Tn * kCeSplit);
    w.idx_live = take(4 * Tp);
    w.ref_g = take(4 * Tp);
    w.ucol = take(4 * Dn);
    w.col_part = take(4 * Dn * kColsumParts);
    w.hidden_g = take(2 * Tp * Dn);
    if (grads) {
        w.ok_y = take(4 * Tp);
        w.lse_g = take(4 * Tp);
        w.coef_g = take(4 * Tp);
        w.tgt_g = take(4 * Tp);
        w.add_g = take(4 * Tp);
        w.scale_g = take(4 * Tp);
        w.gcol = take(4 * Dn);
        w.hidden_s = take(2 * chunk * Dn);
        w.tmax = take(4 * chunk * tiles);
        // fp32 sum of grad_W over the chunks of a call whose result is bf16
        w.gw_acc = take(w16 && Tn > (size_t)kChunkTokens ? 4 * (size_t)V * Dn : 0);
        w.k_part = take(4 * hidden_part_floats(T, V, D));
        w.dz = take(2 * chunk * tiles * BN);
    }
    w.total = o + 1024;
    return w;
}

}  // namespace lm

size_t lmhead_ce_workspace_bytes(int64_t T, int32_t V, int32_t D, bool grad_w_bf16, bool grads) {
    if (V < 1 || D < 1) return 0;
    return lm::ce_workspace(T, V, D, grad_w_bf16, grads).total;
}

}  // namespace rlf

extern "C" rlf_status rlf_fused_lmhead_cross_entropy(const void* hidden, const void* W, int64_t T, int32_t D, int32_t V,
                                                     const int32_t* ids, const uint8_t* mask, float label_smoothing,
                                                     float z_coef, const int64_t* denom, float* logp_out, float* lse_out,
                                                     double* loss_out, void* grad_hidden, void* grad_W, rlf_dtype grad_W_dt,
                                                     int accumulate_grad_W, void* workspace, size_t workspace_bytes,
                                                     int32_t* dev_status, rlf_stream_t stream) {
    using namespace rlf;
    using namespace rlf::lm;
    if (grad_W_dt != RLF_BF16 && grad_W_dt != RLF_F32) return RLF_ERR_DTYPE;
    if (T < 0 || V < 1 || D < 1) return RLF_ERR_SHAPE;
    if (D % 64 != 0 || V % 8 != 0) return RLF_ERR_SHAPE;
    rlf_status st = ce_check_objective(label_smoothing, z_coef);
    if (st != RLF_OK) return st;
    const bool w16 = grad_W && grad_W_dt == RLF_BF16;
    if (T >= (1ll << 30) || V >= (1 << 30) || D >= (1 << 30) || (w16 && accumulate_grad_W)) return RLF_ERR_UNSUPPORTED;
    if (!loss_out) return RLF_ERR_NULL;
    if (T > 0 && (!hidden || !W || !ids || !logp_out)) return RLF_ERR_NULL;
    if (!aligned(hidden, 16) || !aligned(W, 16) || !aligned(grad_hidden, 16) || !aligned(grad_W, 16) || !aligned(ids, 4) ||
        !aligned(logp_out, 4) || !aligned(lse_out, 4) || !aligned(loss_out, 8) || !aligned(denom, 8))
        return RLF_ERR_ALIGN;
    const bool bwd = grad_hidden || grad_W;
    const CeWs w = ce_workspace(T, V, D, w16, bwd);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < w.total) return RLF_ERR_WORKSPACE;
    st = check_arch();
    if (st != RLF_OK) return st;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    char* ws = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(workspace) + 1023) & ~(uintptr_t)1023);
    auto at = [&](size_t off) { return reinterpret_cast<float*>(ws + off); };
    long long* n_mask = reinterpret_cast<long long*>(ws + w.head);
    int* counts = reinterpret_cast<int*>(ws + w.head + 64);
    int* chunk_flag = reinterpret_cast<int*>(ws + w.head + 128);
    constexpr int kFlagWords = 8;                // [0] the chunk's flag, [4 ..] four meeting counters
    int* pace = chunk_flag + 4;
    const long long* dn = denom ? reinterpret_cast<const long long*>(denom) : n_mask;
    float4* terms = reinterpret_cast<float4*>(ws + w.terms);
    const __nv_bfloat16* H = static_cast<const __nv_bfloat16*>(hidden);
    const __nv_bfloat16* Wm = static_cast<const __nv_bfloat16*>(W);
    if (T == 0) {
        // no rows: a zero loss, and a gradient of zero unless it is accumulated
        if (!denom) {
            st = ce_launch_plan(nullptr, nullptr, 0, V, nullptr, counts, n_mask, nullptr, 0, dev_status, s);
            if (st != RLF_OK) return st;
        }
        if (grad_W && !accumulate_grad_W &&
            cudaMemsetAsync(grad_W, 0, (size_t)V * D * (w16 ? 2 : 4), s) != cudaSuccess)
            return RLF_ERR_CUDA;
        return ce_launch_loss(terms, 0, dn, label_smoothing, z_coef, loss_out, s);
    }

    int32_t* idx_live = reinterpret_cast<int32_t*>(ws + w.idx_live);
    int2* list = reinterpret_cast<int2*>(ws + w.list);
    __nv_bfloat16* Hl = reinterpret_cast<__nv_bfloat16*>(ws + w.hidden_g);
    __nv_bfloat16* Hs = reinterpret_cast<__nv_bfloat16*>(ws + w.hidden_s);
    __nv_bfloat16* dz = reinterpret_cast<__nv_bfloat16*>(ws + w.dz);
    const int64_t Tp = (T + 255) & ~(int64_t)255;
    const bool smoothing = label_smoothing > 0.0f;
    const bool row_ref = bwd && g_row_ref.load() != 0;
    float* ucol = smoothing ? at(w.ucol) : nullptr;
    st = ce_launch_plan(ids, mask, T, V, list, counts, n_mask, chunk_flag, kFlagWords, dev_status, s);
    if (st != RLF_OK) return st;
    if (smoothing) {
        st = launch_colsum(Wm, V, D, nullptr, nullptr, 0, at(w.col_part), ucol, s);
        if (st != RLF_OK) return st;
    }
    const float inv_v = 1.0f / (float)V;
    ce_gather_rows_kernel<<<(unsigned)Tp, 128, 0, s>>>(H, Wm, (int)T, D, list, counts, ucol, inv_v, Hl, idx_live, at(w.zy),
                                                       at(w.mean), at(w.ref_g), logp_out, lse_out, terms,
                                                       static_cast<__nv_bfloat16*>(grad_hidden));
    count_launch();
    if (cudaGetLastError() != cudaSuccess) return RLF_ERR_CUDA;

    const bool pair = g_pair.load() != 0;
    CUtensorMap mapW;
    if (!make_map(&mapW, Wm, (uint64_t)V, (uint64_t)D, (uint64_t)D, BK, pair ? BN / 2 : BN)) return RLF_ERR_CUDA;
    // (a bf16 grad_W of a call that fits one built-in chunk is not cut further: its workspace holds no fp32 sum)
    const int tuned_tiles = g_chunk_tiles.load();
    const bool tuned = tuned_tiles > 0 && tuned_tiles * BM < kChunkTokens && !(w16 && T <= kChunkTokens);
    const int64_t chunk_tokens = tuned ? tuned_tiles * BM : kChunkTokens;
    for (int64_t t0 = 0; t0 < T; t0 += chunk_tokens) {
        const int64_t tc = (T - t0) < chunk_tokens ? (T - t0) : chunk_tokens;
        const int64_t tcp = (tc + 255) & ~(int64_t)255;
        CUtensorMap mapHc;
        if (!make_map(&mapHc, Hl + t0 * D, (uint64_t)tc, (uint64_t)D, (uint64_t)D, BK, BM)) return RLF_ERR_CUDA;
        GemmParams z = {};
        z.mode = kLse;
        z.N = V;
        z.n_tiles = (V + BN - 1) / BN;
        z.k_slabs = D / BK;
        z.M = (int)tc;
        z.m_tiles = (int)((tc + BM - 1) / BM);
        // the sweep chooses its splits itself where the live rows' tiles stay in L2 (auto_split)
        z.auto_units = 1;                      // (set to their number by the launch)
        z.nsplit = kCeSplit < z.n_tiles ? kCeSplit : z.n_tiles;
        z.fixed_split = pick_split(z.n_tiles);
        z.n_tiles_per_split = (z.n_tiles + z.nsplit - 1) / z.nsplit;
        z.part = reinterpret_cast<float2*>(ws + w.part);
        z.dev_status = dev_status;
        // the chunk's flag and its launches' meeting counters, zeroed by the plan kernel or, from the second chunk on, here
        if (t0 > 0 && cudaMemsetAsync(chunk_flag, 0, kFlagWords * sizeof(int), s) != cudaSuccess) return RLF_ERR_CUDA;
        z.pace = pace;
        z.pace_is_zero = 1;
        z.live_count = counts;
        z.live_off = (int)t0;
        z.target = list + t0;
        z.target_logit = at(w.zy) + t0;
        if (bwd) {
            z.dz = dz;
            z.dz_nc = 4 * z.n_tiles;
            z.tmax = at(w.tmax);
        }
        CeCombine c = {};
        c.part = z.part; c.nsplit = z.nsplit; c.rows_max = (int)tc; c.list = list; c.count = counts;
        c.off = (int)t0; c.zy_g = at(w.zy); c.mean_g = at(w.mean); c.denom = dn; c.eps = label_smoothing; c.zeta = z_coef;
        c.inv_v = inv_v; c.n_tiles = z.n_tiles; c.fixed_split = z.fixed_split; c.rows_per_unit = (pair ? 2 : 1) * BM; c.logp_out = logp_out; c.lse_out = lse_out; c.terms = terms; c.dev_status = dev_status;
        if (bwd) {
            c.lse_g = at(w.lse_g); c.coef_g = at(w.coef_g); c.tgt_g = at(w.tgt_g);
            c.ok_y = reinterpret_cast<int32_t*>(ws + w.ok_y); c.add_g = at(w.add_g); c.scale_g = at(w.scale_g);
            c.dz = dz; c.dz_nc = z.dz_nc;
        }
        if (grad_W) {
            c.Hl = Hl + t0 * D;
            c.Hs = Hs;
            c.D = D;
        }
        const unsigned row_blocks = (unsigned)(tcp / 8);             // a warp per row, whole multiples of 256 rows
        if (row_ref) {
            z.ref = at(w.ref_g) + t0;
            st = launch_gemm(mapHc, mapW, z, pair, s, &c.sched);
            if (st != RLF_OK) return st;
            CeCombine cr = c;
            cr.ref_g = at(w.ref_g);
            cr.fallback = chunk_flag;
            ce_combine_rows_kernel<<<row_blocks, 256, 0, s>>>(cr);
            count_launch();
            // queued always, run only if some row of the chunk raised the flag
            z.ref = nullptr;
            z.run_flag = chunk_flag;
            z.run_want = 1;
            c.run_flag = chunk_flag;
            z.pace = pace + 1;
        }
        st = launch_gemm(mapHc, mapW, z, pair, s, &c.sched);
        if (st != RLF_OK) return st;
        ce_combine_rows_kernel<<<row_blocks, 256, 0, s>>>(c);
        count_launch();
        if (cudaGetLastError() != cudaSuccess) return RLF_ERR_CUDA;
        if (!bwd) continue;
        const long long dz_items = (tcp / kDzBlockRows) * (long long)z.n_tiles;
        dz_from_e_kernel<true><<<(unsigned)(dz_items < 148 * 8 ? dz_items : 148 * 8), 256, 0, s>>>(
            dz, V, z.n_tiles, z.tmax, (int)tc, counts, (int)t0, c.lse_g, c.coef_g, c.ok_y, nullptr, nullptr, c.tgt_g,
            z.run_flag, 1);
        count_launch();
        const uint64_t dz_rows = (uint64_t)(tcp / kDzBlockRows) * (uint64_t)(4 * z.n_tiles) * kDzBlockRows;
        if (grad_hidden) {
            CUtensorMap mapDzK, mapWn;
            if (!make_map(&mapDzK, dz, dz_rows, kDzBlockCols, kDzBlockCols, BK, BM)) return RLF_ERR_CUDA;
            if (!make_map(&mapWn, Wm, (uint64_t)V, (uint64_t)D, (uint64_t)D, 64, BK)) return RLF_ERR_CUDA;
            GemmParams h = {};
            h.mode = kGradHidden;
            h.M = (int)tc;
            h.N = D;
            h.m_tiles = (int)((tc + BM - 1) / BM);
            h.n_tiles = (D + BN - 1) / BN;
            h.k_slabs = 4 * z.n_tiles;
            h.dz_nc = z.dz_nc;
            h.out_bf16 = static_cast<__nv_bfloat16*>(grad_hidden);
            h.out_stride = D;
            h.dev_status = dev_status;
            h.live_count = counts;
            h.live_off = (int)t0;
            h.row_index = idx_live;
            h.row_scale = c.scale_g + t0;      // 1 without the reference, 0 for a row that was taken out
            h.col_vec = ucol;
            h.row_add = c.add_g + t0;
            h.k_part_floats = (long long)((w.dz - w.k_part) / sizeof(float));
            h.k_split_max = h.k_part_floats > 0 ? hidden_pieces(T, V, D) : 1;
            h.k_part = at(w.k_part);
            h.pace = pace + 2;
            h.pace_is_zero = 1;
            // up to 256 rows fill one pair's accumulator: the second one would multiply nothing
            const bool acc2 = g_acc2.load() != 0 && tc > 2 * BM;
            Sched sched;
            st = launch_gemm_ce(mapDzK, mapWn, mapDzK, h, pair, acc2, s, &sched);
            if (st != RLF_OK) return st;
            if (h.k_split_max > 1) {
                ce_join_hidden_kernel<<<(unsigned)tc, 256, 0, s>>>(
                    h.k_part, h.k_part_floats, D, counts, (int)t0, (int)tc, idx_live, h.row_scale, ucol, h.row_add,
                    (pair ? 2 : 1) * (pair && acc2 ? 2 : 1) * BM, h.k_slabs, sched.workers, h.k_split_max, h.out_bf16);
                count_launch();
            }
        }
        if (grad_W) {
            if (smoothing) {
                st = launch_colsum(Hl + t0 * D, tc, D, c.add_g + t0, counts, (int)t0, at(w.col_part), at(w.gcol), s);
                if (st != RLF_OK) return st;
            }
            CUtensorMap mapDzM, mapHn;
            if (!make_map(&mapDzM, dz, dz_rows, kDzBlockCols, kDzBlockCols, 64, BK)) return RLF_ERR_CUDA;
            if (!make_map(&mapHn, Hs, (uint64_t)tc, (uint64_t)D, (uint64_t)D, 64, BK)) return RLF_ERR_CUDA;
            const bool last = t0 + chunk_tokens >= T;
            GemmParams q = {};
            q.mode = kGradW;
            q.M = V;
            q.N = D;
            q.m_tiles = (V + BM - 1) / BM;
            q.n_tiles = (D + BN - 1) / BN;
            q.k_slabs = (int)((tc + BK - 1) / BK);
            q.dz_nc = z.dz_nc;
            q.out_f32 = w16 ? at(w.gw_acc) : static_cast<float*>(grad_W);
            q.out_stride = D;
            q.accumulate = (accumulate_grad_W || t0 > 0) ? 1 : 0;
            CUtensorMap mapGw = mapDzM;
            if (w16 && last) {                 // bf16 result: rounded once, from the sum over the chunks
                if (!make_map(&mapGw, grad_W, (uint64_t)V, (uint64_t)D, (uint64_t)D, 64, 32)) return RLF_ERR_CUDA;
                q.store_w16 = 1;
                q.add_f32 = t0 > 0 ? at(w.gw_acc) : nullptr;
                q.accumulate = 0;
            }
            q.dev_status = dev_status;
            q.live_count = counts;
            q.live_off = (int)t0;
            q.col_vec = smoothing ? at(w.gcol) : nullptr;
            q.pace_is_zero = 1;
            q.pace = tc > 512 ? pace + 3 : nullptr;      // (few tokens: a unit is shorter than a meeting)
            // (129 to 512 tokens: a unit is mostly drain, which the form with one accumulator per unit overlaps with the next
            // unit: 512 x 2560 x 151936 1.05 ms in all against 1.12; up to 128 the drain is all there is, 637 - 674 us either way)
            st = launch_gemm_ce(mapDzM, mapHn, mapGw, q, pair, g_acc2.load() != 0 && !(tc > 2 * BK && tc <= 8 * BK), s);
            if (st != RLF_OK) return st;
        }
    }
    return ce_launch_loss(terms, T, dn, label_smoothing, z_coef, loss_out, s);
}

extern "C" rlf_status rlf_tune_lmhead(int pair_ctas) {
    if (pair_ctas != 0 && pair_ctas != 1) return RLF_ERR_SHAPE;
    rlf::lm::g_pair = pair_ctas;
    return RLF_OK;
}

extern "C" rlf_status rlf_tune_lmhead_backward(int row_reference, int two_accumulators) {
    if ((row_reference != 0 && row_reference != 1) || (two_accumulators != 0 && two_accumulators != 1)) return RLF_ERR_SHAPE;
    rlf::lm::g_row_ref = row_reference;
    rlf::lm::g_acc2 = two_accumulators;
    return RLF_OK;
}

extern "C" rlf_status rlf_tune_lmhead_pacing(int on) {
    if (on != 0 && on != 1) return RLF_ERR_SHAPE;
    rlf::lm::g_pace = on;
    return RLF_OK;
}

extern "C" rlf_status rlf_tune_lmhead_schedule(int m_block, int max_workers, int chunk_tiles) {
    if (m_block < 0 || m_block > (1 << 20) || max_workers < 0 || chunk_tiles < 0 || (chunk_tiles & 1)) return RLF_ERR_SHAPE;
    rlf::lm::g_m_block = m_block;
    rlf::lm::g_max_workers = max_workers;
    rlf::lm::g_chunk_tiles = chunk_tiles;
    return RLF_OK;
}
