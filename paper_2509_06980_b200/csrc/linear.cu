// Linear layer, forward and backward:
//
//   z = x W^T + b;   y = act(z) (+ residual),   or gated, with W's rows in two halves:  y = act(z_gate) z_up (+ residual)
//   gz = dy act'(z)  (gated: dy z_up act'(z_gate) and dy act(z_gate));   dx = gz W;   dW = gz^T x;   db = sum_t gz
//
// All three products are out[m][n] = sum_k A[m][k] B[n][k] on bf16 operands with fp32 accumulation in tensor memory:
//   y:  A = x,    B = W     (both K-major)
//   dx: A = gz,   B = W^T   (W is stored with n running along its rows: an N-major operand)
//   dW: A = gz^T, B = x^T   (both M-/N-major: the tokens, which are summed over, are the rows)
// and one epilogue serves them: out = act(acc + bias) + residual (accumulation into dW is a residual that is the output itself).
// Two kernels share it:
//   pair    large products: a persistent pair of CTAs multiplies 256 x 256 tiles (tcgen05 cta_group::2), bound by the tensor cores (32768 x
//           10240 x 2560 1.1 ms for a single call, 1.2 - 1.4 one after the other: 0.90 - 0.95 of the rate that the power cap sustains) or,
//           where k is short, by draining the results;
//           one launch takes one product or both of a backward pass;
//   narrow  few rows (decoding, short batches) or few tiles: the operand with the output's columns is streamed in 128-row tiles
//           as the M side of the multiplies, the few rows are their N side, and K is cut over a cluster whose CTAs add up their
//           accumulators through distributed shared memory.  Bound by reading the streamed operand (8 x 2560 x 10240, 52 MB: 12 - 13 us;
//           gated, 105 MB: 21 us; 8 x 4096 x 12288 gated, 201 MB: 34 - 36 us, 5.6 - 5.9 TB/s).
// An output of at most four columns (the values of a critic, a few reward scores) takes no tensor cores: it is bound by
// reading x, and its sums are plain fp32 ones (8191 x 4096 x 1, 67 MB: 14.6 - 15.1 us, 4.6 TB/s; backward, 134 MB: 26 on the GPU, 29 - 30 a
// call).  A gated layer of one or two outputs is no such head: it takes the products above.
#include <atomic>

#include "row.cuh"
#include "umma.cuh"

namespace rlf {
namespace ln {

using tc::instr_desc;
using tc::kSlabBytes;
using tc::make_map;
using tc::map_to_cta;
using tc::mbar_arrive_cluster;
using tc::mbar_expect_tx;
using tc::pair_rank;
using tc::smem_addr;
using tc::smem_desc;
using tc::tc_commit;
using tc::tc_commit2;
using tc::tc_fence_after;
using tc::tc_fence_before;
using tc::tc_ld32;
using tc::tc_ld32_issue;
using tc::tc_ld_wait;
using tc::tc_mma;
using tc::tc_mma2;
using tc::tma_load_2d;
using tc::tma_load_2d_pair;

constexpr int kFewOutputs = 4;

// Bounded wait for a phase of an mbarrier that may take long: every try suspends the thread for up to 10 us.  (Short tries by the
// waiting warps were four fifths of the instructions of a large product, and at the power cap they cost clock.)
__device__ __forceinline__ bool long_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
    if (mbar_try_wait(bar, parity)) return true;
    for (int i = 0; i < (1 << 20); ++i) {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(ok) : "r"(bar), "r"(parity), "r"(10000u) : "memory");
        if (ok) return true;
        if ((i & 63) == 63 && *abort_flag) return false;
    }
    *abort_flag = 1;
    return false;
}

// One lane of a warp.  The issuing warps run their loops as a whole and elect a lane for the copies and multiplies only: with warp-uniform
// loops the operands of those instructions are formed in uniform registers.  As a single thread's loop a 64-deep slab took 580
// clocks to issue, whatever its width, where a 256 x 256 one is multiplied in 512.
__device__ __forceinline__ bool elect_one() {
    uint32_t yes;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
    return yes != 0;
}
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }

// Launches of this file follow one another without a gap (programmatic dependent launch): a kernel may be set up while the one before
// it still runs.  Each lets its successor start at once (once it has its tensor memory: a successor on the same SM that took
// it first would wait for this kernel's end while this one waited for the memory), and reads and writes memory only after
// pdl_wait, that is when everything before it in the stream has finished.
__device__ __forceinline__ void pdl_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// What becomes of an accumulator: out[row][col] = act(acc + bias[col]) (times the up half, when gated) + res[row][col].
struct Epilogue {
    int act, gated;
    int N;                          // output columns
    const void* bias;               // [N], gated [2 N]; nullable
    int bias_bf16;
    const void* res;                // rows of the output's type; nullable
    long long res_stride;
    void* out;
    long long out_stride;
    int out_f32;
    __nv_bfloat16* pre;             // acc + bias as bf16, [rows][N], gated [rows][2 N]; nullable
    long long pre_stride;
    int vec_out, vec_res, vec_pre;  // rows of out, res and pre lie on 16-byte boundaries
};

// ---- activations ------------------------------------------------------------------------------
__device__ __forceinline__ float rcp_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 1 / (1 + e^-x); an e^-x beyond fp32 gives 0
__device__ __forceinline__ float sigmoid(float x) { return rcp_approx(1.0f + ex2_approx(-kLog2e * x)); }
// Standard normal distribution and e^(-z^2/2).  With t = 1 / (1 + 0.43 |z| / sqrt 2), erfc(x) e^(x^2) is a smooth function of t; the
// polynomial is its least relative deviation of degree 8 over x in [0, 10] (1e-7, in fp32 arithmetic 2.6e-7), fitted for this purpose.
// (The library's normal distribution took four times the instructions: 2048 x 1024 x 4096 with GELU 46 us, so 26.)
__device__ __forceinline__ float normal_cdf(float z, float& e) {
    const float t = rcp_approx(fmaf(0.43f * 0.70710678f, fabsf(z), 1.0f));
    e = ex2_approx(-0.5f * kLog2e * z * z);
    float g = 0.036572903f;
    g = fmaf(g, t, -0.15404779f);
    g = fmaf(g, t, 0.1899436f);
    g = fmaf(g, t, -0.041152104f);
    g = fmaf(g, t, 0.12254031f);
    g = fmaf(g, t, 0.102736264f);
    g = fmaf(g, t, 0.12214691f);
    g = fmaf(g, t, 0.12125991f);
    const float tail = g * t * e;
    return z < 0.0f ? tail : 1.0f - tail;
}
constexpr float kGeluRoot = 0.7978845608028654f, kGeluCube = 0.044715f, kInvSqrt2Pi = 0.3989422804014327f;

// (the tanh form: 0.5 (1 + tanh u) = sigmoid(2 u))
template <int ACT> __device__ __forceinline__ float act_value(float z) {
    if (ACT == RLF_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if (ACT == RLF_ACT_SILU) return z * sigmoid(z);
    if (ACT == RLF_ACT_GELU) {
        float e;
        return z * normal_cdf(z, e);
    }
    if (ACT == RLF_ACT_GELU_TANH) return z * sigmoid(2.0f * kGeluRoot * z * fmaf(kGeluCube * z, z, 1.0f));
    return z;
}
template <int ACT> __device__ __forceinline__ float act_slope(float z) {
    if (ACT == RLF_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if (ACT == RLF_ACT_SILU) {
        const float s = sigmoid(z);
        return s * fmaf(z, 1.0f - s, 1.0f);
    }
    if (ACT == RLF_ACT_GELU) {
        float e;
        const float c = normal_cdf(z, e);
        return fmaf(z * kInvSqrt2Pi, e, c);
    }
    if (ACT == RLF_ACT_GELU_TANH) {
        const float s = sigmoid(2.0f * kGeluRoot * z * fmaf(kGeluCube * z, z, 1.0f));
        // (s (1 - s) is zero long before |z| = 100; z^2 that overflows would make its product NaN)
        return s + z * s * (1.0f - s) * 2.0f * kGeluRoot * fmaf(3.0f * kGeluCube, fminf(z * z, 1e4f), 1.0f);
    }
    return 1.0f;
}
// The same on two values at a time: packed arithmetic leaves the epilogue to the exponentials and reciprocals (two a value), which
// are then what bounds it.
__device__ __forceinline__ f2 f2_each(f2 v, float (*f)(float)) {
    float a, b;
    f2_split(v, a, b);
    return f2_make(f(a), f(b));
}
__device__ __forceinline__ f2 f2_of(float v) { return f2_make(v, v); }
__device__ __forceinline__ f2 sigmoid2(f2 minus_log2e_x) {      // of x, given -x log2 e
    const f2 e = f2_each(minus_log2e_x, ex2_approx);
    return f2_each(f2_add(e, f2_of(1.0f)), rcp_approx);
}
template <int ACT> __device__ __forceinline__ f2 act_value2(f2 z) {
    if (ACT == RLF_ACT_SILU) return f2_mul(z, sigmoid2(f2_mul(z, f2_of(-kLog2e))));
    if (ACT == RLF_ACT_GELU_TANH) {
        const f2 u = f2_mul(z, f2_of(-2.0f * kGeluRoot * kLog2e));
        return f2_mul(z, sigmoid2(f2_mul(u, f2_fma(f2_mul(z, f2_of(kGeluCube)), z, f2_of(1.0f)))));
    }
    if (ACT == RLF_ACT_GELU) {
        float a, b, p, q;
        f2_split(z, a, b);
        const f2 t = f2_each(f2_fma(f2_make(fabsf(a), fabsf(b)), f2_of(0.43f * 0.70710678f), f2_of(1.0f)), rcp_approx);
        const f2 e = f2_each(f2_mul(f2_mul(z, f2_of(-0.5f * kLog2e)), z), ex2_approx);
        f2 g = f2_of(0.036572903f);
        g = f2_fma(g, t, f2_of(-0.15404779f));
        g = f2_fma(g, t, f2_of(0.1899436f));
        g = f2_fma(g, t, f2_of(-0.041152104f));
        g = f2_fma(g, t, f2_of(0.12254031f));
        g = f2_fma(g, t, f2_of(0.102736264f));
        g = f2_fma(g, t, f2_of(0.12214691f));
        g = f2_fma(g, t, f2_of(0.12125991f));
        f2_split(f2_mul(f2_mul(g, t), e), p, q);
        return f2_mul(z, f2_make(a < 0.0f ? p : 1.0f - p, b < 0.0f ? q : 1.0f - q));
    }
    float a, b;
    f2_split(z, a, b);
    return f2_make(act_value<ACT>(a), act_value<ACT>(b));
}
template <int ACT, int N> __device__ __forceinline__ void act_all(float (&v)[N]) {
    if constexpr (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) f2_split(act_value2<ACT>(f2_make(v[i], v[i + 1])), v[i], v[i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = act_value<ACT>(v[i]);
    }
}
template <int N> __device__ __forceinline__ void activate(int act, float (&v)[N]) {
    switch (act) {
        case RLF_ACT_RELU: act_all<RLF_ACT_RELU, N>(v); break;
        case RLF_ACT_SILU: act_all<RLF_ACT_SILU, N>(v); break;
        case RLF_ACT_GELU: act_all<RLF_ACT_GELU, N>(v); break;
        case RLF_ACT_GELU_TANH: act_all<RLF_ACT_GELU_TANH, N>(v); break;
        default: break;
    }
}
__device__ __forceinline__ float slope_of(int act, float z) {
    switch (act) {
        case RLF_ACT_RELU: return act_slope<RLF_ACT_RELU>(z);
        case RLF_ACT_SILU: return act_slope<RLF_ACT_SILU>(z);
        case RLF_ACT_GELU: return act_slope<RLF_ACT_GELU>(z);
        case RLF_ACT_GELU_TANH: return act_slope<RLF_ACT_GELU_TANH>(z);
        default: return 1.0f;
    }
}
__device__ __forceinline__ float value_of(int act, float z) {
    float v[1] = {z};
    activate<1>(act, v);
    return v[0];
}

__device__ __forceinline__ float load_any(const void* p, int f32, long long i) {
    return f32 ? static_cast<const float*>(p)[i] : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}
__device__ __forceinline__ void store_any(void* p, int f32, long long i, float v) {
    if (f32) static_cast<float*>(p)[i] = v;
    else static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
}

// ---- large products: pairs of CTAs, 256-row tiles ---------------------------------------------
constexpr int kBK = 64;
constexpr int kTileRows = 128;                        // rows of a tile that a CTA holds
// One accumulator (256 rows) per pair, double-buffered in tensor memory so that a tile drains under the next one's multiplies; or two
// (512 rows) that share every slab of B they stage: three quarters of the traffic from L2 per flop, but all of tensor memory.  Their
// drains overlap the next tile's first slabs in part: accumulator 0 restarts while accumulator 1 still drains.
constexpr int kABytes = kTileRows * kBK * 2, kBBytes = 128 * kBK * 2;
template <int ACC> struct PairCfg {
    static constexpr int kStages = ACC == 1 ? 6 : 4;
    static constexpr int kStageBytes = ACC * kABytes + kBBytes;
};
constexpr int kRingBytes = 6 * (kABytes + kBBytes);
static_assert(PairCfg<1>::kStages * PairCfg<1>::kStageBytes == kRingBytes && PairCfg<2>::kStages * PairCfg<2>::kStageBytes == kRingBytes, "one ring");
constexpr int kDrainWarps = 8;
constexpr int kPairThreads = 64 + 32 * kDrainWarps;
constexpr int kDrainTile = 4096;                      // bytes of a drain warp's output tile: 32 rows of 32 columns, fp32 or two of bf16, or of 64 bf16 columns
constexpr int kDrainBytes = kDrainWarps * (kDrainTile + 128);
constexpr int kPairSmem = kRingBytes + kDrainBytes + 1024 + 256;
static_assert(kPairSmem <= 227 * 1024, "the most shared memory a CTA can have");

// One launch multiplies one product or two (a backward pass' dx and dW: no launch and no ragged last wave between them).
struct PairProblem {
    int M;                          // output rows
    int m_units, n_tiles, k_slabs;  // 256-row units, column tiles, 64-deep slabs
    int bn;                         // accumulator columns of a tile (gated: half of them gate, half up)
    int a_mn, b_mn;                 // operand stored with the summed axis along its rows
    int group;                      // row units that are taken together (see the raster)
    int up_row;                     // gated: B's row with which the up half begins
    int wide;                       // results leave 64 columns at a time
    Epilogue e;
};
struct PairParams {
    PairProblem q[2];
    long long units0, units;        // tiles of the first product, of both
    int mixed;                      // an output is fp32, or leaves 64 columns at a time: a drain tile is then one store's at a time
    int32_t* dev_status;
};
struct alignas(64) PairMaps {
    CUtensorMap a[2], b[2], out[2], pre;
};

struct PairCtl {
    unsigned long long full[6], empty[6], tmem_full[2], tmem_empty[2];
    uint32_t tmem_base;
    volatile int abort_flag;
};
static_assert(sizeof(PairCtl) <= 256, "the barriers have 256 bytes behind the stage ring");

// A drain warp's output tiles.  Results leave as 32 x 32 tiles by TMA stores (rows of 64 or 128 bytes, swizzled so that the threads'
// 16-byte pieces meet no bank twice): whole sectors, and clipped at the last row and column.  (One row per thread stored straight
// to memory is 16 bytes of a sector at a time; those writes took as much of L2 as the operands: 8192 x 2560 x 10240 with two
// accumulators 413 us.)  Rows on no 16-byte boundary are stored by element, a row's 32 columns at a time.
struct Drain {
    unsigned char* tile;            // kDrainTile bytes
    float* bias;                    // 32 floats
    int lane, next;
};
template <bool F32>
__device__ __forceinline__ void store_piece(Drain& d, const CUtensorMap* map, bool tma, int third, bool mixed, void* out, long long stride,
                                            int row0, int M, int col, int nvalid, const float (&v)[32]) {
    const int lane = d.lane;
    if (tma) {
        // the store that read this tile last has read it (the other bf16 tile's may still be on its way)
        if (lane == 0) {
            if (F32 || mixed) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            else asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
        }
        __syncwarp();
        const uint32_t at = smem_addr(d.tile) + (F32 ? 0u : (uint32_t)d.next * 2048u);
        d.next ^= 1;
        if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};"
                             :: "r"(at + (uint32_t)(lane * 128 + ((i ^ (lane & 7)) << 4))), "f"(v[4 * i]), "f"(v[4 * i + 1]), "f"(v[4 * i + 2]),
                                "f"(v[4 * i + 3]) : "memory");
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};"
                             :: "r"(at + (uint32_t)(lane * 64 + ((i ^ ((lane >> 1) & 3)) << 4))), "r"(pack_bf16x2(v[8 * i], v[8 * i + 1])),
                                "r"(pack_bf16x2(v[8 * i + 2], v[8 * i + 3])), "r"(pack_bf16x2(v[8 * i + 4], v[8 * i + 5])),
                                "r"(pack_bf16x2(v[8 * i + 6], v[8 * i + 7])) : "memory");
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
            if (row0 < M)
                asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
                             :: "l"(map), "r"(at), "r"(col), "r"(third), "r"(row0) : "memory");
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
        return;
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
    float* t = reinterpret_cast<float*>(d.tile);
#pragma unroll
    for (int i = 0; i < 32; ++i) t[lane * 32 + (i ^ lane)] = v[i];
    __syncwarp();
    const int rows = min(32, M - row0);
    if (lane < nvalid) {
#pragma unroll 4
        for (int r = 0; r < rows; ++r) store_any(out, F32, (long long)(row0 + r) * stride + col + lane, t[r * 32 + (lane ^ r)]);
    }
    __syncwarp();
}
// 32 rows of 64 bf16 columns, a whole line each: half the loads, fences and stores that two tiles of 32 columns take.  Where K is
// short the drain is what a tile takes, and its time is theirs, one after the other (13312 x 128 x 5120 54 -> 47 us).
__device__ __forceinline__ void store_wide(Drain& d, const CUtensorMap* map, int row0, int M, int col, const uint32_t (&q)[32]) {
    if (d.lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
    const uint32_t at = smem_addr(d.tile);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};"
                     :: "r"(at + (uint32_t)(d.lane * 128 + ((i ^ (d.lane & 7)) << 4))), "r"(q[4 * i]), "r"(q[4 * i + 1]), "r"(q[4 * i + 2]),
                        "r"(q[4 * i + 3]) : "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (d.lane == 0) {
        if (row0 < M)
            asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
                         :: "l"(map), "r"(at), "r"(col), "r"(0), "r"(row0) : "memory");
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
}
// A 32 x 32 piece of the residual on its way: 32 columns of this thread's row where rows lie on 16-byte boundaries, else this
// lane's column of the 32 rows (by row, element after element, a warp touches 32 rows at once: 2047 x 1024 x 4099 91 us, so
// 32).  It is fetched before the piece's accumulator is waited for.
struct Residual {
    uint32_t q[32];
    bool by_row;
};
__device__ __forceinline__ void fetch_residual(const Epilogue& e, int row, int M, int lane, int col, int nvalid, Residual& r) {
    r.by_row = e.vec_res && nvalid == 32;
    if (r.by_row) {
        if (row >= M) return;
        const char* from = static_cast<const char*>(e.res) + (row * e.res_stride + col) * (e.out_f32 ? 4 : 2);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i >= 4 && !e.out_f32) break;
            const uint4 q = reinterpret_cast<const uint4*>(from)[i];
            r.q[4 * i] = q.x; r.q[4 * i + 1] = q.y; r.q[4 * i + 2] = q.z; r.q[4 * i + 3] = q.w;
        }
    } else {
        // (no condition between the loads; what lies beyond the last row or column is read from there and not used)
        const int row0 = row - lane;
        const long long at = col + min(lane, nvalid - 1);
        if (e.out_f32) {
#pragma unroll
            for (int i = 0; i < 32; ++i) r.q[i] = static_cast<const unsigned*>(e.res)[min(row0 + i, M - 1) * e.res_stride + at];
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) r.q[i] = static_cast<const unsigned short*>(e.res)[min(row0 + i, M - 1) * e.res_stride + at];
        }
    }
}
__device__ __forceinline__ void add_residual(const Epilogue& e, Drain& d, const Residual& r, float (&v)[32]) {
    if (!r.by_row) {
        if (d.lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
        float* t = reinterpret_cast<float*>(d.tile);
#pragma unroll
        for (int i = 0; i < 32; ++i) t[i * 32 + (d.lane ^ i)] = __uint_as_float(e.out_f32 ? r.q[i] : r.q[i] << 16);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] += t[d.lane * 32 + (i ^ d.lane)];
        __syncwarp();
    } else if (e.out_f32) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] += __uint_as_float(r.q[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) { v[2 * i] += bf_lo(r.q[i]); v[2 * i + 1] += bf_hi(r.q[i]); }
    }
}

template <int ACC>
__global__ void __launch_bounds__(kPairThreads, 1)
linear_pair_kernel(const __grid_constant__ PairMaps maps, const __grid_constant__ PairParams p) {
    constexpr int kStages = PairCfg<ACC>::kStages, kStageBytes = PairCfg<ACC>::kStageBytes;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw = smem_addr(smem_raw);
    const uint32_t ring = (raw + 1023u) & ~1023u;          // operand stages sit on 1024-byte boundaries (swizzle atom)
    unsigned char* drain = smem_raw + (ring - raw) + kRingBytes;
    PairCtl* ctl = reinterpret_cast<PairCtl*>(smem_raw + (ring - raw) + kRingBytes + kDrainBytes);
    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int rank = uniform((int)pair_rank());
    const int worker = blockIdx.x >> 1, workers = gridDim.x >> 1;
    const long long units = p.units;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(smem_addr(&ctl->full[s]), 1);
            mbar_init(smem_addr(&ctl->empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_addr(&ctl->tmem_full[b]), 1);
            mbar_init(smem_addr(&ctl->tmem_empty[b]), 2 * kDrainWarps);
        }
        ctl->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(smem_addr(&ctl->tmem_base)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                                    // both CTAs' barriers exist before either signals the other
    tc_fence_after();
    pdl_start();
    pdl_wait();
    const uint32_t tmem_base = (uint32_t)uniform((int)ctl->tmem_base);

    // Raster: groups of row units; inside a group row units fastest, so that the workers running at one time cover a block of
    // about as many rows as columns and share both operands through L2.
    auto unit_at = [&](long long u, int& m, int& n) -> int {
        const int which = u >= p.units0 ? 1 : 0;
        const PairProblem& q = p.q[which];
        if (which) u -= p.units0;
        const long long per_group = (long long)q.group * q.n_tiles;
        const int g = (int)(u / per_group);
        const int within = (int)(u - g * per_group), rows_here = min(q.group, q.m_units - g * q.group);
        n = within / rows_here;
        m = g * q.group + (within - n * rows_here);
        return which;
    };

    if (warp == 0) {
        // ---------------- loads (each CTA its own rows of A and half of B) ----------------
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        const uint32_t full0 = smem_addr(&ctl->full[0]), empty0 = smem_addr(&ctl->empty[0]), lead0 = (uint32_t)uniform((int)map_to_cta(full0, 0));
        for (long long u = worker; u < units && ok; u += workers) {
            int m, n;
            const int which = unit_at(u, m, n);
            const PairProblem& q = p.q[which];
            const CUtensorMap *map_a = &maps.a[which], *map_b = &maps.b[which];
            const int b_rows = q.bn / 2, k_slabs = q.k_slabs, a_mn = q.a_mn, b_mn = q.b_mn;            // (b_rows: rows of B that a CTA stages)
            const int b_row = q.e.gated ? (rank ? q.up_row : 0) + n * b_rows : n * q.bn + rank * b_rows;
            const uint32_t stage_tx = (uint32_t)(ACC * kABytes + b_rows * kBK * 2);
            for (int kb = 0; kb < k_slabs; ++kb) {
                if (!__all_sync(0xffffffffu, long_wait(empty0 + 8 * stage, phase ^ 1u, &ctl->abort_flag))) { ok = false; break; }
                if (elect_one()) {
                    const uint32_t bar = lead0 + 8 * stage;             // the leader's barrier
                    const uint32_t sb = ring + stage * kStageBytes + ACC * kABytes;
                    if (rank == 0) mbar_expect_tx(full0 + 8 * stage, 2 * stage_tx);
#pragma unroll
                    for (int a = 0; a < ACC; ++a) {
                        const uint32_t sa = ring + stage * kStageBytes + a * kABytes;
                        const int a_row = (2 * (ACC * m + a) + rank) * kTileRows;
                        if (!a_mn) {
                            tma_load_2d_pair(sa, map_a, bar, kb * kBK, a_row);
                        } else {
#pragma unroll
                            for (int j = 0; j < kTileRows / 64; ++j) tma_load_2d_pair(sa + j * kSlabBytes, map_a, bar, a_row + j * 64, kb * kBK);
                        }
                    }
                    if (!b_mn) {
                        tma_load_2d_pair(sb, map_b, bar, kb * kBK, b_row);
                    } else {
                        tma_load_2d_pair(sb, map_b, bar, b_row, kb * kBK);
                        if (b_rows > 64) tma_load_2d_pair(sb + kSlabBytes, map_b, bar, b_row + 64, kb * kBK);
                    }
                }
                __syncwarp();
                if (++stage == kStages) { stage = 0; phase ^= 1u; }
            }
        }
    } else if (warp == 1) {
        // ---------------- multiplies (the leader CTA) ----------------
        if (rank == 0) {
            uint32_t idesc = 0, a_step = 0, b_step = 0;
            uint64_t ad0 = 0, bd0 = 0;
            int k_slabs = 0;
            int stage = 0, buf = 0;
            uint32_t phase = 0, tphase = 0;                // bit b: parity of accumulator b
            bool ok = true;
            const uint32_t full0 = smem_addr(&ctl->full[0]), empty0 = smem_addr(&ctl->empty[0]);
            auto ready = [&](int st, uint32_t ph) {
                ok = __all_sync(0xffffffffu, long_wait(full0 + 8 * st, ph, &ctl->abort_flag));
                tc_fence_after();
            };
            auto drained = [&](int b) {
                ok = __all_sync(0xffffffffu, long_wait(smem_addr(&ctl->tmem_empty[b]), ((tphase >> b) & 1u) ^ 1u, &ctl->abort_flag));
                tphase ^= 1u << b;
                tc_fence_after();
            };
            auto multiply = [&](int st, int a, int b, bool first) {
                const uint64_t ad = ad0 + (uint64_t)((st * kStageBytes + a * kABytes) >> 4), bd = bd0 + (uint64_t)((st * kStageBytes) >> 4);
#pragma unroll
                for (int k = 0; k < kBK / 16; ++k)
                    tc_mma2(tmem_base + (uint32_t)b * 256u, ad + (uint64_t)(k * a_step), bd + (uint64_t)(k * b_step), idesc, first && k == 0 ? 0u : 1u);
            };
            auto advance = [&](int& st, uint32_t& ph) {
                if (++st == kStages) { st = 0; ph ^= 1u; }
            };
            for (long long u = worker; u < units && ok; u += workers) {
                const PairProblem& q = p.q[u >= p.units0 ? 1 : 0];
                idesc = instr_desc(q.a_mn, q.b_mn, 2 * kTileRows, q.bn);
                a_step = q.a_mn ? (16 * 128) >> 4 : 32 >> 4;
                b_step = q.b_mn ? (16 * 128) >> 4 : 32 >> 4;
                ad0 = smem_desc(ring, q.a_mn);
                bd0 = smem_desc(ring + ACC * kABytes, q.b_mn);
                k_slabs = q.k_slabs;
                if constexpr (ACC == 1) {
                    drained(buf);
                    for (int kb = 0; kb < k_slabs && ok; ++kb) {
                        ready(stage, phase);
                        if (!ok) break;
                        if (elect_one()) {
                            multiply(stage, 0, buf, kb == 0);
                            tc_commit2(empty0 + 8 * stage);              // frees the stage in both CTAs when these retire
                            if (kb + 1 == k_slabs) tc_commit2(smem_addr(&ctl->tmem_full[buf]));
                        }
                        __syncwarp();
                        advance(stage, phase);
                    }
                    if (!ok) break;
                    buf ^= 1;
                } else {
                    // accumulator 0 takes the ring's slabs while accumulator 1 may still be draining, which then catches up
                    const int ahead = min(kStages, k_slabs);
                    drained(0);
                    int st = stage;
                    uint32_t ph = phase;
                    for (int kb = 0; kb < ahead && ok; ++kb) {
                        ready(st, ph);
                        if (!ok) break;
                        if (elect_one()) {
                            multiply(st, 0, 0, kb == 0);
                            if (kb + 1 == k_slabs) tc_commit2(smem_addr(&ctl->tmem_full[0]));
                        }
                        __syncwarp();
                        advance(st, ph);
                    }
                    if (ok) drained(1);
                    for (int kb = 0; kb < k_slabs && ok; ++kb) {
                        if (kb >= ahead) {
                            ready(stage, phase);
                            if (!ok) break;
                        }
                        if (elect_one()) {
                            if (kb >= ahead) {
                                multiply(stage, 0, 0, false);
                                if (kb + 1 == k_slabs) tc_commit2(smem_addr(&ctl->tmem_full[0]));
                            }
                            multiply(stage, 1, 1, kb == 0);
                            tc_commit2(empty0 + 8 * stage);
                            if (kb + 1 == k_slabs) tc_commit2(smem_addr(&ctl->tmem_full[1]));
                        }
                        __syncwarp();
                        advance(stage, phase);
                    }
                    if (!ok) break;
                }
            }
        }
    } else {
        // ---------------- epilogue: one row per thread, two warps share a row's 32-column pieces ----------------
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        Drain d;
        d.tile = drain + (warp - 2) * kDrainTile;
        d.bias = reinterpret_cast<float*>(drain + kDrainWarps * kDrainTile) + (warp - 2) * 32;
        d.lane = lane;
        d.next = 0;
        int buf = 0;
        uint32_t tphase = 0;
        for (long long u = worker; u < units; u += workers) {
            int m, n;
            const int which = unit_at(u, m, n);
            const Epilogue& e = p.q[which].e;
            const CUtensorMap* map_out = &maps.out[which];
            const int width = e.gated ? p.q[which].bn / 2 : p.q[which].bn, M = p.q[which].M;
            const bool wide = p.q[which].wide;
            bool alive = true;
            // the tile's bias and first piece of the residual are fetched before its accumulator is waited for
            float bias[4] = {0.0f, 0.0f, 0.0f, 0.0f};      // this lane's column in each of this warp's pieces (gated: gate, up, gate, up)
            if (e.bias) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int c = e.gated ? half + (k & 2) : wide ? 2 * half + (k & 1) + 2 * (k & 2) : half + 2 * k, col = n * width + c * 32 + lane;
                    if (c < width / 32 && col < e.N) bias[k] = load_any(e.bias, !e.bias_bf16, (e.gated && (k & 1) ? e.N : 0) + col);
                }
            }
#pragma unroll 1
            for (int a = 0; a < ACC && alive; ++a) {
            const int row = (2 * (ACC * m + a) + rank) * kTileRows + quarter * 32 + lane;
            Residual r;
            auto fetch = [&](int c) {
                const int col = n * width + c * 32;
                if (c < width / 32 && col < e.N) fetch_residual(e, row, M, lane, col, min(32, e.N - col), r);
            };
            if (e.res) fetch(half);
            int got = 0;
            if (lane == 0) got = long_wait(smem_addr(&ctl->tmem_full[buf]), (tphase >> buf) & 1u, &ctl->abort_flag) ? 1 : 0;
            if (!__shfl_sync(0xffffffffu, got, 0)) {
                alive = false;
                break;
            }
            tc_fence_after();
            const uint32_t t_row = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)buf * 256u;
            if (wide) {
#pragma unroll 1
                for (int g = half; 2 * g < width / 32; g += 2) {
                    const int col = n * width + g * 64;
                    if (col >= e.N) break;
                    uint32_t lo[32], hi[32];
                    tc_ld32_issue(t_row + (uint32_t)(g * 64), lo);
                    tc_ld32_issue(t_row + (uint32_t)(g * 64 + 32), hi);
                    tc_ld_wait(lo);
                    tc_ld_wait(hi);
                    uint32_t packed[32];
                    auto finish = [&](const uint32_t (&raw)[32], int h) {      // bias and activation; to bf16
                        float v[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(raw[i]);
                        if (e.bias) {
                            d.bias[lane] = g == half ? bias[h] : bias[2 + h];
                            __syncwarp();
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const float4 q = reinterpret_cast<const float4*>(d.bias)[i];
                                v[4 * i] += q.x; v[4 * i + 1] += q.y; v[4 * i + 2] += q.z; v[4 * i + 3] += q.w;
                            }
                            __syncwarp();
                        }
                        activate<32>(e.act, v);
#pragma unroll
                        for (int i = 0; i < 16; ++i) packed[16 * h + i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
                    };
                    finish(lo, 0);
                    finish(hi, 1);
                    store_wide(d, map_out, row - lane, M, col, packed);
                }
            } else
#pragma unroll 1
            for (int c = half; c < width / 32; c += 2) {
                const int col = n * width + c * 32;
                if (col >= e.N) break;                     // (warp-uniform)
                const int nvalid = min(32, e.N - col);
                uint32_t raw_v[32];
                float v[32];
                auto take = [&](uint32_t at, int half_of_w) {    // accumulator columns + bias
                    tc_ld32(t_row + at, raw_v);
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(raw_v[i]);
                    const int shift = half_of_w ? e.N : 0;
                    if (e.bias) {
                        const int k = e.gated ? (c & ~1) + half_of_w : c >> 1;
                        d.bias[lane] = k == 0 ? bias[0] : k == 1 ? bias[1] : k == 2 ? bias[2] : bias[3];
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float4 q = reinterpret_cast<const float4*>(d.bias)[i];
                            v[4 * i] += q.x; v[4 * i + 1] += q.y; v[4 * i + 2] += q.z; v[4 * i + 3] += q.w;
                        }
                        __syncwarp();
                    }
                    if (e.pre) store_piece<false>(d, &maps.pre, e.vec_pre, half_of_w, p.mixed, e.pre + shift, e.pre_stride, row - lane, M, col, nvalid, v);
                };
                take((uint32_t)(c * 32), 0);
                activate<32>(e.act, v);
                if (e.gated) {
                    float g[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) g[i] = v[i];
                    take((uint32_t)(width + c * 32), 1);
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] *= g[i];
                }
                if (e.res) {
                    add_residual(e, d, r, v);
                    fetch(c + 2);
                }
                if (e.out_f32) store_piece<true>(d, map_out, e.vec_out, 0, true, e.out, e.out_stride, row - lane, M, col, nvalid, v);
                else store_piece<false>(d, map_out, e.vec_out, 0, p.mixed, e.out, e.out_stride, row - lane, M, col, nvalid, v);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(map_to_cta(smem_addr(&ctl->tmem_empty[buf]), 0));
            tphase ^= 1u << buf;
            buf ^= 1;
            }
            if (!alive) break;
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");     // the last tiles are written before their memory goes
    }

    tc_fence_before();
    __syncthreads();
    if (ctl->abort_flag) {
        // copies or multiplies may still be in flight: give them time before the memory is released
        if (threadIdx.x == 0 && p.dev_status) atomicOr(p.dev_status, RLF_DEV_TIMEOUT);
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    }
    cluster_sync_all();                                    // the peer may still be signalling this CTA's barriers until here
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(tmem_base), "r"(512u) : "memory");
    }
}

// ---- few rows, or few tiles: the streamed form -------------------------------------------------
// out[j][i] = sum_k S[i][k] F[j][k]: S is streamed in tiles of 128 i (gated: 64 gate rows and the 64 up rows that belong to them),
// F's rows j, up to 256 in a tile, are the N side.  A cluster of `split` CTAs takes one tile, each a part of K.
// Tensor memory: a CTA takes nn / 512 of it (at least 32 columns) and more than that share of the shared memory, in every
// shape below, so that CTAs which are on an SM together never wait for one another's columns.
constexpr int kNarrowThreads = 192;
constexpr int kNarrowPitch = 132;                     // floats between two j of the staged accumulator
constexpr int kMaxNarrowStages = 12;

struct NarrowParams {
    int J;                          // output rows
    int k_slabs, nn, stages;
    int s_mn, f_mn;                 // operand stored with the summed axis along its rows
    int up_row;
    Epilogue e;
    int32_t* dev_status;
};
struct NarrowCtl {
    unsigned long long full[kMaxNarrowStages], empty[kMaxNarrowStages], tmem_full;
    uint32_t tmem_base;
    volatile int abort_flag;
};
static_assert(sizeof(NarrowCtl) <= 256, "the barriers have 256 bytes behind the stage ring");

__host__ __device__ constexpr int narrow_stage_bytes(int nn) { return kABytes + nn * kBK * 2; }
__host__ __device__ constexpr int narrow_ring_bytes(int nn, int stages) {
    const int r = stages * narrow_stage_bytes(nn), staged = nn * kNarrowPitch * 4;
    return r > staged ? r : (staged + 255) / 256 * 256;
}

__device__ __forceinline__ void tma_prefetch_2d(const CUtensorMap* map, int x, int y) {
    asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global [%0, {%1, %2}];" :: "l"(map), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ float4 ld_cluster_f4(uint32_t local_addr, uint32_t rank) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(map_to_cta(local_addr, rank)) : "memory");
    return v;
}
// four columns of a row: bias, then `pre`
__device__ __forceinline__ void narrow_bias_pre(const Epilogue& e, int row, int col, int nvalid, int shift, float (&z)[4]) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (e.bias && k < nvalid) z[k] += load_any(e.bias, !e.bias_bf16, shift + col + k);
    if (e.pre) {
        __nv_bfloat16* d = e.pre + row * e.pre_stride + shift + col;
        if (e.vec_pre && nvalid == 4) {
            *reinterpret_cast<uint2*>(d) = make_uint2(pack_bf16x2(z[0], z[1]), pack_bf16x2(z[2], z[3]));
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k < nvalid) d[k] = __float2bfloat16_rn(z[k]);
        }
    }
}

__global__ void __launch_bounds__(kNarrowThreads)
linear_narrow_kernel(const __grid_constant__ CUtensorMap map_s, const __grid_constant__ CUtensorMap map_f, const NarrowParams p) {
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw = smem_addr(smem_raw);
    const uint32_t ring = (raw + 1023u) & ~1023u;
    float* staged = reinterpret_cast<float*>(smem_raw + (ring - raw));
    const int stage_bytes = narrow_stage_bytes(p.nn);
    NarrowCtl* ctl = reinterpret_cast<NarrowCtl*>(smem_raw + (ring - raw) + narrow_ring_bytes(p.nn, p.stages));
    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int split = uniform((int)cluster_nctarank()), rank = uniform((int)cluster_ctarank());
    const int it = blockIdx.x / split, jt = blockIdx.y;
    const int k0 = (int)((long long)p.k_slabs * rank / split), k1 = (int)((long long)p.k_slabs * (rank + 1) / split);
    const uint32_t columns = p.nn < 32 ? 32u : (uint32_t)p.nn;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(smem_addr(&ctl->full[s]), 1);
            mbar_init(smem_addr(&ctl->empty[s]), 1);
        }
        mbar_init(smem_addr(&ctl->tmem_full), 1);
        ctl->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(smem_addr(&ctl->tmem_base)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_start();
    const uint32_t tmem_base = (uint32_t)uniform((int)ctl->tmem_base);

    const uint32_t full0 = smem_addr(&ctl->full[0]), empty0 = smem_addr(&ctl->empty[0]);
    const int i0 = p.e.gated ? it * 64 : it * 128, i1 = p.e.gated ? p.up_row + i0 : i0 + 64;
    // the streamed operand's first slabs are on their way to L2 while the kernel before this one ends (L2 takes its writes too)
    if (warp == 0 && elect_one())
        for (int kb = k0; kb < k1 && kb < k0 + p.stages; ++kb) {
            tma_prefetch_2d(&map_s, p.s_mn ? i0 : kb * kBK, p.s_mn ? kb * kBK : i0);
            tma_prefetch_2d(&map_s, p.s_mn ? i1 : kb * kBK, p.s_mn ? kb * kBK : i1);
        }
    __syncwarp();
    pdl_wait();
    if (warp == 0) {
        int stage = 0;
        uint32_t phase = 0;
        for (int kb = k0; kb < k1; ++kb) {
            if (!__all_sync(0xffffffffu, long_wait(empty0 + 8 * stage, phase ^ 1u, &ctl->abort_flag))) break;
            if (elect_one()) {
                const uint32_t bar = full0 + 8 * stage;
                const uint32_t ss = ring + stage * stage_bytes, sf = ss + kABytes;
                mbar_expect_tx(bar, (uint32_t)stage_bytes);
                if (p.s_mn) {
                    tma_load_2d(ss, &map_s, bar, i0, kb * kBK);
                    tma_load_2d(ss + kSlabBytes, &map_s, bar, i1, kb * kBK);
                } else {
                    tma_load_2d(ss, &map_s, bar, kb * kBK, i0);
                    tma_load_2d(ss + kSlabBytes, &map_s, bar, kb * kBK, i1);
                }
                if (p.f_mn) {
                    for (int j = 0; j < p.nn / 64; ++j) tma_load_2d(sf + j * kSlabBytes, &map_f, bar, jt * p.nn + j * 64, kb * kBK);
                } else {
                    tma_load_2d(sf, &map_f, bar, kb * kBK, jt * p.nn);
                }
            }
            __syncwarp();
            if (++stage == p.stages) { stage = 0; phase ^= 1u; }
        }
    } else if (warp == 1) {
        const uint32_t idesc = instr_desc(p.s_mn, p.f_mn, 128, p.nn);
        const uint32_t s_step = p.s_mn ? (16 * 128) >> 4 : 32 >> 4, f_step = p.f_mn ? (16 * 128) >> 4 : 32 >> 4;
        const uint64_t sd0 = smem_desc(ring, p.s_mn), fd0 = smem_desc(ring + kABytes, p.f_mn);
        int stage = 0;
        uint32_t phase = 0;
        for (int kb = k0; kb < k1; ++kb) {
            if (!__all_sync(0xffffffffu, long_wait(full0 + 8 * stage, phase, &ctl->abort_flag))) break;
            tc_fence_after();
            if (elect_one()) {
                const uint64_t at = (uint64_t)((stage * stage_bytes) >> 4);
#pragma unroll
                for (int k = 0; k < kBK / 16; ++k)
                    tc_mma(tmem_base, sd0 + at + (uint64_t)(k * s_step), fd0 + at + (uint64_t)(k * f_step), idesc, (kb > k0 || k) ? 1u : 0u);
                tc_commit(empty0 + 8 * stage);
                if (kb + 1 == k1) tc_commit(smem_addr(&ctl->tmem_full));
            }
            __syncwarp();
            if (++stage == p.stages) { stage = 0; phase ^= 1u; }
        }
    } else {
        // the accumulator goes to shared memory as [j][i] (the ring's memory: every copy has been multiplied by then)
        int got = 0;
        if (lane == 0) got = long_wait(smem_addr(&ctl->tmem_full), 0, &ctl->abort_flag) ? 1 : 0;
        if (__shfl_sync(0xffffffffu, got, 0)) {
            tc_fence_after();
            const int i = (warp & 3) * 32 + lane;
#pragma unroll 1
            for (int c = 0; c < p.nn; c += 32) {
                uint32_t v[32];
                tc_ld32(tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)c, v);
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (c + j < p.nn) staged[(c + j) * kNarrowPitch + i] = __uint_as_float(v[j]);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (ctl->abort_flag) {
        if (threadIdx.x == 0 && p.dev_status) atomicOr(p.dev_status, RLF_DEV_TIMEOUT);
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    }
    cluster_sync_all();                                    // every CTA's part is staged
    // the tile's rows j are dealt over the cluster; parts are added in rank order
    const Epilogue& e = p.e;
    const int rows = min(p.nn, p.J - jt * p.nn);
    const int j0 = rows * rank / split, j1 = rows * (rank + 1) / split;
    const int groups = e.gated ? 16 : 32;                  // of four columns
    const uint32_t base = smem_addr(staged);
    for (int x = threadIdx.x; x < (j1 - j0) * groups; x += kNarrowThreads) {
        const int j = j0 + x / groups, g = x % groups;
        const int row = jt * p.nn + j, col = it * 4 * groups + 4 * g;
        const int nvalid = min(4, e.N - col);
        if (nvalid <= 0) continue;
        float z[4] = {0.0f, 0.0f, 0.0f, 0.0f}, up[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        const uint32_t at = base + (uint32_t)(j * kNarrowPitch + 4 * g) * 4u;
#pragma unroll 4
        for (int q = 0; q < split; ++q) {
            const float4 a = ld_cluster_f4(at, (uint32_t)q);
            z[0] += a.x; z[1] += a.y; z[2] += a.z; z[3] += a.w;
            if (e.gated) {
                const float4 b = ld_cluster_f4(at + 256u, (uint32_t)q);
                up[0] += b.x; up[1] += b.y; up[2] += b.z; up[3] += b.w;
            }
        }
        narrow_bias_pre(e, row, col, nvalid, 0, z);
        activate<4>(e.act, z);
        if (e.gated) {
            narrow_bias_pre(e, row, col, nvalid, e.N, up);
#pragma unroll
            for (int k = 0; k < 4; ++k) z[k] *= up[k];
        }
        const long long o = row * e.out_stride + col, ro = row * e.res_stride + col;
        if (e.vec_out && e.vec_res && nvalid == 4) {
            if (e.out_f32) {
                if (e.res) {
                    const float4 r = *reinterpret_cast<const float4*>(static_cast<const float*>(e.res) + ro);
                    z[0] += r.x; z[1] += r.y; z[2] += r.z; z[3] += r.w;
                }
                *reinterpret_cast<float4*>(static_cast<float*>(e.out) + o) = make_float4(z[0], z[1], z[2], z[3]);
            } else {
                if (e.res) {
                    const uint2 r = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(e.res) + ro);
                    z[0] += bf_lo(r.x); z[1] += bf_hi(r.x); z[2] += bf_lo(r.y); z[3] += bf_hi(r.y);
                }
                *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(e.out) + o) = make_uint2(pack_bf16x2(z[0], z[1]), pack_bf16x2(z[2], z[3]));
            }
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k < nvalid) {
                    if (e.res) z[k] += load_any(e.res, e.out_f32, ro + k);
                    store_any(e.out, e.out_f32, o + k, z[k]);
                }
        }
    }
    cluster_sync_all();                                    // the others have read this CTA's part
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem_base), "r"(columns) : "memory");
    }
}

// ---- at most four outputs ------------------------------------------------------------------------
// Forward: a warp takes R tokens; its lanes run along the row, 16 bytes of x and of each weight row at a time.  (No __restrict__ on what is
// read: it lets loads take the path for data that nothing writes while the kernel runs, and the launch before, under which this one
// is set up, may be writing x.)
template <int N, int R>
__global__ void __launch_bounds__(256)
linear_few_fwd_kernel(const __nv_bfloat16* x, long long x_stride, const __nv_bfloat16* W, long long T, int D, const Epilogue e) {
    pdl_start();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const long long t0 = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * R;
    if (t0 >= T) return;
    const int nvec = D / 8;
    const uint4* xr[R];
#pragma unroll
    for (int r = 0; r < R; ++r) xr[r] = reinterpret_cast<const uint4*>(x + min(t0 + r, T - 1) * x_stride);
    f2 acc[R][N];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int n = 0; n < N; ++n) acc[r][n] = 0ull;
#pragma unroll(N <= 2 ? 4 : 2)
    for (int c = lane; c < nvec; c += 32) {
        uint4 xv[R];
#pragma unroll
        for (int r = 0; r < R; ++r) xv[r] = xr[r][c];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const uint4 wv = reinterpret_cast<const uint4*>(W + (long long)n * D)[c];
            const uint32_t w[4] = {wv.x, wv.y, wv.z, wv.w};
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const uint32_t q[4] = {xv[r].x, xv[r].y, xv[r].z, xv[r].w};
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[r][n] = f2_fma(f2_make(bf_lo(q[k]), bf_hi(q[k])), f2_make(bf_lo(w[k]), bf_hi(w[k])), acc[r][n]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const float s = warp_sum(f2_sum(acc[r][n]));
            const long long t = t0 + r;
            if (lane != (r * N + n) % 32 || t >= T) continue;
            const float z = s + (e.bias ? load_any(e.bias, !e.bias_bf16, n) : 0.0f);
            if (e.pre) e.pre[t * e.pre_stride + n] = __float2bfloat16_rn(z);
            float y = value_of(e.act, z);
            if (e.res) y += load_any(e.res, e.out_f32, t * e.res_stride + n);
            store_any(e.out, e.out_f32, t * e.out_stride + n, y);
        }
}

struct FewBwd {
    const void* dy;
    long long dy_stride;
    int dy_f32, act;
    const __nv_bfloat16* pre;       // [T, N], nullable
    const __nv_bfloat16* x;
    long long x_stride;
    const __nv_bfloat16* W;         // [N, D]
    __nv_bfloat16* dx;              // [T, D], nullable
    float* part_w;                  // [slices][N][D], nullable
    float* part_b;                  // [slices][N], nullable
    long long T, rows;              // tokens, tokens of a slice
    int D;
};
// Backward: a CTA takes a slice of tokens and up to 2048 columns, eight to a thread (threadIdx.x); threadIdx.y deals the tokens.
// x is read and dx written once; the sums over tokens leave as one partial row per slice.
constexpr int kFewChunk = 64;                         // tokens whose gz is worked out at a time
template <int N>
__global__ void __launch_bounds__(256)
linear_few_bwd_kernel(const FewBwd p) {
    __shared__ float gz[kFewChunk][N];
    __shared__ float sum[256][9];
    pdl_start();
    pdl_wait();
    const int tx = threadIdx.x, ty = threadIdx.y, nx = blockDim.x, ny = blockDim.y, tid = ty * nx + tx;
    const int col = (blockIdx.x * nx + tx) * 8;
    const bool live = col < p.D;
    const long long t0 = (long long)blockIdx.y * p.rows, t1 = min(p.T, t0 + p.rows);
    f2 w[N][4], acc[N][4];
    float bias[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (live) v = *reinterpret_cast<const uint4*>(p.W + (long long)n * p.D + col);
        const uint32_t q[4] = {v.x, v.y, v.z, v.w};
        bias[n] = 0.0f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            w[n][k] = f2_make(bf_lo(q[k]), bf_hi(q[k]));
            acc[n][k] = 0ull;
        }
    }
    for (long long tc0 = t0; tc0 < t1; tc0 += kFewChunk) {
        const int tokens = (int)min((long long)kFewChunk, t1 - tc0);
        __syncthreads();
        for (int i = tid; i < tokens * N; i += 256) {
            const int r = i / N, n = i - r * N;
            float g = load_any(p.dy, p.dy_f32, (tc0 + r) * p.dy_stride + n);
            if (p.pre) g *= slope_of(p.act, __bfloat162float(p.pre[(tc0 + r) * N + n]));
            gz[r][n] = g;
        }
        __syncthreads();
        if (p.part_b && blockIdx.x == 0 && tid == 0)
            for (int r = 0; r < tokens; ++r)
#pragma unroll
                for (int n = 0; n < N; ++n) bias[n] += gz[r][n];
        if (!live) continue;
        // eight tokens' x at a time: their loads are all under way before the first is used
        for (int r0 = ty; r0 < tokens; r0 += 8 * ny) {
            uint4 v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (p.part_w && r0 + k * ny < tokens) v[k] = ld_stream(reinterpret_cast<const uint4*>(p.x + (tc0 + r0 + k * ny) * p.x_stride + col));
#pragma unroll
            for (int b = 0; b < 8; ++b) {
                const int r = r0 + b * ny;
                if (r >= tokens) break;
                f2 d[4] = {0ull, 0ull, 0ull, 0ull};
                const uint32_t q[4] = {v[b].x, v[b].y, v[b].z, v[b].w};
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    const f2 g = f2_make(gz[r][n], gz[r][n]);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (p.part_w) acc[n][k] = f2_fma(g, f2_make(bf_lo(q[k]), bf_hi(q[k])), acc[n][k]);
                        d[k] = f2_fma(g, w[n][k], d[k]);
                    }
                }
                if (p.dx) {
                    uint32_t o[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        float lo, hi;
                        f2_split(d[k], lo, hi);
                        o[k] = pack_bf16x2(lo, hi);
                    }
                    *reinterpret_cast<uint4*>(p.dx + (tc0 + r) * p.D + col) = make_uint4(o[0], o[1], o[2], o[3]);
                }
            }
        }
    }
    if (p.part_b && blockIdx.x == 0 && tid == 0)
#pragma unroll
        for (int n = 0; n < N; ++n) p.part_b[(long long)blockIdx.y * N + n] = bias[n];
    if (!p.part_w) return;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        float f[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) f2_split(acc[n][k], f[2 * k], f[2 * k + 1]);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[tid][k] = f[k];
        __syncthreads();
        if (ty == 0 && live) {
            for (int y = 1; y < ny; ++y)
#pragma unroll
                for (int k = 0; k < 8; ++k) f[k] += sum[y * nx + tx][k];
            float4* d = reinterpret_cast<float4*>(p.part_w + ((long long)blockIdx.y * N + n) * p.D + col);
            d[0] = make_float4(f[0], f[1], f[2], f[3]);
            d[1] = make_float4(f[4], f[5], f[6], f[7]);
        }
    }
}

// partial rows -> sums, in a fixed order: the first `blocks` CTAs cover 32 columns each of one sum, the others of a second (the bias
// gradient).  Warp w adds the rows w, w + 32, ..., at most 8 of them.
constexpr int kMostParts = 256;
struct Join {
    const float* part[2];
    long long width[2];
    void* out[2];
    int out_f32[2];
    int parts, accumulate, blocks;
};
__global__ void __launch_bounds__(1024)
linear_join_kernel(const Join j) {
    __shared__ float acc[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int which = (int)blockIdx.x >= j.blocks ? 1 : 0;
    const long long col = (long long)(blockIdx.x - (which ? j.blocks : 0)) * 32 + lane, width = j.width[which];
    pdl_start();
    pdl_wait();
    float s = 0.0f;
    if (col < width) {
        const float* part = j.part[which] + col;
        float v[8];                                        // (at most 256 parts: all of a warp's loads at once)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = warp + 32 * i < j.parts ? part[(warp + 32 * i) * width] : 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += v[i];
    }
    acc[warp][lane] = s;
    __syncthreads();
    s = warp_sum(acc[lane][warp]);                         // column `warp` of the block
    const long long c = col - lane + warp;
    if (lane == 0 && c < width) {
        if (j.accumulate) s += load_any(j.out[which], j.out_f32[which], c);
        store_any(j.out[which], j.out_f32[which], c, s);
    }
}

// ---- gradient before the activation --------------------------------------------------------------
struct PreGrad {
    const void* dy;
    long long dy_stride;
    int dy_f32, act, gated;
    const __nv_bfloat16* pre;       // [T, N], gated [T, 2 N]; nullable
    __nv_bfloat16* gz;              // rows of gz_stride; nullable (only the bias gradient is wanted)
    long long gz_stride;
    float* part_b;                  // [slices][N], gated [slices][2 N]; nullable
    long long T, rows;              // tokens, tokens of a slice
    int N;
};
// gz in bf16 (the products' operand: its one rounding) and, in fp32 and unrounded, its sums over a slice of tokens.  A thread keeps V
// columns; threadIdx.y deals the tokens.  V = 8: rows on 16-byte boundaries; 1: any.
template <int V, int ACT, bool GATED>
__global__ void __launch_bounds__(256)
linear_pregrad_kernel(const PreGrad p) {
    __shared__ float sum[8][32 * V + 1];
    pdl_start();
    pdl_wait();
    const int tx = threadIdx.x, ty = threadIdx.y;          // 32 x 8
    const int col = (blockIdx.x * 32 + tx) * V;
    const long long t0 = (long long)blockIdx.y * p.rows, t1 = min(p.T, t0 + p.rows);
    constexpr int H = GATED ? 2 : 1;
    float acc[H][V];
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
        for (int k = 0; k < V; ++k) acc[h][k] = 0.0f;
    const bool with_pre = ACT != RLF_ACT_NONE || GATED;
    if (col < p.N) {
#pragma unroll 2
        for (long long t = t0 + ty; t < t1; t += 8) {
            float g[V], z[H][V], o[H][V];
            if constexpr (V == 8) {
                if (p.dy_f32) {
                    const float4* d = reinterpret_cast<const float4*>(static_cast<const float*>(p.dy) + t * p.dy_stride + col);
                    const float4 a = d[0], b = d[1];
                    g[0] = a.x; g[1] = a.y; g[2] = a.z; g[3] = a.w; g[4] = b.x; g[5] = b.y; g[6] = b.z; g[7] = b.w;
                } else {
                    const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.dy) + t * p.dy_stride + col);
                    const uint32_t q[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) { g[2 * k] = bf_lo(q[k]); g[2 * k + 1] = bf_hi(q[k]); }
                }
                if (with_pre) {
#pragma unroll
                    for (int h = 0; h < H; ++h) {
                        const uint4 a = *reinterpret_cast<const uint4*>(p.pre + (t * H + h) * p.N + col);
                        const uint32_t q[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) { z[h][2 * k] = bf_lo(q[k]); z[h][2 * k + 1] = bf_hi(q[k]); }
                    }
                }
            } else {
                g[0] = load_any(p.dy, p.dy_f32, t * p.dy_stride + col);
                if (with_pre)
#pragma unroll
                    for (int h = 0; h < H; ++h) z[h][0] = __bfloat162float(p.pre[(t * H + h) * p.N + col]);
            }
#pragma unroll
            for (int k = 0; k < V; ++k) {
                if (GATED) {
                    o[0][k] = g[k] * z[H - 1][k] * act_slope<ACT>(z[0][k]);
                    o[H - 1][k] = g[k] * act_value<ACT>(z[0][k]);
                } else {
                    o[0][k] = ACT == RLF_ACT_NONE ? g[k] : g[k] * act_slope<ACT>(z[0][k]);
                }
#pragma unroll
                for (int h = 0; h < H; ++h) acc[h][k] += o[h][k];
            }
            if (p.gz) {
#pragma unroll
                for (int h = 0; h < H; ++h) {
                    __nv_bfloat16* d = p.gz + t * p.gz_stride + (long long)h * p.N + col;
                    if constexpr (V == 8)
                        *reinterpret_cast<uint4*>(d) = make_uint4(pack_bf16x2(o[h][0], o[h][1]), pack_bf16x2(o[h][2], o[h][3]),
                                                                  pack_bf16x2(o[h][4], o[h][5]), pack_bf16x2(o[h][6], o[h][7]));
                    else
                        d[0] = __float2bfloat16_rn(o[h][0]);
                }
            }
        }
    }
    if (!p.part_b) return;
#pragma unroll
    for (int h = 0; h < H; ++h) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < V; ++k) sum[ty][tx * V + k] = acc[h][k];
        __syncthreads();
        const int first = blockIdx.x * 32 * V;
        for (int c = ty * 32 + tx; c < 32 * V && first + c < p.N; c += 256) {
            float s = 0.0f;
#pragma unroll
            for (int y = 0; y < 8; ++y) s += sum[y][c];
            p.part_b[((long long)blockIdx.y * H + h) * p.N + first + c] = s;
        }
    }
}

// ---- host side ------------------------------------------------------------------------------------
static int sm_count() {
    static ResidentTable table;
    return table.get(nullptr, 0, 0, [](int dev) {
        int v = 0;
        cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev);
        return v > 0 ? v : 148;
    });
}

// form of the products for later calls (rlf_tune_linear); 0: chosen per call
static std::atomic<int> g_form{0}, g_tile{0}, g_split{0};

// an operand with `rows` output rows (columns): [rows][K] row-major, or with mn [K][rows] row-major
struct Operand {
    const void* at;
    long long stride;
    int mn;
};

struct Plan {
    int acc;                        // accumulators of a pair; 0: the streamed form
    int tile;                       // pair: accumulator columns; streamed: rows of a tile
    int split;                      // streamed: CTAs that share a tile's K
};
static int div_up(long long a, long long b) { return (int)((a + b - 1) / b); }

// The form of a product is the one with the least estimated time.  The estimates, in us, are fits to sweeps of every form over 100 shapes
// on one B200 (worst miss 25 %).  On 75 others (1 to 32768 tokens, widths of 128 to 14336, gated and not) the form they choose is within
// 5 % of the fastest one 53 times, within 10 % 63 times and within 20 % 72 times; what is further off are launches of 4 to 13 us (2 x 256 x
// 3328 4.7 us, 3.6 without a cluster; 43 x 576 x 576 5.7, 4.4; 862 x 3008 x 192 gated 13.3, 10.8):
//   pair      5 + waves (slabs t + drain), the drain hidden behind the next tile with one accumulator.  A 64-deep slab takes 0.30 us at
//             256 columns, 0.20 at 128 and never less than 0.19 (its issue); two accumulators 0.57 for twice the rows, and all of
//             their drain: 32768 x 10240 x 2560 1093 us against 1156, 32768 x 2560 x 2560 347 against 289.
//   streamed  3.5 + waves (2.5 + slabs t + the cluster's reduction); t is the issue of a slab (0.20 - 0.36) or its bytes at 105 GB/s per SM, shared
//             by the CTAs on it, and the whole is no less than 5 + reading everything once at 6.7 TB/s (ties go to the shorter work).
static double pair_slab(int bn, long long M, int unit) {
    const double slab = bn == 256 ? 0.30 : bn == 192 ? 0.235 : bn == 128 ? 0.20 : 0.19;
    if (M > unit) return slab;
    // a single row unit: all of B comes from HBM, each slab for one pair (100 x 2560 x 10240 gated 0.28 at 192 columns, 0.33 at 256), and a
    // handful of rows are a few lines that every pair asks for (8 x 4096 x 12288 gated 0.49)
    const double alone = (0.13 + bn * 0.00088) * (M <= 16 ? 2.0 : 1.0);
    return slab > alone ? slab : alone;
}
static double pair_cost(int acc, int bn, long long M, int N, int k_slabs, bool gated, int pairs) {
    const long long units = (long long)div_up(M, 256 * acc) * div_up(N, gated ? bn / 2 : bn);
    const double waves = (double)((units + pairs - 1) / pairs), drain = 1.5 + 0.6 * bn / 256.0;
    const double slab = pair_slab(bn, M, 256 * acc);
    if (acc == 1) {
        const double tile = k_slabs * slab;
        return 5.0 + waves * (tile > drain ? tile : drain) + drain;
    }
    return 5.0 + waves * (k_slabs * slab * 1.9 + drain) + drain;
}
// SMs that clusters of `split` CTAs can use at one CTA each: a cluster lies in one GPC, whose SMs are no multiple of it
// (5 x 1640 x 2104 in 17 clusters of 8 that filled an SM each: 11.9 us, with room for two on an SM 6.7).
static int cluster_slots(int split, int sms) { return split >= 8 ? sms * 13 / 16 : split >= 4 ? sms * 15 / 16 : sms; }
static int narrow_ctas_per_sm(int nn) { return nn <= 16 ? 4 : nn <= 64 ? 3 : nn == 128 ? 2 : 1; }      // (with three stages at least)
static double narrow_cost(int nn, int split, long long M, int N, int k_slabs, bool gated, int sms) {
    const int rows = gated ? 2 * N : N;
    const long long tiles = (long long)div_up(N, gated ? 64 : 128) * div_up(M, nn), ctas = tiles * split;
    const int most = narrow_ctas_per_sm(nn), slots = cluster_slots(split, sms);
    const double waves = (double)((ctas + (long long)most * slots - 1) / ((long long)most * slots));
    const double per_sm = ctas > (long long)most * slots ? most : (double)div_up(ctas, slots);
    const double issue = nn <= 32 ? 0.20 : nn == 64 ? 0.215 : nn == 128 ? 0.24 : 0.36, bytes = per_sm * (16384.0 + 128.0 * nn) / 105e3;
    const double reduce = 1.0 + nn * 32.0 / (split * (double)kNarrowThreads) * 0.25;
    const double t = 3.5 + waves * (2.5 + k_slabs / (double)split * (issue > bytes ? issue : bytes) + reduce);
    const double read = 5.0 + 128.0 * k_slabs * ((double)rows + (double)M) / 6.7e6;
    return (t > read ? t : read) + 0.05 * t;
}
static bool wanted_bn(int bn, bool b_mn, int tile) {
    if (b_mn && bn % 128 != 0) return false;
    return !(tile != 0 && bn != tile && tile >= 64 && tile % 64 == 0 && !(b_mn && tile % 128 != 0));
}
static Plan choose(long long M, int N, int k_slabs, bool gated, bool f_mn, bool b_mn, double* cost) {
    const int sms = sm_count();
    const int form = g_form.load(), tile = g_tile.load(), split = g_split.load();
    Plan best = {1, 256, 1};
    double least = 1e300;
    if (form != 2) {
        for (int acc = form == 3 ? 2 : 1; acc <= (form == 1 ? 1 : 2); ++acc)
            for (int bn = 256; bn >= 64; bn -= 64) {
                if (!wanted_bn(bn, b_mn, tile)) continue;
                const double t = pair_cost(acc, bn, M, N, k_slabs, gated, sms / 2);
                if (t < least) { least = t; best = {acc, bn, 1}; }
            }
    }
    if (form == 2 || form == 0) {
        for (int nn = f_mn ? 64 : 16; nn <= 256; nn *= 2) {
            if (form == 2 && (tile == 16 || tile == 32 || tile == 64 || tile == 128 || tile == 256) && !(f_mn && tile < 64) && nn != tile) continue;
            if (div_up(M, nn) > 65535) continue;           // (the launch's second dimension)
            for (int s = 1; s <= 8 && s <= k_slabs; ++s) { // (every CTA has a part of K)
                // clusters of 5 to 7 leave SMs of their GPC over (8 x 10240 x 2560: 7 CTAs 25.7 us, 8 15.0)
                if (split > 0 ? s != (split < k_slabs ? split : k_slabs) : (s & (s - 1)) != 0) continue;
                const double t = narrow_cost(nn, s, M, N, k_slabs, gated, sms);
                if (t < least) { least = t; best = {0, nn, s}; }
            }
            if (nn >= M && tile == 0) break;
        }
    }
    *cost = least;
    return best;
}

static bool opt_in(const void* kernel, int bytes) {
    static ResidentTable table;
    return table.get(kernel, 0, 0, [&](int) {
        const bool ok = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess;
        if (!ok) cudaGetLastError();
        return ok ? 1 : 0;
    }) == 1;
}

static rlf_status launch(const void* kernel, dim3 grid, dim3 threads, int smem, int cluster, void** args, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = threads;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    if (cudaLaunchKernelExC(&cfg, kernel, args) != cudaSuccess) {
        cudaGetLastError();
        return RLF_ERR_CUDA;
    }
    count_launch();
    return RLF_OK;
}

// rows of `halves` x N elements, stored in tiles of 32 rows x 32 columns (bf16 also 64)
static bool make_tile_map(CUtensorMap* map, const void* base, long long rows, int N, int halves, long long stride, bool f32, int columns) {
    const tc::EncodeTiledFn fn = tc::encode_fn();
    if (!fn) return false;
    const int esz = f32 ? 4 : 2;
    const cuuint64_t dims[3] = {(cuuint64_t)N, (cuuint64_t)halves, (cuuint64_t)rows};
    // (a single half: its stride is never taken)
    const cuuint64_t strides[2] = {(cuuint64_t)(halves > 1 ? N : stride) * esz, (cuuint64_t)stride * esz};
    const cuuint32_t box[3] = {(cuuint32_t)columns, 1, 32}, step[3] = {1, 1, 1};
    return fn(map, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, step,
              CU_TENSOR_MAP_INTERLEAVE_NONE, columns * esz == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// out[m][n] = epilogue(sum_k A[m][k] B[n][k]), M rows, e.N columns (gated: B has 2 e.N rows), K terms
struct Product {
    Operand A, B;
    long long M, K;
    Epilogue e;
    int k_slabs() const { return div_up(K, kBK); }
    int rows_b() const { return e.gated ? 2 * e.N : e.N; }
};
static bool encode(CUtensorMap* map, const Operand& o, long long K, long long rows, int box_rows) {
    return o.mn ? make_map(map, o.at, (uint64_t)K, (uint64_t)rows, (uint64_t)o.stride, 64, 64)
                : make_map(map, o.at, (uint64_t)rows, (uint64_t)K, (uint64_t)o.stride, 64, (uint32_t)box_rows);
}
static rlf_status launch_narrow(const Product& g, const Plan& plan, int32_t* dev_status, cudaStream_t s) {
    NarrowParams p = {};
    CUtensorMap ma, mb;
    p.J = (int)g.M; p.k_slabs = g.k_slabs(); p.nn = plan.tile; p.s_mn = g.B.mn; p.f_mn = g.A.mn; p.up_row = g.e.N; p.e = g.e; p.dev_status = dev_status;
    const int i_tiles = div_up(g.e.N, g.e.gated ? 64 : 128), j_tiles = div_up(g.M, plan.tile);
    // the SM's shared memory is shared by the CTAs that come to it (each CTA keeps 1 KB to the system)
    int per_sm = div_up((long long)i_tiles * j_tiles * plan.split, cluster_slots(plan.split, sm_count()));
    for (per_sm = per_sm > 4 ? 4 : per_sm;; --per_sm) {
        p.stages = (228 * 1024 / per_sm - 1024 - 1024 - 256) / narrow_stage_bytes(plan.tile);
        if (p.stages >= 3 || per_sm == 1) break;
    }
    if (p.stages > kMaxNarrowStages) p.stages = kMaxNarrowStages;
    const int smem = narrow_ring_bytes(plan.tile, p.stages) + 1024 + 256;
    if (!encode(&mb, g.B, g.K, g.rows_b(), 64) || !encode(&ma, g.A, g.K, g.M, plan.tile)) return RLF_ERR_CUDA;
    if (!opt_in((const void*)linear_narrow_kernel, 227 * 1024)) return RLF_ERR_CUDA;
    void* args[] = {&mb, &ma, &p};
    return launch((const void*)linear_narrow_kernel, dim3((unsigned)(i_tiles * plan.split), (unsigned)j_tiles), kNarrowThreads, smem, plan.split, args, s);
}
// one product, or two with tiles of their own widths
static rlf_status launch_pair(const Product* g, int count, int acc, const int* bn, int32_t* dev_status, cudaStream_t s) {
    PairParams p = {};
    PairMaps maps;
    for (int i = 0; i < count; ++i) {
        PairProblem& q = p.q[i];
        const Epilogue& e = g[i].e;
        q.M = (int)g[i].M; q.m_units = div_up(g[i].M, 2 * kTileRows * acc); q.k_slabs = g[i].k_slabs(); q.bn = bn[i];
        q.n_tiles = div_up(e.N, e.gated ? bn[i] / 2 : bn[i]);
        q.a_mn = g[i].A.mn; q.b_mn = g[i].B.mn; q.up_row = e.N; q.e = e;
        // about 28 MB of A's rows are live at a time (8192 x 4096 x 16384: groups of 4, 8, 16 units 826, 788, 779 us sustained; 32768 x 10240 x
        // 2560: 1340, 1353, 1370)
        const double panel = 512.0 * acc * (double)g[i].K;
        q.group = panel > 7e6 ? 4 : panel < 1.75e6 ? 16 : (int)(28e6 / panel);
        p.units += (long long)q.m_units * q.n_tiles;
        if (i == 0) p.units0 = p.units;
        if (!encode(&maps.a[i], g[i].A, g[i].K, g[i].M, kTileRows) || !encode(&maps.b[i], g[i].B, g[i].K, g[i].rows_b(), bn[i] / 2)) return RLF_ERR_CUDA;
        // results by 64 columns where the drain is longer than the multiplies; a longer K gains nothing, and with a residual or `pre`,
        // whose pieces are of 32 columns, it loses (8192 x 1024 x 1024 with residual 23 -> 25 us)
        q.wide = !e.out_f32 && !e.gated && !e.pre && !e.res && e.vec_out && bn[i] >= 128 && q.k_slabs <= 8;
        p.mixed |= e.out_f32 || q.wide;
        maps.out[i] = maps.a[i];
        if (e.vec_out && !make_tile_map(&maps.out[i], e.out, g[i].M, e.N, 1, e.out_stride, e.out_f32 != 0, q.wide ? 64 : 32)) return RLF_ERR_CUDA;
    }
    maps.pre = maps.a[0];
    const Epilogue& e = g[0].e;
    if (e.pre && e.vec_pre && !make_tile_map(&maps.pre, e.pre, g[0].M, e.N, e.gated ? 2 : 1, e.pre_stride, false, 32)) return RLF_ERR_CUDA;
    if (count == 1) maps.a[1] = maps.b[1] = maps.out[1] = maps.a[0];
    p.dev_status = dev_status;
    const void* const kernel = acc == 2 ? (const void*)linear_pair_kernel<2> : (const void*)linear_pair_kernel<1>;
    if (!opt_in(kernel, kPairSmem)) return RLF_ERR_CUDA;
    const int pairs = sm_count() / 2;
    const int workers = p.units < pairs ? (int)p.units : pairs;
    void* args[] = {&maps, &p};
    return launch(kernel, dim3((unsigned)(2 * workers)), kPairThreads, kPairSmem, 2, args, s);
}
static rlf_status run(const Product& g, const Plan& plan, int32_t* dev_status, cudaStream_t s) {
    if (plan.acc == 0) return launch_narrow(g, plan, dev_status, s);
    return launch_pair(&g, 1, plan.acc, &plan.tile, dev_status, s);
}
static Plan choose(const Product& g, double* cost) { return choose(g.M, g.e.N, g.k_slabs(), g.e.gated, g.A.mn, g.B.mn, cost); }
static rlf_status product(const Product& g, int32_t* dev_status, cudaStream_t s) {
    double cost;
    return run(g, choose(g, &cost), dev_status, s);
}
// Two products that depend on the same things: in one launch where that is estimated to be an eighth shorter than one after the other
// (backward of 2048 x 1024 x 1024 20 -> 12 us, 1000 x 2560 x 2560 34 -> 24, 4096 x 2560 x 2560 89 -> 76; below that margin it
// loses: 32768 x 1024 x 1024 at 0.99 of the estimate 116 -> 145).  The product with the longer tiles comes first; its tiles and the
// other's are dealt to the pairs as one list.
static rlf_status both_products(const Product& first, const Product& second, int32_t* dev_status, cudaStream_t s) {
    double c0, c1, least = 1e300;
    const Plan p0 = choose(first, &c0), p1 = choose(second, &c1);
    const int tile = g_tile.load(), pairs = sm_count() / 2;
    int bn[2] = {256, 256};
    const bool swap = first.k_slabs() < second.k_slabs();
    const Product &g0 = swap ? second : first, &g1 = swap ? first : second;
    if (g_form.load() <= 1)
        for (int b0 = 256; b0 >= 64; b0 -= 64)
            for (int b1 = 256; b1 >= 64; b1 -= 64) {
                if (!wanted_bn(b0, g0.B.mn, tile) || !wanted_bn(b1, g1.B.mn, tile)) continue;
                double all = 0.0, longest = 0.0, drain = 0.0;
                const Product* const g[2] = {&g0, &g1};
                for (int i = 0; i < 2; ++i) {              // (a single row unit's stream is hidden by the other product)
                    const int b = i ? b1 : b0;
                    const double d = 1.5 + 0.6 * b / 256.0, slabs = g[i]->k_slabs() * pair_slab(b, 1 << 30, 256);
                    const double t = slabs > d ? slabs : d;
                    all += t * div_up(g[i]->M, 256) * (double)div_up(g[i]->e.N, b);
                    longest = t > longest ? t : longest;
                    drain = d;                             // (the last tiles are the second product's)
                }
                const double even = all / pairs + 0.5 * (div_up(g1.M, 256) * (double)div_up(g1.e.N, b1) >= pairs ? longest * 0.5 : longest);
                const double t = 5.0 + (even > longest ? even : longest) + drain;
                if (t < least) { least = t; bn[0] = b0; bn[1] = b1; }
            }
    if (least < 0.87 * (c0 + c1 - 3.0)) {                  // (3 us: the second launch is set up under the first)
        const Product g[2] = {g0, g1};
        return launch_pair(g, 2, 1, bn, dev_status, s);
    }
    const rlf_status st = run(first, p0, dev_status, s);
    return st == RLF_OK ? run(second, p1, dev_status, s) : st;
}

static bool rows_aligned(const void* at, long long stride, int esz) { return aligned(at, 16) && stride * esz % 16 == 0; }

// slices of tokens of the elementwise passes (each leaves one partial row of a weight or bias gradient; a single one is the gradient)
static int token_slices(int64_t T) {
    const int64_t n = (T + 31) / 32;
    return (int)(n < 1 ? 1 : n > kMostParts ? kMostParts : n);
}
static int few_slices(int64_t T) {
    const int64_t n = (T + 7) / 8;
    return (int)(n < 1 ? 1 : n > kMostParts ? kMostParts : n);
}
static long long up8(long long n) { return (n + 7) & ~7ll; }
static size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
// gz, partial rows of grad_bias, partial rows of grad_W, one behind the other
struct BwdWs {
    size_t gz, part_b, part_w, total;
    bool holds(size_t gz_bytes, size_t b_bytes, size_t w_bytes) const {
        return gz_bytes <= part_b - gz && b_bytes <= part_w - part_b && w_bytes <= total - part_w;
    }
};
// The size is asked for by the rows of W.  Up to four of them may be those of a plain layer with as many outputs, which needs partial rows of
// grad_W and no gz, or, an even number, of a gated layer with half as many, which needs gz like any other: there is room for either.
static BwdWs bwd_workspace(int64_t T, int32_t rows, int32_t D) {
    BwdWs w;
    size_t o = 0;
    const bool few = rows <= kFewOutputs;
    const size_t slices = (size_t)(few ? few_slices(T) : token_slices(T));         // (few: the more of the two)
    w.gz = o;     o += few && rows % 2 != 0 ? 0 : up256((size_t)T * (size_t)up8(rows) * 2);
    w.part_b = o; o += up256(slices * (size_t)rows * 4);
    w.part_w = o; o += few ? up256(slices * (size_t)rows * (size_t)D * 4) : 0;
    w.total = o;
    return w;
}

static rlf_status check_linear(int64_t T, int32_t D, int32_t N, int act, int gated) {
    if (T < 0 || D < 1 || N < 1) return RLF_ERR_SHAPE;
    if (D % 8 != 0) return RLF_ERR_SHAPE;
    if (T >= (1 << 30) || D >= (1 << 30) || N >= (1 << 29)) return RLF_ERR_UNSUPPORTED;   // rows and columns are counted in 32 bits
    if (act < RLF_ACT_NONE || act > RLF_ACT_GELU_TANH || (gated != 0 && gated != 1)) return RLF_ERR_UNSUPPORTED;
    return RLF_OK;
}

template <int R>
static const void* few_fwd_kernel(int N) {
    switch (N) {
        case 1: return (const void*)linear_few_fwd_kernel<1, R>;
        case 2: return (const void*)linear_few_fwd_kernel<2, R>;
        case 3: return (const void*)linear_few_fwd_kernel<3, R>;
        default: return (const void*)linear_few_fwd_kernel<4, R>;
    }
}
static const void* few_bwd_kernel(int N) {
    switch (N) {
        case 1: return (const void*)linear_few_bwd_kernel<1>;
        case 2: return (const void*)linear_few_bwd_kernel<2>;
        case 3: return (const void*)linear_few_bwd_kernel<3>;
        default: return (const void*)linear_few_bwd_kernel<4>;
    }
}
template <int V, bool GATED>
static const void* pregrad_kernel(int act) {
    switch (act) {
        case RLF_ACT_RELU: return (const void*)linear_pregrad_kernel<V, RLF_ACT_RELU, GATED>;
        case RLF_ACT_SILU: return (const void*)linear_pregrad_kernel<V, RLF_ACT_SILU, GATED>;
        case RLF_ACT_GELU: return (const void*)linear_pregrad_kernel<V, RLF_ACT_GELU, GATED>;
        case RLF_ACT_GELU_TANH: return (const void*)linear_pregrad_kernel<V, RLF_ACT_GELU_TANH, GATED>;
        default: return (const void*)linear_pregrad_kernel<V, RLF_ACT_NONE, GATED>;
    }
}
// sums of the slices' partial rows of grad_W (nullable) and grad_bias (nullable)
static rlf_status launch_join(int parts, int accumulate, const float* part_w, long long width_w, void* grad_W, int w_f32, const float* part_b,
                              long long width_b, float* grad_bias, cudaStream_t s) {
    Join j = {};
    j.parts = parts;
    j.accumulate = accumulate;
    j.part[0] = part_w; j.width[0] = grad_W ? width_w : 0; j.out[0] = grad_W; j.out_f32[0] = w_f32;
    j.part[1] = part_b; j.width[1] = grad_bias ? width_b : 0; j.out[1] = grad_bias; j.out_f32[1] = 1;
    j.blocks = div_up(j.width[0], 32);
    const unsigned grid = (unsigned)(j.blocks + div_up(j.width[1], 32));
    if (grid == 0) return RLF_OK;
    void* args[] = {&j};
    return launch((const void*)linear_join_kernel, dim3(grid), dim3(1024), 0, 1, args, s);
}

}  // namespace ln

size_t linear_bwd_workspace_bytes(int64_t T, int32_t rows, int32_t D) {
    if (T < 0 || rows < 1 || D < 1) return 0;
    return ln::bwd_workspace(T, rows, D).total;
}

}  // namespace rlf

extern "C" rlf_status rlf_linear_fwd(const void* x, int64_t T, int32_t D, int64_t x_stride, const void* W, int32_t N, const void* bias,
                                     rlf_dtype bias_dt, int act, int gated, const void* residual, int64_t residual_stride, void* y_out,
                                     rlf_dtype y_dt, void* pre_out, int32_t* dev_status, rlf_stream_t stream) {
    using namespace rlf;
    using namespace rlf::ln;
    if ((y_dt != RLF_BF16 && y_dt != RLF_F32) || (bias && bias_dt != RLF_BF16 && bias_dt != RLF_F32)) return RLF_ERR_DTYPE;
    rlf_status st = check_linear(T, D, N, act, gated);
    if (st != RLF_OK) return st;
    if (x_stride < D || (residual && residual_stride < N)) return RLF_ERR_SHAPE;
    if (T == 0) return RLF_OK;
    if (!x || !W || !y_out) return RLF_ERR_NULL;
    const size_t osz = y_dt == RLF_F32 ? 4 : 2;
    if (!aligned(x, 16) || !aligned(W, 16) || x_stride % 8 != 0 || !aligned(bias, bias_dt == RLF_F32 ? 4 : 2) || !aligned(residual, osz) ||
        !aligned(y_out, osz) || !aligned(pre_out, 2) || !aligned(dev_status, 4))
        return RLF_ERR_ALIGN;
    st = check_arch();
    if (st != RLF_OK) return st;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    Epilogue e = {};
    e.act = act; e.gated = gated; e.N = N; e.bias = bias; e.bias_bf16 = bias_dt == RLF_BF16;
    e.res = residual; e.res_stride = residual_stride; e.out = y_out; e.out_stride = N; e.out_f32 = y_dt == RLF_F32;
    e.pre = static_cast<__nv_bfloat16*>(pre_out); e.pre_stride = gated ? 2ll * N : N;
    e.vec_out = rows_aligned(y_out, N, (int)osz);
    e.vec_res = !residual || rows_aligned(residual, residual_stride, (int)osz);
    e.vec_pre = rows_aligned(pre_out, N, 2);
    if (!gated && N <= kFewOutputs) {
        const __nv_bfloat16* xb = static_cast<const __nv_bfloat16*>(x);
        const __nv_bfloat16* wb = static_cast<const __nv_bfloat16*>(W);
        long long xs = x_stride, tokens = T;
        void* args[] = {&xb, &xs, &wb, &tokens, &D, &e};
        const bool two = T >= 8ll * 2 * sm_count();
        return launch(two ? few_fwd_kernel<2>(N) : few_fwd_kernel<1>(N), dim3((unsigned)div_up(T, two ? 16 : 8)), dim3(256), 0, 1, args, s);
    }
    return product({{x, x_stride, 0}, {W, D, 0}, T, D, e}, dev_status, s);
}

extern "C" rlf_status rlf_linear_bwd(const void* grad_y, rlf_dtype grad_y_dt, int64_t grad_y_stride, const void* pre, const void* x, int64_t T,
                                     int32_t D, int64_t x_stride, const void* W, int32_t N, int act, int gated, void* grad_x, void* grad_W,
                                     rlf_dtype grad_W_dt, float* grad_bias, int accumulate, void* workspace, size_t workspace_bytes,
                                     int32_t* dev_status, rlf_stream_t stream) {
    using namespace rlf;
    using namespace rlf::ln;
    if ((grad_y_dt != RLF_BF16 && grad_y_dt != RLF_F32) || (grad_W && grad_W_dt != RLF_BF16 && grad_W_dt != RLF_F32)) return RLF_ERR_DTYPE;
    rlf_status st = check_linear(T, D, N, act, gated);
    if (st != RLF_OK) return st;
    if (x_stride < D || grad_y_stride < N) return RLF_ERR_SHAPE;
    if (accumulate && grad_W && grad_W_dt != RLF_F32) return RLF_ERR_UNSUPPORTED;
    const bool need_pre = act != RLF_ACT_NONE || gated;
    const int rows = gated ? 2 * N : N;
    if (T > 0 && (!grad_y || (need_pre && !pre) || (grad_W && !x) || (grad_x && !W))) return RLF_ERR_NULL;
    const size_t ysz = grad_y_dt == RLF_F32 ? 4 : 2, wsz = grad_W_dt == RLF_F32 ? 4 : 2;
    if (!aligned(grad_y, ysz) || !aligned(pre, 2) || !aligned(x, 16) || x_stride % 8 != 0 || !aligned(W, 16) || !aligned(grad_x, 16) ||
        !aligned(grad_W, grad_W ? wsz : 1) || !aligned(grad_bias, 4) || !aligned(dev_status, 4))
        return RLF_ERR_ALIGN;
    if (T > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < linear_bwd_workspace_bytes(T, rows, D))) return RLF_ERR_WORKSPACE;
    st = check_arch();
    if (st != RLF_OK) return st;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (T == 0) {
        // no tokens: the weights' gradients are zero (or what was accumulated before)
        if (!accumulate && grad_W && cudaMemsetAsync(grad_W, 0, (size_t)rows * (size_t)D * wsz, s) != cudaSuccess) return RLF_ERR_CUDA;
        if (!accumulate && grad_bias && cudaMemsetAsync(grad_bias, 0, (size_t)rows * 4, s) != cudaSuccess) return RLF_ERR_CUDA;
        return RLF_OK;
    }
    if (!grad_x && !grad_W && !grad_bias) return RLF_OK;
    const BwdWs ws = bwd_workspace(T, rows, D);
    char* base = static_cast<char*>(workspace);
    float* part_b = grad_bias ? reinterpret_cast<float*>(base + ws.part_b) : nullptr;
    const int slices = token_slices(T);
    const long long per_slice = (T + slices - 1) / slices;
    const int used = (int)((T + per_slice - 1) / per_slice);

    if (!gated && N <= kFewOutputs) {
        FewBwd p = {};
        p.dy = grad_y; p.dy_stride = grad_y_stride; p.dy_f32 = grad_y_dt == RLF_F32; p.act = act;
        p.pre = need_pre ? static_cast<const __nv_bfloat16*>(pre) : nullptr;
        p.x = static_cast<const __nv_bfloat16*>(x); p.x_stride = x_stride; p.W = static_cast<const __nv_bfloat16*>(W);
        p.dx = static_cast<__nv_bfloat16*>(grad_x); p.part_w = grad_W ? reinterpret_cast<float*>(base + ws.part_w) : nullptr; p.part_b = part_b;
        p.T = T; p.rows = per_slice; p.D = D;
        int nx = 1;
        while (nx < 256 && nx * 8 < D) nx *= 2;
        // as many slices as make whole generations of three CTAs per SM, within what the workspace holds
        const int columns = div_up(D, nx * 8);
        int parts = 3 * sm_count() / columns;
        if (parts > few_slices(T)) parts = few_slices(T);
        if (parts < 1) parts = 1;
        p.rows = (T + parts - 1) / parts;
        parts = div_up(T, p.rows);
        if (!ws.holds(0, p.part_b ? (size_t)parts * N * 4 : 0, p.part_w ? (size_t)parts * N * (size_t)D * 4 : 0)) return RLF_ERR_WORKSPACE;
        void* args[] = {&p};
        st = launch(few_bwd_kernel(N), dim3((unsigned)columns, (unsigned)parts), dim3(nx, 256 / nx), 0, 1, args, s);
        if (st != RLF_OK) return st;
        return launch_join(parts, accumulate, p.part_w, (long long)N * D, grad_W, grad_W_dt == RLF_F32, part_b, N, grad_bias, s);
    }

    // gz: grad_y itself where nothing is to be done to it and TMA can read it
    const bool in_place = !need_pre && grad_y_dt == RLF_BF16 && rows_aligned(grad_y, grad_y_stride, 2);
    Operand gz = {grad_y, grad_y_stride, 0};
    if (!in_place) gz = {base + ws.gz, up8(rows), 0};
    if (!ws.holds(in_place ? 0 : (size_t)T * (size_t)up8(rows) * 2, (size_t)used * rows * 4, 0)) return RLF_ERR_WORKSPACE;
    if ((!in_place && (grad_x || grad_W)) || grad_bias) {
        PreGrad p = {};
        p.dy = grad_y; p.dy_stride = grad_y_stride; p.dy_f32 = grad_y_dt == RLF_F32; p.act = act; p.gated = gated;
        p.pre = need_pre ? static_cast<const __nv_bfloat16*>(pre) : nullptr;
        p.gz = !in_place && (grad_x || grad_W) ? reinterpret_cast<__nv_bfloat16*>(base + ws.gz) : nullptr;
        const bool direct = used == 1 && !accumulate;
        p.gz_stride = up8(rows); p.part_b = direct ? grad_bias : part_b; p.T = T; p.rows = per_slice; p.N = N;
        const bool wide = N % 8 == 0 && rows_aligned(grad_y, grad_y_stride, (int)ysz) && (!p.pre || aligned(p.pre, 16));
        const dim3 grid((unsigned)((N + (wide ? 255 : 31)) / (wide ? 256 : 32)), (unsigned)used);
        const void* kernel = wide ? (gated ? pregrad_kernel<8, true>(act) : pregrad_kernel<8, false>(act))
                                  : (gated ? pregrad_kernel<1, true>(act) : pregrad_kernel<1, false>(act));
        void* args[] = {&p};
        st = launch(kernel, grid, dim3(32, 8), 0, 1, args, s);
        if (st == RLF_OK && grad_bias && !direct) st = launch_join(used, accumulate, nullptr, 0, nullptr, 1, part_b, rows, grad_bias, s);
        if (st != RLF_OK) return st;
    }
    Product gx = {gz, {W, D, 1}, T, rows, {}}, gw = {{gz.at, gz.stride, 1}, {x, x_stride, 1}, rows, T, {}};
    gx.e.N = D; gx.e.out = grad_x; gx.e.out_stride = D; gx.e.vec_out = gx.e.vec_res = 1;
    gw.e.N = D; gw.e.out = grad_W; gw.e.out_stride = D; gw.e.out_f32 = grad_W_dt == RLF_F32;
    gw.e.vec_out = gw.e.vec_res = rows_aligned(grad_W, D, (int)wsz);
    if (accumulate) { gw.e.res = grad_W; gw.e.res_stride = D; }
    if (grad_x && grad_W) return both_products(gx, gw, dev_status, s);
    if (grad_x) return product(gx, dev_status, s);
    return grad_W ? product(gw, dev_status, s) : RLF_OK;
}

extern "C" rlf_status rlf_tune_linear(int form, int tile, int split) {
    if (form < 0 || form > 3 || tile < 0 || tile > 256 || (tile != 16 && tile != 32 && tile % 64 != 0) || split < 0 || split > 8) return RLF_ERR_SHAPE;
    rlf::ln::g_form = form;
    rlf::ln::g_tile = tile;
    rlf::ln::g_split = split;
    return RLF_OK;
}
