// Softmax cross entropy over materialised logits, forward and backward, with label smoothing and a
// z-loss: the supervised counterpart of the log-prob + loss kernels.  Per row with loss weight,
// y = ids[t], N the number of such rows (or the caller's count), eps the smoothing, zeta the z-loss:
//   lse = log sum_v exp z_v
//   l   = (1 - eps) (lse - z_y) + eps (lse - mean_v z_v) + zeta lse^2
//   dL/dz_v = (1/N) [ (1 + 2 zeta lse) p_v - eps/V - (1 - eps) [v = y] ],   p = softmax(z)
// The target column is formed as (1/N) [ 2 zeta lse p_y - S'/S + eps - eps/V ], S' the sum over the
// other columns, so that it keeps its digits when p_y rounds to one.
//
// Kernels, in launch order: ce_count_kernel (only without a given count), the row kernel (writes logp,
// lse, the row's loss terms and grad_logits), ce_loss_kernel (fp64 sums in a fixed order).
// Rows without loss weight are not read at all; their gradient is written as zeros.
#include <map>
#include <mutex>
#include <tuple>

#include "common.cuh"
#include "row.cuh"

namespace rlf {
namespace ce {

// workspace: [0] int64 count of rows with loss weight; [256 ..) one float4 of loss terms per token:
// {lse - z_y, lse - mean z (0 without smoothing), lse, 1 if the row counts}
constexpr size_t kWsTermsOff = 256;

struct RowParams {
    const void* logits;
    void* grad;                 // nullable
    long long stride;           // elements
    long long T;
    int V;
    const int32_t* ids;
    const uint8_t* mask;        // nullable: every row counts
    const long long* denom;     // device count of rows with loss weight
    float* logp_out;
    float* lse_out;             // nullable
    float4* terms;
    int32_t* dev_status;
    float eps, zeta;
};

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

constexpr int kTargetNone = -1, kTargetBad = -2;
// target id of a row, kTargetNone for a row without loss weight (its id is not looked at), kTargetBad
// for one whose id lies outside the vocabulary
__device__ __forceinline__ int row_target(const int32_t* ids, const uint8_t* mask, long long t, int V) {
    if (mask && mask[t] == 0) return kTargetNone;
    const int y = ids[t];
    return (y >= 0 && y < V) ? y : kTargetBad;
}

// what a row leaves behind once its statistics are known; returns whether it takes part
struct RowStats {
    float lse, logp, smooth;
    bool ok;
};
__device__ __forceinline__ RowStats row_stats(float M, float S, float zy, float mean_z, float eps) {
    RowStats r;
    const float ln_s = logf(S);
    r.lse = M + ln_s;
    r.logp = (zy - M) - ln_s;
    r.smooth = eps > 0.0f ? (M - mean_z) + ln_s : 0.0f;
    r.ok = (M > -INFINITY) && (M < INFINITY) && (S > 0.0f) && (S < INFINITY) && (fabsf(r.lse) < INFINITY) &&
           (fabsf(r.logp) < INFINITY) && (fabsf(r.smooth) < INFINITY);
    return r;
}
__device__ __forceinline__ void write_row(const RowParams& p, long long t, const RowStats& r) {
    const float nan = __int_as_float(0x7fc00000);
    p.logp_out[t] = r.ok ? r.logp : nan;
    if (p.lse_out) p.lse_out[t] = r.ok ? r.lse : nan;
    p.terms[t] = r.ok ? make_float4(-r.logp, r.smooth, r.lse, 1.0f) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
}

// Any type, vocabulary and alignment: one CTA per row, three sweeps (max; sums; gradient), of which the
// later ones are served by L2 when the row fits there.
constexpr int kGenThreads = 256;
template <typename T>
__global__ void __launch_bounds__(kGenThreads)
ce_row_general_kernel(const RowParams p) {
    __shared__ float red[2][kGenThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const long long N = *p.denom;
    const float inv_n = 1.0f / (float)(N > 1 ? N : 1), inv_v = 1.0f / (float)p.V;
    int status = 0;
    auto gather = [&](float a, float b, bool take_max, float& ra, float& rb) {
        if (lane == 0) { red[0][warp] = a; red[1][warp] = b; }
        __syncthreads();
        ra = red[0][0];
        rb = red[1][0];
        for (int w = 1; w < kGenThreads / 32; ++w) {
            ra = take_max ? fmaxf(ra, red[0][w]) : ra + red[0][w];
            rb += red[1][w];
        }
        __syncthreads();
    };
    for (long long t = blockIdx.x; t < p.T; t += gridDim.x) {
        const T* z = static_cast<const T*>(p.logits) + t * p.stride;
        T* g = p.grad ? static_cast<T*>(p.grad) + t * p.stride : nullptr;
        const int y = row_target(p.ids, p.mask, t, p.V);
        RowStats r = {};
        float M = 0.0f, S = 1.0f, others = 0.0f;
        if (y >= 0) {
            const float zy = to_f<T>(z[y]);
            float m = -INFINITY, dummy;
            bool nan = false;
            for (int v = tid; v < p.V; v += kGenThreads) {
                const float zv = to_f<T>(z[v]);
                m = fmaxf(m, zv);
                nan |= zv != zv;
            }
            m = warp_max(nan ? INFINITY : m);          // a NaN must not pass for a finite row
            gather(m, 0.0f, true, M, dummy);
            const float Ms = (M == -INFINITY) ? 0.0f : M;
            float s = 0.0f, q = 0.0f;
            for (int v = tid; v < p.V; v += kGenThreads) {
                const float zv = to_f<T>(z[v]);
                s += (v == y) ? 0.0f : ex2_approx((zv - Ms) * kLog2e);
                q = fmaf(zv, inv_v, q);
            }
            s = warp_sum(s);
            q = warp_sum(q);
            float Q;
            gather(s, q, false, others, Q);
            S = others + ex2_approx((zy - Ms) * kLog2e);
            r = row_stats(M, S, zy, Q, p.eps);
        }
        if (tid == 0) {
            write_row(p, t, r);
            if (y == kTargetBad) status |= RLF_DEV_BAD_TARGET;
            else if (y >= 0 && !r.ok) status |= RLF_DEV_NONFINITE;
        }
        if (g == nullptr) continue;
        if (!r.ok) {
            for (int v = tid; v < p.V; v += kGenThreads) g[v] = from_f<T>(0.0f);
            continue;
        }
        const float a = inv_n * (1.0f + 2.0f * p.zeta * r.lse) / S, u = inv_n * p.eps * inv_v;
        const float gy = inv_n * (2.0f * p.zeta * r.lse * ((S - others) / S) - others / S + p.eps) - u;
        for (int v = tid; v < p.V; v += kGenThreads)
            g[v] = from_f<T>(v == y ? gy : fmaf(a, ex2_approx((to_f<T>(z[v]) - M) * kLog2e), -u));
    }
    if (tid == 0 && status && p.dev_status) atomicOr(p.dev_status, status);
}

// ---------------------------------------------------------------------------------------------
// Cluster row kernel: a thread-block cluster owns one row at a time and holds the WHOLE row in registers
// (NV 16-byte vectors per thread), so it crosses HBM once in each direction.
//   * cp.async brings a thread's vectors into its own slots of a staging buffer and the slots are queued again
//     with the cluster's next row as soon as they are in registers, so loads of row r + 1 run under row r;
//   * max, exponentials and sums per warp; every warp sends its (max, sum) to every CTA of the cluster as
//     asynchronous distributed-shared-memory stores that credit an mbarrier, and waits (bounded) on its own
//     CTA's mbarrier: no thread barrier and no fence in the loop;
//   * the exponentials replace the logits in the registers (bf16 logits: rounded to bf16, one rounding that the
//     gradient carries besides its own; fp32 logits: in fp32) and the gradient is one multiply-add per element.
// Bound by HBM: the exponential unit is used about half the time at the copy rate of bf16 rows.
// EDGE serves rows that start on no 16-byte boundary or whose length fills no vector: a row is then the aligned
// vectors that cover it, with the elements that are not its own set to -inf in the staging slot, and those two
// vectors' gradients stored element by element.  All loads stay inside the logits' own memory: the last vector
// is copied up to the row's end, and the first vector of the first row element by element (before it there may
// be nothing); another row's first vector starts in the row before it.
constexpr int kSmemBudget = 220 * 1024;
constexpr int stage_bytes(int threads, int nv) { return nv * threads * 16; }
constexpr int ctas_per_sm(int threads, int nv) {
    const int by_regs = 65536 / (64 * threads);
    const int by_smem = kSmemBudget / (stage_bytes(threads, nv) + 4096);
    const int m = by_regs < by_smem ? by_regs : by_smem;
    return m < 1 ? 1 : m;
}
// exponents of bf16 rows are formed by one multiply-add from a rounded -max log2 e; rows whose maximum is huge in
// magnitude subtract first
constexpr float kRobustAbove = 2048.0f;

struct ClusterParams {
    RowParams r;
    int per_cta_vec;            // vectors of a row per CTA of the cluster
    float inv_v;                // 1 / V
};

template <typename T> struct Elem;
template <> struct Elem<__nv_bfloat16> {
    static constexpr int kPer = 8;
    static __device__ __forceinline__ uint32_t neg_inf() { return 0xFF80FF80u; }
    static __device__ __forceinline__ void store_neg_inf(void* at) {
        asm volatile("st.shared.b16 [%0], %1;" :: "r"(smem_u32(at)), "h"((unsigned short)0xff80u) : "memory");
    }
};
template <> struct Elem<float> {
    static constexpr int kPer = 4;
    static __device__ __forceinline__ uint32_t neg_inf() { return 0xFF800000u; }
    static __device__ __forceinline__ void store_neg_inf(void* at) {
        asm volatile("st.shared.b32 [%0], %1;" :: "r"(smem_u32(at)), "r"(0xFF800000u) : "memory");
    }
};
__device__ __forceinline__ void cp_async16_part(void* smem_dst, const void* gmem_src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(smem_u32(smem_dst)), "l"(gmem_src), "r"(bytes) : "memory");
}

template <typename T, int THREADS, int NV, bool EDGE, int CMAX>
__global__ void __launch_bounds__(THREADS, ctas_per_sm(THREADS, NV))
ce_row_cluster_kernel(const ClusterParams cp) {
    const RowParams& p = cp.r;
    constexpr bool BF = sizeof(T) == 2;
    constexpr int VE = Elem<T>::kPer;
    constexpr int NWARPS = THREADS / 32;
    constexpr int MAXE = CMAX * NWARPS;
    extern __shared__ __align__(16) uint4 stage[];            // [NV][THREADS], slot (i, tid) private to thread tid
    __shared__ __align__(8) float2 pair_slot[2][MAXE];        // per row parity: every warp's (max, sum)
    __shared__ float mean_slot[2][MAXE];                      // ... its share of the mean logit (with smoothing)
    __shared__ float zy_slot[2];
    __shared__ __align__(16) uint4 edge_slot[EDGE ? 2 : 1];   // gradients of a row's first and last vector
    __shared__ __align__(8) unsigned long long row_bar[2];

    const int csize = (int)cluster_nctarank(), crank = (int)cluster_ctarank();
    const int cluster_id = blockIdx.x / csize, num_clusters = gridDim.x / csize;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int npairs = csize * NWARPS;
    const int vbeg = crank * cp.per_cta_vec + tid;            // this thread's vectors: vbeg + i THREADS
    const int vcap = (crank + 1) * cp.per_cta_vec;
    const bool smooth = p.eps > 0.0f;
    const int nrows = (int)p.T;

    // a row as aligned vectors: elements of its first vector that precede it, and its number of vectors
    auto row_head = [&](int row) -> int {
        if (!EDGE) return 0;
        return (int)((reinterpret_cast<uintptr_t>(p.logits) / sizeof(T) + (unsigned long long)((long long)row * p.stride)) % VE);
    };
    auto row_vecs = [&](int head) -> int { return EDGE ? (head + p.V + VE - 1) / VE : p.V / VE; };
    auto count_valid = [&](int nvec) -> int {
        const int vend = min(nvec, vcap);
        return vend > vbeg ? min(NV, (vend - vbeg + THREADS - 1) / THREADS) : 0;
    };
    // 1 / N, re-read where it is used: a register held across the passes costs more than an L1 hit
    auto weight = [&]() -> float {
        const long long N = *p.denom;
        return 1.0f / (float)(N > 1 ? N : 1);
    };
    const int nvalid_all = EDGE ? 0 : count_valid(p.V / VE);

    auto prefetch = [&](int row, bool have) {
        if (have) {
            const int head = row_head(row);
            const T* src = static_cast<const T*>(p.logits) + (long long)row * p.stride - head;
            const int nvec = row_vecs(head), nvalid = EDGE ? count_valid(nvec) : nvalid_all;
            const int last_bytes = EDGE ? (head + p.V - (nvec - 1) * VE) * (int)sizeof(T) : 16;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (i >= nvalid) continue;
                const int v = vbeg + i * THREADS;
                uint4* dst = stage + i * THREADS + tid;
                if (EDGE && v == 0 && head != 0 && row == 0) {
                    T* d = reinterpret_cast<T*>(dst);
                    for (int e = head; e < VE && e < head + p.V; ++e) d[e] = src[e];
                } else if (EDGE && v == nvec - 1) {
                    cp_async16_part(dst, src + (long long)v * VE, last_bytes);
                } else {
                    cp_async16_cg(dst, src + (long long)v * VE);
                }
            }
        }
        cp_async_commit();
    };

    if (tid == 0) {
        mbar_init(smem_u32(&row_bar[0]), 1);
        mbar_init(smem_u32(&row_bar[1]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    int y = cluster_id < nrows ? row_target(p.ids, p.mask, cluster_id, p.V) : kTargetNone;
    int y_next = cluster_id + num_clusters < nrows ? row_target(p.ids, p.mask, cluster_id + num_clusters, p.V) : kTargetNone;
    prefetch(cluster_id, y >= 0);
    // every CTA of the cluster is running before any peer may address its shared memory
    cluster_sync_all();

    const uint32_t row_bytes = (uint32_t)npairs * (smooth ? 12u : 8u) + 4u;
    int status = 0;
    int it = 0;                          // rows exchanged so far: rows without loss weight need no exchange
    bool gave_up = false;
    for (int k = cluster_id; k < nrows; k += num_clusters) {
        const int next = k + num_clusters;
        const int head = row_head(k);
        const int nvec = row_vecs(head), nvalid = EDGE ? count_valid(nvec) : nvalid_all;
        RowStats st = {};
        float M = 0.0f, S = 1.0f, others = 0.0f, m_ws = 0.0f;
        uint4 d[NV];
        if (y >= 0) {
            const int parity = it & 1;
            const uint32_t bar = smem_u32(&row_bar[parity]);
            cp_async_wait_all();
            if (tid == 0) mbar_arrive_expect_tx(bar, row_bytes);
            if (EDGE) {
                // what lies in the first and the last vector beside the row is not part of it
                const int tail = head + p.V - (nvec - 1) * VE;          // elements of the last vector up to the row's end
                if (vbeg == 0 && nvalid > 0)
                    for (int e = 0; e < head; ++e) Elem<T>::store_neg_inf(reinterpret_cast<T*>(&stage[tid]) + e);
                const int lrel = nvec - 1 - vbeg;
                if (lrel >= 0 && (lrel & (THREADS - 1)) == 0 && lrel / THREADS < nvalid)
                    for (int e = tail; e < VE; ++e) Elem<T>::store_neg_inf(reinterpret_cast<T*>(&stage[lrel + tid]) + e);
            }
            // the mean logit, from the staging slots (the row's own elements only)
            if (smooth) {
                float q = 0.0f;
                const float inv_v = cp.inv_v;
#pragma unroll 2
                for (int i = 0; i < nvalid; ++i) {
                    const int v = vbeg + i * THREADS;
                    const uint4 x = stage[i * THREADS + tid];
                    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
                    if (EDGE && (v == 0 || v == nvec - 1)) {
                        const T* e = reinterpret_cast<const T*>(&stage[i * THREADS + tid]);
                        for (int j = 0; j < VE; ++j)
                            if (v * VE + j >= head && v * VE + j < head + p.V) q = fmaf(to_f<T>(e[j]), inv_v, q);
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if (BF) {
                                q = fmaf(bf_lo(w[j]), inv_v, q);
                                q = fmaf(bf_hi(w[j]), inv_v, q);
                            } else {
                                q = fmaf(__uint_as_float(w[j]), inv_v, q);
                            }
                        }
                    }
                }
                q = warp_sum(q);
                if (lane < csize)
                    st_async_f1(smem_u32(&mean_slot[parity][crank * NWARPS + warp]), bar, (uint32_t)lane, q);
            }
            // the owner of the target column sends its logit to every CTA and takes it out of the sums: the
            // target's gradient needs the sum over the OTHER columns
            const int ye = y + head, yrel = ye / VE - vbeg;
            const bool own_y = yrel >= 0 && (yrel & (THREADS - 1)) == 0 && yrel / THREADS < nvalid;
            if (own_y) {
                T* sv = reinterpret_cast<T*>(&stage[yrel + tid]) + ye % VE;
                const float zt = to_f<T>(*sv);
                for (int r = 0; r < csize; ++r) st_async_f1(smem_u32(&zy_slot[parity]), bar, (uint32_t)r, zt);
                Elem<T>::store_neg_inf(sv);
            }
            const uint32_t ninf = Elem<T>::neg_inf();
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (i < nvalid) d[i] = stage[i * THREADS + tid];
                else d[i] = make_uint4(ninf, ninf, ninf, ninf);
            }
            float m_w;
            if (BF) {
                uint32_t mx = ninf;
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    mx = max_bf16x2(mx, max_bf16x2(max_bf16x2(d[i].x, d[i].y), max_bf16x2(d[i].z, d[i].w)));
                m_w = fmaxf(bf_lo(mx), bf_hi(mx));
            } else {
                m_w = -INFINITY;
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    m_w = fmaxf(m_w, fmaxf(fmaxf(__uint_as_float(d[i].x), __uint_as_float(d[i].y)),
                                           fmaxf(__uint_as_float(d[i].z), __uint_as_float(d[i].w))));
            }
            prefetch(next, y_next >= 0);             // the slots are in registers: queue the next row
            m_w = ord2f(__reduce_max_sync(0xffffffffu, f2ord(m_w)));
            m_ws = (m_w == -INFINITY) ? 0.0f : m_w;
            float s0 = 0.0f, s1 = 0.0f;
            if (BF && fabsf(m_ws) <= kRobustAbove) {
                const float off = -m_ws * kLog2e;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    uint32_t* w = reinterpret_cast<uint32_t*>(&d[i]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float e0 = ex2_approx(fmaf(bf_lo(w[j]), kLog2e, off)), e1 = ex2_approx(fmaf(bf_hi(w[j]), kLog2e, off));
                        s0 += e0;
                        s1 += e1;
                        w[j] = pack_bf16x2(e0, e1);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    uint32_t* w = reinterpret_cast<uint32_t*>(&d[i]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (BF) {
                            const float e0 = ex2_approx((bf_lo(w[j]) - m_ws) * kLog2e), e1 = ex2_approx((bf_hi(w[j]) - m_ws) * kLog2e);
                            s0 += e0;
                            s1 += e1;
                            w[j] = pack_bf16x2(e0, e1);
                        } else {
                            const float e0 = ex2_approx((__uint_as_float(w[j]) - m_ws) * kLog2e);
                            if (j & 1) s1 += e0;
                            else s0 += e0;
                            w[j] = __float_as_uint(e0);
                        }
                    }
                }
            }
            const float s_w = warp_sum(s0 + s1);
            if (lane < csize) st_async_f2(smem_u32(&pair_slot[parity][crank * NWARPS + warp]), bar, (uint32_t)lane, m_w, s_w);
            if (!gave_up && !mbar_wait_bounded(bar, (uint32_t)(it >> 1) & 1u)) {
                gave_up = true;
                status |= RLF_DEV_TIMEOUT;
            }
            ++it;
            // merge all warps' pairs of the row, lanes in parallel, identically in every warp
            M = -INFINITY;
            float2 e[(MAXE + 31) / 32];
            float Q = 0.0f;
#pragma unroll
            for (int j = 0; j < (MAXE + 31) / 32; ++j) {
                const int i = lane + 32 * j;
                e[j] = i < npairs ? pair_slot[parity][i] : make_float2(-INFINITY, 0.0f);
                if (smooth && i < npairs) Q += mean_slot[parity][i];
                M = fmaxf(M, e[j].x);
            }
            M = ord2f(__reduce_max_sync(0xffffffffu, f2ord(M)));
            const float zy = zy_slot[parity];
            M = fmaxf(M, zy);
            others = 0.0f;
#pragma unroll
            for (int j = 0; j < (MAXE + 31) / 32; ++j)
                if (e[j].x != -INFINITY) others += e[j].y * ex2_approx((e[j].x - M) * kLog2e);
            others = warp_sum(others);
            if (smooth) Q = warp_sum(Q);
            S = others + ex2_approx((zy - M) * kLog2e);
            st = row_stats(M, S, zy, Q, p.eps);
        } else {
            prefetch(next, y_next >= 0);
        }
        if (crank == 0 && tid == 0) {
            write_row(p, k, st);
            if (y == kTargetBad) status |= RLF_DEV_BAD_TARGET;
            else if (y >= 0 && !st.ok) status |= RLF_DEV_NONFINITE;
        }
        if (p.grad != nullptr) {
            T* g_row = static_cast<T*>(p.grad) + (long long)k * p.stride;
            uint4* dst = reinterpret_cast<uint4*>(g_row - head) + vbeg;
            float a = 0.0f, u = 0.0f;
            if (st.ok) {
                // entries are a e - u: the registers hold 2^((z - m_w) log2e)
                const float inv_n = weight();
                a = inv_n * (1.0f + 2.0f * p.zeta * st.lse) / S * ex2_approx((m_ws - M) * kLog2e);
                u = inv_n * p.eps * cp.inv_v;
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (i >= nvalid) continue;
                uint4 o = make_uint4(0u, 0u, 0u, 0u);
                if (st.ok) {
                    uint32_t* w = reinterpret_cast<uint32_t*>(&o);
                    const uint32_t* x = reinterpret_cast<const uint32_t*>(&d[i]);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        w[j] = BF ? pack_bf16x2(fmaf(bf_lo(x[j]), a, -u), fmaf(bf_hi(x[j]), a, -u))
                                  : __float_as_uint(fmaf(__uint_as_float(x[j]), a, -u));
                }
                const int v = vbeg + i * THREADS;
                if (EDGE && v == 0) edge_slot[0] = o;
                else if (EDGE && v == nvec - 1) edge_slot[1] = o;
                else st_stream(dst + i * THREADS, o);
            }
            if (EDGE) {
                // the row's own elements of its first and last vector, by the thread that has just put them down
                const int lrel = nvec - 1 - vbeg;
                const bool first = vbeg == 0 && nvalid > 0;
                const bool last = nvec > 1 && lrel >= 0 && (lrel & (THREADS - 1)) == 0 && lrel / THREADS < nvalid;
                for (int side = 0; side < 2; ++side) {
                    if (!(side == 0 ? first : last)) continue;
                    const T* o = reinterpret_cast<const T*>(&edge_slot[side]);
                    const int base = (side == 0 ? 0 : nvec - 1) * VE - head;        // column of the vector's element 0
                    for (int e = 0; e < VE; ++e)
                        if (base + e >= 0 && base + e < p.V) g_row[base + e] = o[e];
                }
            }
            if (st.ok) {
                // the target id again, by its owner (not held in a register across the passes)
                const int yt = p.ids[k], ye = yt + head, yrel = ye / VE - vbeg;
                if (yrel >= 0 && (yrel & (THREADS - 1)) == 0 && yrel / THREADS < nvalid) {
                    const float py = 1.0f - others / S;
                    g_row[yt] = from_f<T>(weight() * (2.0f * p.zeta * st.lse * py - others / S + p.eps) - u);
                }
            }
        }
        y = y_next;
        // needed when that row's loads are queued, in the next iteration
        y_next = (long long)next + num_clusters < nrows ? row_target(p.ids, p.mask, next + num_clusters, p.V) : kTargetNone;
    }
    if (status && p.dev_status) atomicOr(p.dev_status, status);
    // a warp that gave up: peers' stores of the last rows may still be on their way into this CTA
    if (gave_up)
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    cluster_sync_all();                  // no CTA leaves while a peer could still address its shared memory
}

// ---- launch shape ---------------------------------------------------------------------------
typedef void (*RowKernel)(const ClusterParams);
struct RowShape { int cluster, threads, nv; };

template <typename T, int THREADS, bool EDGE, int CMAX>
static RowKernel kernel_for_nv(int nv) {
    switch (nv) {
        case 1: return ce_row_cluster_kernel<T, THREADS, 1, EDGE, CMAX>;
        case 2: return ce_row_cluster_kernel<T, THREADS, 2, EDGE, CMAX>;
        case 3: return ce_row_cluster_kernel<T, THREADS, 3, EDGE, CMAX>;
        case 4: return ce_row_cluster_kernel<T, THREADS, 4, EDGE, CMAX>;
        case 5: return ce_row_cluster_kernel<T, THREADS, 5, EDGE, CMAX>;
        case 6: return ce_row_cluster_kernel<T, THREADS, 6, EDGE, CMAX>;
        case 7: return ce_row_cluster_kernel<T, THREADS, 7, EDGE, CMAX>;
        case 8: return ce_row_cluster_kernel<T, THREADS, 8, EDGE, CMAX>;
        case 9: return ce_row_cluster_kernel<T, THREADS, 9, EDGE, CMAX>;
        case 10: return ce_row_cluster_kernel<T, THREADS, 10, EDGE, CMAX>;
    }
    return nullptr;
}
// the wider shapes hold rows of 20481 vectors and more: 6 to 10 vectors per thread
template <typename T, int THREADS, bool EDGE>
static RowKernel wide_kernel_for_nv(int nv) {
    switch (nv) {
        case 6: return ce_row_cluster_kernel<T, THREADS, 6, EDGE, 16>;
        case 7: return ce_row_cluster_kernel<T, THREADS, 7, EDGE, 16>;
        case 8: return ce_row_cluster_kernel<T, THREADS, 8, EDGE, 16>;
        case 9: return ce_row_cluster_kernel<T, THREADS, 9, EDGE, 16>;
        case 10: return ce_row_cluster_kernel<T, THREADS, 10, EDGE, 16>;
    }
    return nullptr;
}
template <typename T, bool EDGE>
static RowKernel row_kernel(const RowShape& sh) {
    if (sh.cluster <= 8) return kernel_for_nv<T, 256, EDGE, 8>(sh.nv);
    return sh.threads == 256 ? wide_kernel_for_nv<T, 256, EDGE>(sh.nv) : wide_kernel_for_nv<T, 512, EDGE>(sh.nv);
}

// 16-byte vectors of a row per CTA: an even split rounded up to whole 128-byte lines
static int per_cta_vectors(int nvec, int cluster) { return (((nvec + cluster - 1) / cluster) + 7) & ~7; }

// The smallest cluster of 256-thread CTAs that holds a row of nvec vectors with at most 10 per thread (1, 2, 4
// or 8 CTAs; then 10 and 16, beyond the portable size), then 16 CTAs of 512 threads.  false: no shape holds it.
static bool pick_shape(int nvec, RowShape* out) {
    static const int clusters[] = {1, 2, 4, 8, 10, 16};
    for (int th = 256; th <= 512; th *= 2)
        for (int c : clusters) {
            if (th == 512 && c != 16) continue;
            int nv = (per_cta_vectors(nvec, c) + th - 1) / th;
            if (nv > 10) continue;
            if (c > 8 && nv < 6) nv = 6;
            *out = {c, th, nv};
            return true;
        }
    return false;
}

static void cluster_config(cudaLaunchConfig_t* cfg, cudaLaunchAttribute* at, int grid, const RowShape& sh, cudaStream_t s) {
    *cfg = cudaLaunchConfig_t{};
    cfg->gridDim = dim3(grid);
    cfg->blockDim = dim3(sh.threads);
    cfg->dynamicSmemBytes = (size_t)stage_bytes(sh.threads, sh.nv);
    cfg->stream = s;
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = sh.cluster;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    cfg->attrs = at;
    cfg->numAttrs = 1;
}

// clusters of this shape that are resident at once (0: the device takes none); cached per device, kernel and
// cluster size, and opts the kernel in to its staging buffer on the way
static int resident_clusters(RowKernel k, const RowShape& sh) {
    static std::mutex mu;
    static std::map<std::tuple<int, RowKernel, int>, int> cache;
    int dev = 0;
    cudaGetDevice(&dev);
    std::lock_guard<std::mutex> lock(mu);
    const auto key = std::make_tuple(dev, k, sh.cluster);
    const auto hit = cache.find(key);
    if (hit != cache.end()) return hit->second;
    int n = 0;
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute at[1];
    cluster_config(&cfg, at, sh.cluster * 148 * 8, sh, nullptr);
    if (cudaFuncSetAttribute((const void*)k, cudaFuncAttributeMaxDynamicSharedMemorySize, stage_bytes(sh.threads, sh.nv)) != cudaSuccess ||
        (sh.cluster > 8 && cudaFuncSetAttribute((const void*)k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) ||
        cudaOccupancyMaxActiveClusters(&n, (void*)k, &cfg) != cudaSuccess) {
        cudaGetLastError();
        n = 0;
    }
    cache[key] = n;
    return n;
}

// A cluster handles about two dozen rows before it retires (whole generations of what is resident at once): with
// one generation of persistent clusters all of them load, then all of them store, in step for the whole launch.
constexpr int kRowsPerCluster = 24;
static int clusters_for(int resident, long long rows) {
    const long long per_generation = (long long)resident * kRowsPerCluster;
    long long nc = (rows + per_generation - 1) / per_generation * resident;
    if (nc > rows) nc = rows;
    return (int)(nc < (1 << 26) ? nc : (1 << 26));
}

// number of rows with loss weight (one CTA; integer sum)
__global__ void __launch_bounds__(1024)
ce_count_kernel(const uint8_t* __restrict__ mask, long long T, long long* __restrict__ count) {
    __shared__ int red[32];
    int c = 0;
    if (mask == nullptr) {
        if (threadIdx.x == 0) *count = T;
        return;
    }
    const long long head = min(T, (long long)((16 - (reinterpret_cast<uintptr_t>(mask) & 15)) & 15));
    for (long long t = threadIdx.x; t < head; t += 1024) c += mask[t] != 0;
    const uint4* m4 = reinterpret_cast<const uint4*>(mask + head);
    const long long n4 = (T - head) / 16;
    for (long long i = threadIdx.x; i < n4; i += 1024) {
        const uint4 v = m4[i];
        // 0xff in every non-zero byte
        c += (__popc(__vcmpne4(v.x, 0u)) + __popc(__vcmpne4(v.y, 0u)) + __popc(__vcmpne4(v.z, 0u)) +
              __popc(__vcmpne4(v.w, 0u))) >> 3;
    }
    for (long long t = head + 16 * n4 + threadIdx.x; t < T; t += 1024) c += mask[t] != 0;
    c = __reduce_add_sync(0xffffffffu, c);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = c;
    __syncthreads();
    if (threadIdx.x == 0) {
        long long s = 0;
        for (int w = 0; w < 32; ++w) s += red[w];
        *count = s;
    }
}

// loss terms -> loss_out[4] in fp64.  Every thread adds its tokens in index order, then a fixed tree: the
// same order on every launch.
constexpr int kLossThreads = 1024;
__global__ void __launch_bounds__(kLossThreads)
ce_loss_kernel(const float4* __restrict__ terms, long long T, const long long* __restrict__ denom, float eps, float zeta,
               double* __restrict__ loss_out) {
    __shared__ double red[3][kLossThreads / 32];
    double a = 0.0, b = 0.0, c = 0.0;
    for (long long t = threadIdx.x; t < T; t += kLossThreads) {
        const float4 r = terms[t];
        if (r.w == 0.0f) continue;
        a += (double)r.x;
        b += (double)r.y;
        c += (double)r.z * (double)r.z;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, o);
        b += __shfl_xor_sync(0xffffffffu, b, o);
        c += __shfl_xor_sync(0xffffffffu, c, o);
    }
    if ((threadIdx.x & 31) == 0) {
        red[0][threadIdx.x >> 5] = a;
        red[1][threadIdx.x >> 5] = b;
        red[2][threadIdx.x >> 5] = c;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        a = b = c = 0.0;
        for (int w = 0; w < kLossThreads / 32; ++w) {
            a += red[0][w];
            b += red[1][w];
            c += red[2][w];
        }
        const long long N = *denom;
        const double nd = (double)(N > 1 ? N : 1);
        loss_out[0] = ((1.0 - (double)eps) * a + (double)eps * b + (double)zeta * c) / nd;
        loss_out[1] = a / nd;
        loss_out[2] = b / nd;
        loss_out[3] = c / nd;
    }
}

// The cluster kernel wherever a shape holds the row and the gradient rows sit like the logits rows within their
// 16-byte vectors; otherwise (rows beyond 81,920 vectors, a gradient buffer of another alignment) the general one,
// which reads a row three times (V = 151936 bf16, 8192 rows: 3.69 ms against 1.07).
static rlf_status launch_rows(const RowParams& p, rlf_dtype dt, cudaStream_t s) {
    const size_t esz = dt == RLF_BF16 ? 2 : 4;
    const int ve = (int)(16 / esz);
    const bool edge = p.V % ve != 0 || p.stride % ve != 0 || !aligned(p.logits, 16);
    const bool same = !p.grad || (reinterpret_cast<uintptr_t>(p.grad) - reinterpret_cast<uintptr_t>(p.logits)) % 16 == 0;
    // a row on no boundary may take one vector more than its length fills
    const long long nvec = edge ? ((long long)p.V + 2 * ve - 2) / ve : p.V / ve;
    RowShape sh;
    if (same && nvec < (1 << 24) && pick_shape((int)nvec, &sh)) {
        const RowKernel k = dt == RLF_BF16 ? (edge ? row_kernel<__nv_bfloat16, true>(sh) : row_kernel<__nv_bfloat16, false>(sh))
                                           : (edge ? row_kernel<float, true>(sh) : row_kernel<float, false>(sh));
        const int resident = k ? resident_clusters(k, sh) : 0;
        if (resident > 0) {
            ClusterParams cp;
            cp.r = p;
            cp.per_cta_vec = per_cta_vectors((int)nvec, sh.cluster);
            cp.inv_v = 1.0f / (float)p.V;
            cudaLaunchConfig_t cfg;
            cudaLaunchAttribute at[1];
            cluster_config(&cfg, at, clusters_for(resident, p.T) * sh.cluster, sh, s);
            if (cudaLaunchKernelEx(&cfg, k, cp) != cudaSuccess) {
                cudaGetLastError();
                return RLF_ERR_CUDA;
            }
            count_launch();
            return RLF_OK;
        }
    }
    const int grid = (int)(p.T < 148 * 8 ? p.T : 148 * 8);
    if (dt == RLF_BF16) ce_row_general_kernel<__nv_bfloat16><<<grid, kGenThreads, 0, s>>>(p);
    else ce_row_general_kernel<float><<<grid, kGenThreads, 0, s>>>(p);
    count_launch();
    return cuda_ok(cudaGetLastError());
}

}  // namespace ce

rlf_status ce_launch_count(const uint8_t* mask, int64_t T, long long* count, cudaStream_t s) {
    ce::ce_count_kernel<<<1, 1024, 0, s>>>(mask, T, count);
    count_launch();
    return cuda_ok(cudaGetLastError());
}
rlf_status ce_launch_loss(const void* terms, int64_t T, const long long* denom, float eps, float zeta, double* loss_out,
                          cudaStream_t s) {
    ce::ce_loss_kernel<<<1, ce::kLossThreads, 0, s>>>(static_cast<const float4*>(terms), T, denom, eps, zeta, loss_out);
    count_launch();
    return cuda_ok(cudaGetLastError());
}
rlf_status ce_check_objective(float label_smoothing, float z_coef) {
    if (!(label_smoothing >= 0.0f && label_smoothing <= 1.0f)) return RLF_ERR_UNSUPPORTED;
    if (!(z_coef >= 0.0f && z_coef < INFINITY)) return RLF_ERR_UNSUPPORTED;
    return RLF_OK;
}
size_t cross_entropy_workspace_bytes(int64_t T) { return ce::kWsTermsOff + 16 * (size_t)(T > 0 ? T : 0); }

}  // namespace rlf

extern "C" rlf_status rlf_cross_entropy_fwd_bwd(const void* logits, rlf_dtype dt, int64_t T, int32_t V, int64_t row_stride,
                                                const int32_t* ids, const uint8_t* mask, float label_smoothing, float z_coef,
                                                const int64_t* denom, float* logp_out, float* lse_out, double* loss_out,
                                                void* grad_logits, void* workspace, size_t workspace_bytes,
                                                int32_t* dev_status, rlf_stream_t stream) {
    using namespace rlf;
    using namespace rlf::ce;
    if (dt != RLF_BF16 && dt != RLF_F32) return RLF_ERR_DTYPE;
    if (T < 0 || V < 1 || row_stride < V) return RLF_ERR_SHAPE;
    rlf_status st = ce_check_objective(label_smoothing, z_coef);
    if (st != RLF_OK) return st;
    if (T >= (1ll << 31)) return RLF_ERR_UNSUPPORTED;
    if (!loss_out) return RLF_ERR_NULL;
    if (T > 0 && (!logits || !ids || !logp_out)) return RLF_ERR_NULL;
    const size_t esz = dt == RLF_BF16 ? 2 : 4;
    if (!aligned(logits, esz) || !aligned(grad_logits, esz) || !aligned(ids, 4) || !aligned(logp_out, 4) ||
        !aligned(lse_out, 4) || !aligned(loss_out, 8) || !aligned(denom, 8))
        return RLF_ERR_ALIGN;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < cross_entropy_workspace_bytes(T)) return RLF_ERR_WORKSPACE;
    st = check_arch();
    if (st != RLF_OK) return st;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    const long long* dn = reinterpret_cast<const long long*>(denom);
    if (!dn) {
        st = ce_launch_count(mask, T, reinterpret_cast<long long*>(ws), s);
        if (st != RLF_OK) return st;
        dn = reinterpret_cast<const long long*>(ws);
    }
    RowParams p;
    p.logits = logits; p.grad = grad_logits; p.stride = row_stride; p.T = T; p.V = V; p.ids = ids; p.mask = mask;
    p.denom = dn; p.logp_out = logp_out; p.lse_out = lse_out; p.terms = reinterpret_cast<float4*>(ws + kWsTermsOff);
    p.dev_status = dev_status; p.eps = label_smoothing; p.zeta = z_coef;
    if (T > 0) {
        st = launch_rows(p, dt, s);
        if (st != RLF_OK) return st;
    }
    return ce_launch_loss(p.terms, T, dn, label_smoothing, z_coef, loss_out, s);
}
