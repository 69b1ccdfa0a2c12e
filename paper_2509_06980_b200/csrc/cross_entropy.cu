// Softmax cross entropy over materialised logits, forward and backward, with label smoothing and a
// z-loss: the supervised counterpart of the log-prob + loss kernels.  Per row with loss weight,
// y = ids[t], N the number of such rows (or the caller's count), eps the smoothing, zeta the z-loss:
//   lse = log sum_v exp z_v
//   l   = (1 - eps) (lse - z_y) + eps (lse - mean_v z_v) + zeta lse^2
//   dL/dz_v = (1/N) [ (1 + 2 zeta lse) p_v - eps/V - (1 - eps) [v = y] ],   p = softmax(z)
// The target column is formed as (1/N) [ 2 zeta lse p_y - S'/S + eps - eps/V ], S' the sum over the
// other columns, so that it keeps its digits when p_y rounds to one.
//
// Kernels, in launch order: ce_plan_kernel (work list: the rows that carry loss, then the others; their
// count), the row kernel (writes logp, lse, the row's loss terms and grad_logits), ce_loss_kernel (fp64 sums in
// a fixed order).  Rows without loss weight are not read at all; their gradient is written as zeros.
// Without a gradient many long rows take ce_stream_kernel and ce_stream_join_kernel in place of the row kernel.
#include <type_traits>

#include "common.cuh"
#include "row.cuh"

namespace rlf {
namespace ce {

// workspace: [0] int64 number of rows with mask != 0; [64] int number of live rows; [256 ..) one float4 of loss terms
// per token, {lse - z_y, lse - mean z (0 without smoothing), lse, 1 if the row counts}; then the work list, one
// int2 per token: {row, target id} of the live rows in order, then {row, -1} of the others; then the streaming form's parts
constexpr size_t kWsTermsOff = 256;
constexpr size_t ws_list_off(int64_t T) { return kWsTermsOff + 16 * (size_t)(T > 0 ? T : 0); }

struct RowParams {
    const void* logits;
    void* grad;                 // nullable
    long long stride;           // elements
    long long T;
    int V;
    const int2* list;           // {row, target id} of the live rows, then {row, -1} of the others
    const int* n_live;
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
    for (long long k = blockIdx.x; k < p.T; k += gridDim.x) {
        const int2 job = p.list[k];
        const long long t = job.x;
        const int y = job.y;
        const T* z = static_cast<const T*>(p.logits) + t * p.stride;
        T* g = p.grad ? static_cast<T*>(p.grad) + t * p.stride : nullptr;
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
            if (y >= 0 && !r.ok) status |= RLF_DEV_NONFINITE;
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
// is copied up to the row's end, and a first vector that starts before the logits do element by element (row 0's,
// and those of the few rows after it that lie in the same vector when rows are shorter than one); any other row's
// first vector starts in a row before it.
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
// (the rounding is the same for every exponent of a warp and known: sums and gradients are put right by offset_error; without it
// a log-prob is off by up to 8e-5 at |max| = 2000)

struct ClusterParams {
    RowParams r;
    int per_cta_vec;            // vectors of a row per CTA of the cluster
    float inv_v;                // 1 / V
    // launch constants, kept out of the registers
    int csize, num_clusters;
    uint32_t row_bytes;         // bytes that every CTA receives per exchanged row
    // rows whose first vector starts before the logits do (none where the base is aligned).  A launch constant, and row 0 named
    // beside it: compared with row * stride in the loop it cost spills (4096 x 151937 bf16 368 -> 393 us; 373 without row 0)
    int first_rows;
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
// elements [from, to) of a 16-byte vector in shared memory stay, the others become -inf
template <typename T>
__device__ __forceinline__ void keep_elements(uint4* at, int from, int to) {
    uint4 v = *at;
    uint32_t* w = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (sizeof(T) == 2) {
            const uint32_t lo = (2 * j >= from && 2 * j < to) ? w[j] & 0xffffu : 0xFF80u;
            const uint32_t hi = (2 * j + 1 >= from && 2 * j + 1 < to) ? w[j] & 0xffff0000u : 0xFF800000u;
            w[j] = lo | hi;
        } else if (j < from || j >= to) {
            w[j] = 0xFF800000u;
        }
    }
    *at = v;
}
__device__ __forceinline__ void cp_async16_part(void* smem_dst, const void* gmem_src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(smem_u32(smem_dst)), "l"(gmem_src), "r"(bytes) : "memory");
}

// Programmatic dependent launch: the next kernel of a call may be set up while this one runs; it waits here before it
// reads anything that an earlier kernel wrote.
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_trigger() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
// Bounded wait for a row's exchange (about a second).  What it remembers of a wait that ran out sits in shared
// memory: a register carried through the row loop costs spills.
__device__ __forceinline__ void wait_row(uint32_t bar, uint32_t parity, int* timed_out) {
    for (int i = 0; i < kWaitPolls; ++i) {
        if (mbar_try_wait(bar, parity)) return;
        if ((i & 1023) == 1023 && *reinterpret_cast<volatile int*>(timed_out)) return;
    }
    *reinterpret_cast<volatile int*>(timed_out) = 1;
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

    __shared__ float inv_n_s;
    __shared__ int timed_out;                                 // a wait ran out: no wait is taken again, the loops end, reported
    __shared__ __align__(8) int2 job_slot[8];                 // ring of work-list entries, fetched three rows ahead

    const int crank = (int)cluster_ctarank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
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
    const int nvalid_all = EDGE ? 0 : count_valid(p.V / VE);

    auto prefetch = [&](int row) {
        const int head = row_head(row);
        const T* row0 = static_cast<const T*>(p.logits) + (long long)row * p.stride - head;
        const uint4* src = reinterpret_cast<const uint4*>(row0) + vbeg;
        uint4* dst = stage + tid;
        const int nvec = row_vecs(head), nvalid = EDGE ? count_valid(nvec) : nvalid_all;
        const int last_bytes = EDGE ? (head + p.V - (nvec - 1) * VE) * (int)sizeof(T) : 16;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (i < nvalid) {
                const int v = vbeg + i * THREADS;
                if (EDGE && v == 0 && (row == 0 || row < cp.first_rows) && head != 0) {
                    T* d = reinterpret_cast<T*>(dst + i * THREADS);
                    for (int e = head; e < VE && e < head + p.V; ++e) d[e] = row0[e];
                } else if (EDGE && v == nvec - 1) {
                    cp_async16_part(dst + i * THREADS, src + i * THREADS, last_bytes);
                } else {
                    cp_async16_cg(dst + i * THREADS, src + i * THREADS);
                }
            }
        }
    };

    if (tid == 0) {
        mbar_init(smem_u32(&row_bar[0]), 1);
        mbar_init(smem_u32(&row_bar[1]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        timed_out = 0;
    }
    pdl_wait();
    pdl_trigger();
    if (tid == 0) {
        const long long N = *p.denom;
        inv_n_s = 1.0f / (float)(N > 1 ? N : 1);
    }
    const int cluster_id = blockIdx.x / cp.csize;
    const int n_live = *p.n_live;
    // thread 0 fetches the entry of this cluster's j-th row, in the cp.async group of an earlier row's data
    auto fetch_job = [&](int j) {
        const long long at = (long long)cluster_id + (long long)j * cp.num_clusters;
        if (tid == 0 && at < n_live)
            asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" :: "r"(smem_u32(&job_slot[j & 7])), "l"(p.list + at) : "memory");
    };
    auto job_row = [&](int j) -> int { return reinterpret_cast<const volatile int*>(job_slot)[2 * (j & 7)]; };
    auto job_target = [&](int j) -> int { return reinterpret_cast<const volatile int*>(job_slot)[2 * (j & 7) + 1]; };
    for (int j = 0; j < 3; ++j) fetch_job(j);
    cp_async_wait_all();
    __syncthreads();
    if (cluster_id < n_live) prefetch(job_row(0));
    cp_async_commit();
    // every CTA of the cluster is running before any peer may address its shared memory
    cluster_sync_all();

    // a row's own elements of its first and last vector, by the thread that has put them into edge_slot
    auto store_edges = [&](T* g_row, int head, int nvec, int nvalid) {
        const int lrel = nvec - 1 - vbeg;
        const bool first = vbeg == 0 && nvalid > 0;
        const bool last = nvec > 1 && lrel >= 0 && (lrel & (THREADS - 1)) == 0 && lrel / THREADS < nvalid;
        if (first || last) {
#pragma unroll 1
            for (int side = first ? 0 : 1; side <= (last ? 1 : 0); ++side) {
                const uint4 o = edge_slot[side];
                const T* oe = reinterpret_cast<const T*>(&o);
                const int base = (side == 0 ? 0 : nvec - 1) * VE - head;    // column of the vector's element 0
#pragma unroll
                for (int e = 0; e < VE; ++e)
                    if (base + e >= 0 && base + e < p.V) g_row[base + e] = oe[e];
            }
        }
    };
    auto zero_row = [&](int row, int head, int nvec, int nvalid) {
        T* g_row = static_cast<T*>(p.grad) + (long long)row * p.stride;
        uint4* dst = reinterpret_cast<uint4*>(g_row - head) + vbeg;
        const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
        for (int i = 0; i < nvalid; ++i) {
            const int v = vbeg + i * THREADS;
            if (EDGE && v == 0) edge_slot[0] = zero;
            else if (EDGE && v == nvec - 1) edge_slot[1] = zero;
            else st_stream(dst + i * THREADS, zero);
        }
        if (EDGE) store_edges(g_row, head, nvec, nvalid);
    };
    int it = 0;
    int k = cluster_id;
    for (; k < n_live; k += cp.num_clusters, ++it) {
        const int head = row_head(job_row(it));
        const int nvec = row_vecs(head), nvalid = EDGE ? count_valid(nvec) : nvalid_all;
        float m_ws;
        uint4 d[NV];
        {
            const int parity = it & 1;
            const uint32_t bar = smem_u32(&row_bar[parity]);
            cp_async_wait_all();
            if (tid == 0) mbar_arrive_expect_tx(bar, cp.row_bytes);
            if (EDGE) {
                // what lies in the first and the last vector beside the row is not part of it
                const int tail = head + p.V - (nvec - 1) * VE;          // elements of the last vector up to the row's end
                if (vbeg == 0 && nvalid > 0) keep_elements<T>(&stage[tid], head, VE);
                const int lrel = nvec - 1 - vbeg;
                if (lrel >= 0 && (lrel & (THREADS - 1)) == 0 && lrel / THREADS < nvalid) keep_elements<T>(&stage[lrel + tid], 0, tail);
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
                if (lane < cp.csize)
                    st_async_f1(smem_u32(&mean_slot[parity][crank * NWARPS + warp]), bar, (uint32_t)lane, q);
            }
            // the owner of the target column sends its logit to every CTA and takes it out of the sums: the
            // target's gradient needs the sum over the OTHER columns
            const int ye = job_target(it) + head, yrel = ye / VE - vbeg;
            const bool own_y = yrel >= 0 && (yrel & (THREADS - 1)) == 0 && yrel / THREADS < nvalid;
            if (own_y) {
                T* sv = reinterpret_cast<T*>(&stage[yrel + tid]) + ye % VE;
                const float zt = to_f<T>(*sv);
                for (int r = 0; r < cp.csize; ++r) st_async_f1(smem_u32(&zy_slot[parity]), bar, (uint32_t)r, zt);
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
            // the slots are in registers: queue the next row
            if ((long long)k + cp.num_clusters < n_live) prefetch(job_row(it + 1));
            fetch_job(it + 3);
            cp_async_commit();
            m_w = ord2f(__reduce_max_sync(0xffffffffu, f2ord(m_w)));
            m_ws = (m_w == -INFINITY) ? 0.0f : m_w;
            float s0 = 0.0f, s1 = 0.0f;
            if (BF && fabsf(m_ws) <= kRobustAbove) {
                const float off = -__fmul_rn(m_ws, kLog2e);
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
                s0 = fmaf(s0, offset_error(m_ws), s0);
                s1 = fmaf(s1, offset_error(m_ws), s1);
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
            if (lane < cp.csize) st_async_f2(smem_u32(&pair_slot[parity][crank * NWARPS + warp]), bar, (uint32_t)lane, m_w, s_w);
            wait_row(bar, (uint32_t)(it >> 1) & 1u, &timed_out);
            // merge all warps' pairs of the row, lanes in parallel, identically in every warp
            const int npairs = cp.csize * NWARPS;
            float M = -INFINITY;
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
            float others = 0.0f;
#pragma unroll
            for (int j = 0; j < (MAXE + 31) / 32; ++j)
                // (a warp whose logits are all -inf has the sum 0; one whose logits are -inf and NaN has the same maximum and the
                // sum NaN, which takes the row out)
                others += e[j].x == -INFINITY ? e[j].y : e[j].y * ex2_approx((e[j].x - M) * kLog2e);
            others = warp_sum(others);
            if (smooth) Q = warp_sum(Q);
            const float S = others + ex2_approx((zy - M) * kLog2e);
            const RowStats st = row_stats(M, S, zy, Q, p.eps);
            if (crank == 0 && tid == 0) {
                write_row(p, job_row(it), st);
                if (!st.ok && p.dev_status) atomicOr(p.dev_status, RLF_DEV_NONFINITE);
            }
            if (p.grad != nullptr) {
                if (!st.ok) {
                    zero_row(job_row(it), head, nvec, nvalid);
                } else {
                    // entries are a e - u: the registers hold 2^((z - m_w) log2e)
                    // (fast divisions, two ulp: an exact one holds a slow path that the row in the registers is spilled for)
                    float a = __fdividef(inv_n_s * (1.0f + 2.0f * p.zeta * st.lse), S) * ex2_approx((m_ws - M) * kLog2e);
                    if (BF && fabsf(m_ws) <= kRobustAbove) a = fmaf(a, offset_error(m_ws), a);
                    const float u = inv_n_s * p.eps * cp.inv_v;
                    T* g_row = static_cast<T*>(p.grad) + (long long)job_row(it) * p.stride;
                    uint4* dst = reinterpret_cast<uint4*>(g_row - head) + vbeg;
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        if (i >= nvalid) continue;
                        uint4 o;
                        uint32_t* w = reinterpret_cast<uint32_t*>(&o);
                        const uint32_t* x = reinterpret_cast<const uint32_t*>(&d[i]);
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            w[j] = BF ? pack_bf16x2(fmaf(bf_lo(x[j]), a, -u), fmaf(bf_hi(x[j]), a, -u))
                                      : __float_as_uint(fmaf(__uint_as_float(x[j]), a, -u));
                        const int v = vbeg + i * THREADS;
                        if (EDGE && v == 0) edge_slot[0] = o;
                        else if (EDGE && v == nvec - 1) edge_slot[1] = o;
                        else st_stream(dst + i * THREADS, o);
                    }
                    if (EDGE) store_edges(g_row, head, nvec, nvalid);
                    // (the target id is re-read from its slot, not held in a register across the passes)
                    const int yt = job_target(it), yr = (yt + head) / VE - vbeg;
                    if (yr >= 0 && (yr & (THREADS - 1)) == 0 && yr / THREADS < nvalid) {
                        const float rest = __fdividef(others, S);                       // 1 - p_y
                        g_row[yt] = from_f<T>(inv_n_s * (2.0f * p.zeta * st.lse * (1.0f - rest) - rest + p.eps) - u);
                    }
                }
            }
        }
    }
    // rows without loss weight (or without such a target) are not read, their gradient is zeros.  Among live rows the exchange
    // keeps a row's edge_slot apart from the next row's; here, where the last vector may be another thread's, the barrier does:
    // every thread has stored its edges of the last live row before a slot becomes zero.
    if (EDGE) __syncthreads();
    for (; k < nrows; k += cp.num_clusters) {
        const int row = p.list[k].x;
        if (crank == 0 && tid == 0) write_row(p, row, RowStats{});
        if (p.grad == nullptr) continue;
        const int head = row_head(row), nvec = row_vecs(head);
        zero_row(row, head, nvec, EDGE ? count_valid(nvec) : nvalid_all);
    }
    // a warp that gave up: peers' stores of the last rows may still be on their way into this CTA
    if (*reinterpret_cast<volatile int*>(&timed_out)) {
        if (lane == 0 && p.dev_status) atomicOr(p.dev_status, RLF_DEV_TIMEOUT);
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    }
    cluster_sync_all();                  // no CTA leaves while a peer could still address its shared memory
}

// ---------------------------------------------------------------------------------------------
// Forward only, long rows: without a gradient nobody has to hold a row.  A work unit is one chunk of a live row (up to
// 256 x NV vectors); every warp leaves its (max, sum, share of the mean) of a unit and a second kernel joins a row's.  No
// exchange and no barrier: a thread reads only the staging slots that it filled itself, so that the warps of a CTA drift
// and loads and exponentials overlap.  Bound by HBM.  EDGE as in the cluster kernel.
constexpr int kStreamThreads = 256, kStreamWarps = kStreamThreads / 32, kStreamNV = 8, kStreamCtasPerSm = 4;
constexpr int kStreamUnits = 8;              // units per CTA: it then retires, as the cluster kernel's CTAs do

struct StreamParams {
    RowParams r;
    int chunks, per_chunk_vec;               // of a row; vectors of a chunk (the last may hold fewer)
    float inv_v;
    float4* part;                            // [live row][chunks][kStreamWarps]: max, sum 2^((z - max) log2 e), sum z / V, -
};
// chunks of a row that covers nvec vectors
static int stream_chunks(int64_t nvec) { return (int)((nvec + kStreamThreads * kStreamNV - 1) / (kStreamThreads * kStreamNV)); }

template <typename T, bool EDGE>
__global__ void __launch_bounds__(kStreamThreads, kStreamCtasPerSm)
ce_stream_kernel(const StreamParams sp) {
    const RowParams& p = sp.r;
    constexpr bool BF = sizeof(T) == 2;
    constexpr int VE = Elem<T>::kPer, THREADS = kStreamThreads, NV = kStreamNV;
    extern __shared__ __align__(16) uint4 stage[];            // [NV][THREADS], slot (i, tid) private to thread tid
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const bool smooth = p.eps > 0.0f;
    // the elements of a vector, two at a time
    auto for_pairs = [](const uint4& v, auto f) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        if constexpr (BF) {
#pragma unroll
            for (int j = 0; j < 4; ++j) f(f2_make(bf_lo(w[j]), bf_hi(w[j])));
        } else {
            f(f2_make(__uint_as_float(w[0]), __uint_as_float(w[1])));
            f(f2_make(__uint_as_float(w[2]), __uint_as_float(w[3])));
        }
    };
    struct Unit { int head, nvec, vbeg, nvalid; };
    auto unit = [&](long long u, int row) -> Unit {
        Unit q;
        q.head = EDGE ? (int)((reinterpret_cast<uintptr_t>(p.logits) / sizeof(T) + (unsigned long long)((long long)row * p.stride)) % VE) : 0;
        q.nvec = EDGE ? (q.head + p.V + VE - 1) / VE : p.V / VE;
        const int chunk = (int)(u % sp.chunks);
        q.vbeg = chunk * sp.per_chunk_vec + tid;
        const int vend = min(q.nvec, (chunk + 1) * sp.per_chunk_vec);
        q.nvalid = vend > q.vbeg ? (vend - q.vbeg + THREADS - 1) / THREADS : 0;
        return q;
    };
    pdl_wait();
    pdl_trigger();
    const long long units = (long long)*p.n_live * sp.chunks, step = gridDim.x;
    auto row_of = [&](long long u) -> int { return u < units ? p.list[u / sp.chunks].x : 0; };
    auto prefetch = [&](long long u, int row) {
        if (u < units) {
            const Unit q = unit(u, row);
            const T* row0 = static_cast<const T*>(p.logits) + (long long)row * p.stride - q.head;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i < q.nvalid) {
                    const int v = q.vbeg + i * THREADS;
                    const uint4* src = reinterpret_cast<const uint4*>(row0) + v;
                    uint4* dst = stage + i * THREADS + tid;
                    if (EDGE && v == 0 && q.head != 0 && row == 0) {        // (rows are longer than a vector here)
                        T* e = reinterpret_cast<T*>(dst);
                        for (int j = q.head; j < VE && j < q.head + p.V; ++j) e[j] = row0[j];
                    } else if (EDGE && v == q.nvec - 1) {
                        cp_async16_part(dst, src, (q.head + p.V - v * VE) * (int)sizeof(T));
                    } else {
                        cp_async16_cg(dst, src);
                    }
                }
        }
        cp_async_commit();
    };
    long long u = blockIdx.x;
    int row = row_of(u), row_next = row_of(u + step);          // (entries of the list are fetched a unit ahead of their data)
    prefetch(u, row);
    for (; u < units; u += step) {
        const Unit q = unit(u, row);
        cp_async_wait_all();
        float mean = 0.0f;
        if (EDGE) {
            // what lies in the first and the last vector beside the row is not part of it
            if (q.vbeg == 0 && q.nvalid > 0) keep_elements<T>(&stage[tid], q.head, VE);
            const int lrel = q.nvec - 1 - q.vbeg;
            if (lrel >= 0 && lrel % THREADS == 0 && lrel / THREADS < q.nvalid)
                keep_elements<T>(&stage[lrel + tid], 0, q.head + p.V - (q.nvec - 1) * VE);
        }
        const uint32_t ninf = Elem<T>::neg_inf();
        uint4 d[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (i < q.nvalid) d[i] = stage[i * THREADS + tid];
            else d[i] = make_uint4(ninf, ninf, ninf, ninf);
        }
        if (smooth) {
            const f2 inv2 = f2_make(sp.inv_v, sp.inv_v);
            f2 mean2 = 0ull;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int v = q.vbeg + i * THREADS;
                if (i >= q.nvalid) continue;
                if (EDGE && (v == 0 || v == q.nvec - 1)) {
                    const T* e = reinterpret_cast<const T*>(&stage[i * THREADS + tid]);
                    for (int j = 0; j < VE; ++j)
                        if (v * VE + j >= q.head && v * VE + j < q.head + p.V) mean = fmaf(to_f<T>(e[j]), sp.inv_v, mean);
                    continue;
                }
                for_pairs(d[i], [&](f2 z) { mean2 = f2_fma(z, inv2, mean2); });
            }
            mean = warp_sum(mean + f2_sum(mean2));
        }
        prefetch(u + step, row_next);                          // the slots are in registers
        row = row_next;
        row_next = row_of(u + 2 * step);
        float m;
        if (BF) {
            uint32_t mx = ninf;
#pragma unroll
            for (int i = 0; i < NV; ++i) mx = max_bf16x2(mx, max_bf16x2(max_bf16x2(d[i].x, d[i].y), max_bf16x2(d[i].z, d[i].w)));
            m = fmaxf(bf_lo(mx), bf_hi(mx));
        } else {
            m = -INFINITY;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(d[i].x), __uint_as_float(d[i].y)),
                                   fmaxf(__uint_as_float(d[i].z), __uint_as_float(d[i].w))));
        }
        m = ord2f(__reduce_max_sync(0xffffffffu, f2ord(m)));
        const float ms = (m == -INFINITY) ? 0.0f : m;
        const bool fold = BF && fabsf(ms) <= kRobustAbove;     // as in the cluster kernel
        const float off = -__fmul_rn(ms, kLog2e);
        const f2 off2 = f2_make(off, off), ms2 = f2_make(-ms, -ms), c2 = f2_make(kLog2e, kLog2e);
        f2 sum2 = 0ull;
        auto add = [&](auto folded) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                for_pairs(d[i], [&](f2 z) {
                    float a, b;
                    f2_split(decltype(folded)::value ? f2_fma(z, c2, off2) : f2_mul(f2_add(z, ms2), c2), a, b);
                    sum2 = f2_add(sum2, f2_make(ex2_approx(a), ex2_approx(b)));
                });
        };
        if (fold) add(std::true_type{});
        else add(std::false_type{});
        float s = warp_sum(f2_sum(sum2));
        if (fold) s = fmaf(s, offset_error(ms), s);
        if (lane == 0) sp.part[u * kStreamWarps + warp] = make_float4(m, s, mean, 0.0f);
    }
    cp_async_wait_all();
}

// one warp per entry of the work list: a live row's parts are joined, any other row gets its NaNs
template <typename T>
__global__ void __launch_bounds__(256)
ce_stream_join_kernel(const StreamParams sp) {
    const RowParams& p = sp.r;
    const int lane = threadIdx.x & 31, per_row = sp.chunks * kStreamWarps;
    const long long k = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    pdl_wait();
    pdl_trigger();
    if (k >= p.T) return;
    const int2 job = p.list[k];
    RowStats r = {};
    if (k < *p.n_live) {
        const float4* part = sp.part + k * per_row;
        const float zy = to_f<T>(static_cast<const T*>(p.logits)[(long long)job.x * p.stride + job.y]);
        float M = -INFINITY, S = 0.0f, Q = 0.0f;
        for (int c = lane; c < per_row; c += 32) M = fmaxf(M, part[c].x);
        M = ord2f(__reduce_max_sync(0xffffffffu, f2ord(M)));
        for (int c = lane; c < per_row; c += 32) {
            const float4 e = part[c];
            // (a part of -inf logits has the sum 0, or NaN where it held a NaN)
            S += e.x == -INFINITY ? e.y : e.y * ex2_approx((e.x - M) * kLog2e);
            Q += e.z;
        }
        r = row_stats(M, warp_sum(S), zy, warp_sum(Q), p.eps);
        if (lane == 0 && !r.ok && p.dev_status) atomicOr(p.dev_status, RLF_DEV_NONFINITE);
    }
    if (lane == 0) write_row(p, job.x, r);
}

// ---- launch shape ---------------------------------------------------------------------------
typedef void (*RowKernel)(const ClusterParams);
struct RowShape { int cluster, threads, nv; };

// one CTA per row for rows of up to 1024 vectors: 64 or 128 threads, an even number of vectors each
template <typename T, int THREADS, bool EDGE>
static RowKernel narrow_kernel(int nv) {
    switch (nv) {
        case 2: return ce_row_cluster_kernel<T, THREADS, 2, EDGE, 1>;
        case 4: return ce_row_cluster_kernel<T, THREADS, 4, EDGE, 1>;
        case 6: return ce_row_cluster_kernel<T, THREADS, 6, EDGE, 1>;
        case 8: return ce_row_cluster_kernel<T, THREADS, 8, EDGE, 1>;
    }
    return nullptr;
}
// clusters of 1 to 8 CTAs, or (CMAX = 16) of 10 and 16: 6 to 10 vectors per thread
template <typename T, int THREADS, bool EDGE, int CMAX>
static RowKernel wide_kernel(int nv) {
    switch (nv) {
        case 6: return ce_row_cluster_kernel<T, THREADS, 6, EDGE, CMAX>;
        case 7: return ce_row_cluster_kernel<T, THREADS, 7, EDGE, CMAX>;
        case 8: return ce_row_cluster_kernel<T, THREADS, 8, EDGE, CMAX>;
        case 9: return ce_row_cluster_kernel<T, THREADS, 9, EDGE, CMAX>;
        case 10: return EDGE ? nullptr : ce_row_cluster_kernel<T, THREADS, 10, false, CMAX>;
    }
    return nullptr;
}
template <typename T, bool EDGE>
static RowKernel row_kernel(const RowShape& sh) {
    if (sh.threads == 64) return narrow_kernel<T, 64, EDGE>(sh.nv);
    if (sh.threads == 128) return narrow_kernel<T, 128, EDGE>(sh.nv);
    if (sh.threads == 512) return wide_kernel<T, 512, EDGE, 16>(sh.nv);
    return sh.cluster <= 8 ? wide_kernel<T, 256, EDGE, 8>(sh.nv) : wide_kernel<T, 256, EDGE, 16>(sh.nv);
}

// 16-byte vectors of a row per CTA: an even split rounded up to whole 128-byte lines
static int per_cta_vectors(int nvec, int cluster) { return (((nvec + cluster - 1) / cluster) + 7) & ~7; }

// Rows of up to 512 vectors go to one CTA of 64 threads, up to 1024 to one of 128 (what a short row costs is its chain of
// latencies, so as many rows as possible are under way: 65536 x 2048 bf16 took 229 us as 256 threads a row, 139 as 64);
// longer ones to the smallest cluster of 256-thread CTAs that holds them (1, 2, 4 or 8 CTAs; then 10 and 16, beyond
// the portable size), the longest to 16 CTAs of 512 threads.  At most 10 vectors per thread (9 with EDGE, 8 in the
// small CTAs): the most that the registers hold without spilling more than a few words.  false: no shape holds it.
static bool pick_shape(int nvec, bool edge, RowShape* out) {
    static const RowShape shapes[] = {{1, 64, 8}, {1, 128, 8}, {1, 256, 10}, {2, 256, 10}, {4, 256, 10},
                                      {8, 256, 10}, {10, 256, 10}, {16, 256, 10}, {16, 512, 10}};
    for (const RowShape& sh : shapes) {
        int nv = (per_cta_vectors(nvec, sh.cluster) + sh.threads - 1) / sh.threads;
        if (nv > (edge && sh.nv > 9 ? 9 : sh.nv)) continue;
        if (sh.threads < 256) nv = (nv + 1) & ~1;
        else if (nv < 6) nv = 6;
        *out = {sh.cluster, sh.threads, nv};
        return true;
    }
    return false;
}

// at: two attributes, the second (programmatic dependent launch) added by the launch itself
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
    static ResidentTable table;
    return table.get((const void*)k, sh.cluster, sh.threads, [&](int) {
        int n = 0;
        cudaLaunchConfig_t cfg;
        cudaLaunchAttribute at[2];
        cluster_config(&cfg, at, sh.cluster * 148 * 8, sh, nullptr);
        if (cudaFuncSetAttribute((const void*)k, cudaFuncAttributeMaxDynamicSharedMemorySize, stage_bytes(sh.threads, sh.nv)) != cudaSuccess ||
            (sh.cluster > 8 && cudaFuncSetAttribute((const void*)k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) ||
            cudaOccupancyMaxActiveClusters(&n, (void*)k, &cfg) != cudaSuccess) {
            cudaGetLastError();
            n = 0;
        }
        return n;
    });
}

// A cluster handles about ten rows before it retires (whole generations of what is resident at once): with one
// generation of persistent clusters all of them load, then all of them store, in step for the whole launch
// (8192 x 151936 bf16, rows per cluster 8 / 10 / 14 / 20 / 32 / 100: 784 / 785 / 790 / 799 / 817 / 1082 us).
constexpr int kRowsPerCluster = 10;
static int clusters_for(int resident, long long rows) {
    const long long per_generation = (long long)resident * kRowsPerCluster;
    long long nc = (rows + per_generation - 1) / per_generation * resident;
    if (nc > rows) nc = rows;
    return (int)(nc < (1 << 26) ? nc : (1 << 26));
}

// ---- the small kernels around the row kernel ---------------------------------------------------
// Both run as one cluster of up to 8 CTAs (one SM each): a single CTA needs 30 us for 65536 tokens, a grid would need a
// second launch to join its parts.
constexpr int kPlanThreads = 1024, kPlanPer = 8, kMaxPlanCtas = 8;
constexpr int kPlanTokens = kPlanThreads * kPlanPer;         // tokens per CTA and step

// the 32-bit word at the same shared-memory place in CTA `rank` of the cluster
__device__ __forceinline__ int ld_cluster_int(const int* local, int rank) {
    uint32_t remote;
    int v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(smem_u32(local)), "r"(rank));
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(remote) : "memory");
    return v;
}
__device__ __forceinline__ double ld_cluster_double(const double* local, int rank) {
    uint32_t remote;
    double v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(smem_u32(local)), "r"(rank));
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(remote) : "memory");
    return v;
}

// mask and ids -> the work list: {row, target id} of the rows with loss weight and a target inside the vocabulary, in
// order, then {row, -1} of the others (from the end backwards); *n_live of the first kind, and the number of rows with
// mask != 0.  CTA r takes the r-th stretch of kPlanTokens tokens of every step, a thread every 1024th token of it.
__global__ void __launch_bounds__(kPlanThreads)
ce_plan_kernel(const int32_t* __restrict__ ids, const uint8_t* __restrict__ mask, int T, int V, int2* __restrict__ list,
               int* __restrict__ n_live, long long* __restrict__ n_mask, int* __restrict__ zero, int zero_words,
               int32_t* __restrict__ dev_status) {
    __shared__ int piece[kPlanPer * 32];     // live rows of each (k, warp) of this CTA, then their exclusive sums
    __shared__ int cta_live[2];              // live rows of this CTA in a step, two steps in turn
    __shared__ int cta_masked;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int csize = (int)cluster_nctarank(), crank = (int)cluster_ctarank();
    pdl_trigger();
    if (crank == 0 && tid < zero_words) zero[tid] = 0;       // flags and counters of the caller's later launches
    int base = 0, masked_in = 0, step = 0;
    bool bad = false;
    for (long long s0 = 0; s0 < T; s0 += (long long)csize * kPlanTokens, step ^= 1) {
        const long long t0 = s0 + (long long)crank * kPlanTokens;
        int y[kPlanPer];
        unsigned b[kPlanPer];
        int in[kPlanPer];
#pragma unroll
        for (int k = 0; k < kPlanPer; ++k) {
            const long long t = t0 + 1024 * k + tid;
            in[k] = t < T ? (mask ? mask[t] : 1) : 0;
            y[k] = t < T ? ids[t] : 0;
        }
#pragma unroll
        for (int k = 0; k < kPlanPer; ++k) {
            const bool live = in[k] && y[k] >= 0 && y[k] < V;
            masked_in += in[k] != 0;
            bad |= in[k] && !live;
            b[k] = __ballot_sync(0xffffffffu, live);
            if (lane == 0) piece[k * 32 + warp] = __popc(b[k]);
        }
        __syncthreads();
        if (warp == 0) {
            // exclusive sums of the 256 pieces in row order, eight per lane
            int c[kPlanPer], mine = 0;
#pragma unroll
            for (int k = 0; k < kPlanPer; ++k) {
                c[k] = piece[lane * kPlanPer + k];
                mine += c[k];
            }
            int incl = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int up = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += up;
            }
            int at = incl - mine;
#pragma unroll
            for (int k = 0; k < kPlanPer; ++k) {
                piece[lane * kPlanPer + k] = at;
                at += c[k];
            }
            if (lane == 31) cta_live[step] = incl;
        }
        if (csize > 1) cluster_sync_all();
        else __syncthreads();
        int before = base, total = 0;
        for (int r = 0; r < csize; ++r) {
            const int n = csize > 1 ? ld_cluster_int(&cta_live[step], r) : cta_live[step];
            if (r < crank) before += n;
            total += n;
        }
#pragma unroll
        for (int k = 0; k < kPlanPer; ++k) {
            const long long t = t0 + 1024 * k + tid;
            const int at = before + piece[k * 32 + warp] + __popc(b[k] & ((1u << lane) - 1u));
            if ((b[k] >> lane) & 1u) list[at] = make_int2((int)t, y[k]);
            else if (t < T) list[T - 1 - ((int)t - at)] = make_int2((int)t, -1);
        }
        base += total;
        __syncthreads();                     // the pieces are free for the next step
    }
    if (bad && dev_status) atomicOr(dev_status, RLF_DEV_BAD_TARGET);
    masked_in = __reduce_add_sync(0xffffffffu, masked_in);
    if (lane == 0) piece[warp] = masked_in;
    __syncthreads();
    if (tid == 0) {
        int n = 0;
        for (int w = 0; w < 32; ++w) n += piece[w];
        cta_masked = n;
    }
    if (csize > 1) cluster_sync_all();
    if (crank == 0 && tid == 0) {
        long long n = 0;
        for (int r = 0; r < csize; ++r) n += csize > 1 ? ld_cluster_int(&cta_masked, r) : cta_masked;
        *n_mask = n;
        *n_live = base;
    }
    if (csize > 1) cluster_sync_all();       // no CTA leaves while another may read its shared memory
}

// loss terms -> loss_out[4] in fp64.  Every thread adds its tokens in index order, then a fixed tree over the CTA and the
// CTAs in order: the same order on every launch.
constexpr int kLossThreads = 1024;
__global__ void __launch_bounds__(kLossThreads)
ce_loss_kernel(const float4* __restrict__ terms, long long T, const long long* __restrict__ denom, float eps, float zeta,
               double* __restrict__ loss_out) {
    __shared__ double red[3][kLossThreads / 32];
    __shared__ double cta_sum[3];
    const int csize = (int)cluster_nctarank(), crank = (int)cluster_ctarank();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    pdl_wait();
    double a = 0.0, b = 0.0, c = 0.0;
#pragma unroll 4
    for (long long t = (long long)crank * kLossThreads + threadIdx.x; t < T; t += (long long)csize * kLossThreads) {
        const float4 r = terms[t];
        if (r.w != 0.0f) {
            a += (double)r.x;
            b += (double)r.y;
            c += (double)r.z * (double)r.z;
        }
    }
    auto tree = [](double v) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    };
    a = tree(a);
    b = tree(b);
    c = tree(c);
    if (lane == 0) {
        red[0][warp] = a;
        red[1][warp] = b;
        red[2][warp] = c;
    }
    __syncthreads();
    if (warp < 3) {
        const double v = tree(red[warp][lane]);
        if (lane == 0) cta_sum[warp] = v;
    }
    if (csize > 1) cluster_sync_all();
    else __syncthreads();
    if (crank == 0 && threadIdx.x == 0) {
        double q[3] = {0.0, 0.0, 0.0};
        for (int k = 0; k < 3; ++k)
            for (int r = 0; r < csize; ++r) q[k] += csize > 1 ? ld_cluster_double(&cta_sum[k], r) : cta_sum[k];
        const long long N = *denom;
        const double nd = (double)(N > 1 ? N : 1);
        loss_out[0] = ((1.0 - (double)eps) * q[0] + (double)eps * q[1] + (double)zeta * q[2]) / nd;
        loss_out[1] = q[0] / nd;
        loss_out[2] = q[1] / nd;
        loss_out[3] = q[2] / nd;
    }
    if (csize > 1) cluster_sync_all();
}

// one cluster of `ctas` CTAs; pdl: the launch may overlap the end of the kernel before it (the kernel waits by itself)
template <typename... Args>
static rlf_status launch_cluster(void (*k)(Args...), int ctas, int threads, bool pdl, cudaStream_t s, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[2];
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(threads);
    cfg.stream = s;
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = ctas;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = pdl ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, k, args...) != cudaSuccess) {
        cudaGetLastError();
        return RLF_ERR_CUDA;
    }
    count_launch();
    return RLF_OK;
}
// a launch whose kernel waits by itself for the kernel before it
template <typename P>
static rlf_status launch_after(void (*k)(const P), long long grid, int threads, int smem, cudaStream_t s, const P& p) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, k, p) != cudaSuccess) {
        cudaGetLastError();
        return RLF_ERR_CUDA;
    }
    count_launch();
    return RLF_OK;
}
static int small_ctas(int64_t T, int64_t per_cta) {
    const int64_t n = (T + per_cta - 1) / per_cta;
    return (int)(n < 1 ? 1 : n < kMaxPlanCtas ? n : kMaxPlanCtas);
}

// vectors of 16 bytes that a row may take: one more than its length fills when it lies on no boundary
static int64_t row_vectors(int32_t V, int ve, bool edge) { return edge ? ((int64_t)V + 2 * ve - 2) / ve : V / ve; }
// Forward only, the streaming form against the cluster kernel (which a row of up to 2560 vectors needs one CTA of): 8192 rows
// of 151936 bf16 426 us (5.8 TB/s) against 527, 4096 of fp32 365 (6.8 TB/s) against 495, 8192 of 24000 bf16 104 either way;
// 512 rows of 151936 bf16 48 us against 50, 8 rows 28 against 26 (one launch more).
static bool streams(int64_t T, int64_t nvec) { return nvec > 2560 && T >= 512; }
static size_t ws_part_off(int64_t T) { return (ws_list_off(T) + 8 * (size_t)(T > 0 ? T : 0) + 15) & ~(size_t)15; }
static size_t part_bytes(int64_t T, int32_t V, rlf_dtype dt) {
    const int64_t nvec = row_vectors(V, dt == RLF_BF16 ? 8 : 4, true);
    return streams(T, nvec) ? 16 * (size_t)T * stream_chunks(nvec) * kStreamWarps : 0;
}

// The cluster kernel wherever a shape holds the row and the gradient rows sit like the logits rows within their
// 16-byte vectors; otherwise (rows beyond 81,920 vectors, a gradient buffer of another alignment) the general one,
// which reads a row three times (V = 151936 bf16, 8192 rows: 3.69 ms against 0.79).
// Forward only, rows beyond one CTA: the streaming form (parts: the workspace's room for its partials).
static rlf_status launch_rows(const RowParams& p, rlf_dtype dt, float4* parts, cudaStream_t s) {
    const size_t esz = dt == RLF_BF16 ? 2 : 4;
    const int ve = (int)(16 / esz);
    const bool edge = p.V % ve != 0 || p.stride % ve != 0 || !aligned(p.logits, 16);
    const bool same = !p.grad || (reinterpret_cast<uintptr_t>(p.grad) - reinterpret_cast<uintptr_t>(p.logits)) % 16 == 0;
    const int64_t nvec = row_vectors(p.V, ve, edge);
    RowShape sh;
    if (!p.grad && streams(p.T, nvec)) {
        StreamParams sp;
        sp.r = p;
        sp.chunks = stream_chunks(nvec);
        sp.per_chunk_vec = (int)((nvec + sp.chunks - 1) / sp.chunks);
        sp.inv_v = 1.0f / (float)p.V;
        sp.part = parts;
        const long long units = (long long)p.T * sp.chunks, resident = 148ll * kStreamCtasPerSm;
        long long grid = (units + kStreamUnits - 1) / kStreamUnits;
        if (grid < resident) grid = resident < units ? resident : units;
        if (grid > (1 << 30)) grid = 1 << 30;
        void (*k)(const StreamParams) = dt == RLF_BF16 ? (edge ? ce_stream_kernel<__nv_bfloat16, true> : ce_stream_kernel<__nv_bfloat16, false>)
                                                       : (edge ? ce_stream_kernel<float, true> : ce_stream_kernel<float, false>);
        const rlf_status st = launch_after(k, grid, kStreamThreads, kStreamNV * kStreamThreads * 16, s, sp);
        if (st != RLF_OK) return st;
        return launch_after(dt == RLF_BF16 ? ce_stream_join_kernel<__nv_bfloat16> : ce_stream_join_kernel<float>, (p.T + 7) / 8, 256, 0, s, sp);
    }
    if (same && nvec < (1 << 24) && pick_shape((int)nvec, edge, &sh)) {
        const RowKernel k = dt == RLF_BF16 ? (edge ? row_kernel<__nv_bfloat16, true>(sh) : row_kernel<__nv_bfloat16, false>(sh))
                                           : (edge ? row_kernel<float, true>(sh) : row_kernel<float, false>(sh));
        const int resident = k ? resident_clusters(k, sh) : 0;
        if (resident > 0) {
            ClusterParams cp;
            cp.r = p;
            cp.per_cta_vec = per_cta_vectors((int)nvec, sh.cluster);
            cp.inv_v = 1.0f / (float)p.V;
            cudaLaunchConfig_t cfg;
            cudaLaunchAttribute at[2];
            cp.csize = sh.cluster;
            const long long lead = (long long)(reinterpret_cast<uintptr_t>(p.logits) % 16 / esz);
            cp.first_rows = lead > 0 ? (int)((ve - lead + p.stride - 1) / p.stride) : 0;
            cp.num_clusters = clusters_for(resident, p.T);
            cp.row_bytes = (uint32_t)(sh.cluster * (sh.threads / 32)) * (p.eps > 0.0f ? 12u : 8u) + 4u;
            cluster_config(&cfg, at, cp.num_clusters * sh.cluster, sh, s);
            at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
            at[1].val.programmaticStreamSerializationAllowed = 1;
            cfg.numAttrs = 2;
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

rlf_status ce_launch_plan(const int32_t* ids, const uint8_t* mask, int64_t T, int32_t V, void* list, int* n_live,
                          long long* n_mask, int* zero, int zero_words, int32_t* dev_status, cudaStream_t s) {
    return ce::launch_cluster(ce::ce_plan_kernel, ce::small_ctas(T, ce::kPlanTokens), ce::kPlanThreads, false, s, ids, mask,
                              (int)T, (int)V, static_cast<int2*>(list), n_live, n_mask, zero, zero_words, dev_status);
}
rlf_status ce_launch_loss(const void* terms, int64_t T, const long long* denom, float eps, float zeta, double* loss_out,
                          cudaStream_t s) {
    return ce::launch_cluster(ce::ce_loss_kernel, ce::small_ctas(T, 4 * ce::kLossThreads), ce::kLossThreads, true, s,
                              static_cast<const float4*>(terms), (long long)T, denom, eps, zeta, loss_out);
}
rlf_status ce_check_objective(float label_smoothing, float z_coef) {
    if (!(label_smoothing >= 0.0f && label_smoothing <= 1.0f)) return RLF_ERR_UNSUPPORTED;
    if (!(z_coef >= 0.0f && z_coef < INFINITY)) return RLF_ERR_UNSUPPORTED;
    return RLF_OK;
}
size_t cross_entropy_workspace_bytes(int64_t T, int32_t V, rlf_dtype dt) {
    return V < 1 ? 0 : ce::ws_part_off(T) + ce::part_bytes(T, V, dt);
}

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
    if (T >= (1ll << 30) || V >= (1 << 30)) return RLF_ERR_UNSUPPORTED;      // the kernels count both in 32 bits
    if (!loss_out) return RLF_ERR_NULL;
    if (T > 0 && (!logits || !ids || !logp_out)) return RLF_ERR_NULL;
    const size_t esz = dt == RLF_BF16 ? 2 : 4;
    if (!aligned(logits, esz) || !aligned(grad_logits, esz) || !aligned(ids, 4) || !aligned(logp_out, 4) ||
        !aligned(lse_out, 4) || !aligned(loss_out, 8) || !aligned(denom, 8))
        return RLF_ERR_ALIGN;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < cross_entropy_workspace_bytes(T, V, dt)) return RLF_ERR_WORKSPACE;
    st = check_arch();
    if (st != RLF_OK) return st;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    int2* list = reinterpret_cast<int2*>(ws + ws_list_off(T));
    long long* n_mask = reinterpret_cast<long long*>(ws);
    int* n_live = reinterpret_cast<int*>(ws + 64);
    st = ce_launch_plan(ids, mask, T, V, list, n_live, n_mask, nullptr, 0, dev_status, s);
    if (st != RLF_OK) return st;
    const long long* dn = denom ? reinterpret_cast<const long long*>(denom) : n_mask;
    RowParams p;
    p.logits = logits; p.grad = grad_logits; p.stride = row_stride; p.T = T; p.V = V; p.list = list; p.n_live = n_live;
    p.denom = dn; p.logp_out = logp_out; p.lse_out = lse_out; p.terms = reinterpret_cast<float4*>(ws + kWsTermsOff);
    p.dev_status = dev_status; p.eps = label_smoothing; p.zeta = z_coef;
    if (T > 0) {
        st = launch_rows(p, dt, reinterpret_cast<float4*>(ws + ws_part_off(T)), s);
        if (st != RLF_OK) return st;
    }
    return ce_launch_loss(p.terms, T, dn, label_smoothing, z_coef, loss_out, s);
}
