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
        const int grid = (int)(T < 148 * 8 ? T : 148 * 8);
        if (dt == RLF_BF16) ce_row_general_kernel<__nv_bfloat16><<<grid, kGenThreads, 0, s>>>(p);
        else ce_row_general_kernel<float><<<grid, kGenThreads, 0, s>>>(p);
        count_launch();
        if (cudaGetLastError() != cudaSuccess) return RLF_ERR_CUDA;
    }
    return ce_launch_loss(p.terms, T, dn, label_smoothing, z_coef, loss_out, s);
}
