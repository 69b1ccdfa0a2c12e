// The norm in front of the LM head, forward and backward: layer norm and its RMS form, with the
// residual addition and the gradient of the residual stream folded in.
//
//   h = x (+ residual);   layer: mu = mean(h), r = 1 / sqrt(mean((h - mu)^2) + eps);   RMS: mu = 0, r = 1 / sqrt(mean(h^2) + eps)
//   y = (h - mu) r w (+ b)
// and, with xh = (h - mu) r and g = dy w,
//   dx = r (g - [layer] mean(g) - xh mean(g xh)) (+ grad_skip);   dw = sum_t dy xh;   db = sum_t dy
//
// Both directions are bound by HBM: a row is read once and written once (about 10 arithmetic
// instructions per element).  All sums and statistics are fp32; the sum h is rounded to the
// activations' type only where it is stored, and y is formed from the unrounded h.
#include "common.cuh"

namespace rlf {
namespace nm {

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// element i of a weight vector of either type
__device__ __forceinline__ float ld_w(const void* w, int w_bf16, int i) {
    return w_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(w)[i]) : static_cast<const float*>(w)[i];
}

struct FwdParams {
    const void* x;
    const void* res;            // nullable
    long long x_stride;         // elements; x and res
    const void* w;
    const void* b;              // nullable
    int w_bf16;
    int layer;
    void* sum;                  // [T, D], nullable
    void* y;                    // [T, D]
    float* mean;                // nullable
    float* rstd;                // nullable
    long long T;
    int D;
    float eps;
};

struct BwdParams {
    const void* dy;
    long long dy_stride;
    const void* x;
    long long x_stride;
    const void* w;
    int w_bf16;
    int layer;
    const float* mean;          // layer only
    const float* rstd;
    const void* skip;           // [T, D], nullable
    void* dx;                   // [T, D], nullable
    float* part;                // partial sums of dw, then of db: [parts][D] each; NULL: neither is wanted
    float* part_b;
    long long T;
    int D;
};

constexpr int kGenThreads = 256;

// sum over the CTA, the same value in every thread; `red` holds one float per warp
__device__ __forceinline__ float cta_sum(float v, float* red) {
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.0f;
    for (int w = 0; w < (int)(blockDim.x >> 5); ++w) s += red[w];
    return s;
}

// Any width and alignment: one CTA per row, the row read once per pass (later passes are served by L2).
// A thread handles the same elements in every pass and reads each before it writes it.
template <typename T>
__global__ void __launch_bounds__(kGenThreads)
norm_fwd_general_kernel(const FwdParams p) {
    __shared__ float red[kGenThreads / 32];
    const float inv_d = 1.0f / (float)p.D;
    for (long long t = blockIdx.x; t < p.T; t += gridDim.x) {
        const T* x = static_cast<const T*>(p.x) + t * p.x_stride;
        const T* res = p.res ? static_cast<const T*>(p.res) + t * p.x_stride : nullptr;
        auto h = [&](int i) { return to_f<T>(x[i]) + (res ? to_f<T>(res[i]) : 0.0f); };
        float mu = 0.0f;
        if (p.layer) {
            float s = 0.0f;
            for (int i = threadIdx.x; i < p.D; i += kGenThreads) s += h(i);
            mu = cta_sum(s, red) * inv_d;
        }
        float q = 0.0f;
        for (int i = threadIdx.x; i < p.D; i += kGenThreads) {
            const float c = h(i) - mu;
            q = fmaf(c, c, q);
        }
        const float r = rsqrtf(cta_sum(q, red) * inv_d + p.eps);
        for (int i = threadIdx.x; i < p.D; i += kGenThreads) {
            const float v = h(i);
            float o = (v - mu) * r * ld_w(p.w, p.w_bf16, i);
            if (p.b) o += ld_w(p.b, p.w_bf16, i);
            if (p.sum) static_cast<T*>(p.sum)[t * p.D + i] = from_f<T>(v);
            static_cast<T*>(p.y)[t * p.D + i] = from_f<T>(o);
        }
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[t] = mu;
            if (p.rstd) p.rstd[t] = r;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kGenThreads)
norm_bwd_general_kernel(const BwdParams p) {
    __shared__ float red[kGenThreads / 32];
    const float inv_d = 1.0f / (float)p.D;
    for (long long t = blockIdx.x; t < p.T; t += gridDim.x) {
        const T* x = static_cast<const T*>(p.x) + t * p.x_stride;
        const T* dy = static_cast<const T*>(p.dy) + t * p.dy_stride;
        const float mu = p.layer ? p.mean[t] : 0.0f, r = p.rstd[t];
        float a = 0.0f, b = 0.0f;
        for (int i = threadIdx.x; i < p.D; i += kGenThreads) {
            const float g = to_f<T>(dy[i]) * ld_w(p.w, p.w_bf16, i);
            a = fmaf(g, (to_f<T>(x[i]) - mu) * r, a);
            b += g;
        }
        a = cta_sum(a, red) * inv_d;
        b = p.layer ? cta_sum(b, red) * inv_d : 0.0f;
        for (int i = threadIdx.x; i < p.D; i += kGenThreads) {
            const float g = to_f<T>(dy[i]) * ld_w(p.w, p.w_bf16, i);
            float o = r * (g - b - (to_f<T>(x[i]) - mu) * r * a);
            if (p.skip) o += to_f<T>(static_cast<const T*>(p.skip)[t * p.D + i]);
            static_cast<T*>(p.dx)[t * p.D + i] = from_f<T>(o);
        }
    }
}

// Weight gradients for any width: a CTA covers 32 columns of one slice of rows, 8 rows at a time
// (warp w takes rows w, w + 8, ...), and leaves one partial row for its slice.
template <typename T>
__global__ void __launch_bounds__(256)
norm_dw_general_kernel(const BwdParams p, long long rows_per_slice) {
    __shared__ float acc_w[8][32], acc_b[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + lane;
    const long long t0 = (long long)blockIdx.y * rows_per_slice;
    const long long t1 = min(p.T, t0 + rows_per_slice);
    float sw = 0.0f, sb = 0.0f;
    if (col < p.D)
        for (long long t = t0 + warp; t < t1; t += 8) {
            const float mu = p.layer ? p.mean[t] : 0.0f;
            const float dy = to_f<T>(static_cast<const T*>(p.dy)[t * p.dy_stride + col]);
            sw = fmaf(dy, (to_f<T>(static_cast<const T*>(p.x)[t * p.x_stride + col]) - mu) * p.rstd[t], sw);
            sb += dy;
        }
    acc_w[warp][lane] = sw;
    acc_b[warp][lane] = sb;
    __syncthreads();
    if (warp == 0 && col < p.D) {
        for (int w = 1; w < 8; ++w) {
            sw += acc_w[w][lane];
            sb += acc_b[w][lane];
        }
        if (p.part) p.part[(long long)blockIdx.y * p.D + col] = sw;
        if (p.part_b) p.part_b[(long long)blockIdx.y * p.D + col] = sb;
    }
}

// partial rows -> gradient, added in a fixed order (results are run-to-run identical).  A CTA covers 32
// columns; warp w adds the partials w, w + 8, ... and the eight sums are added in order.
__global__ void __launch_bounds__(256)
norm_dw_reduce_kernel(const float* __restrict__ part, const float* __restrict__ part_b, int parts, int D, int accumulate,
                      float* __restrict__ dw, float* __restrict__ db) {
    __shared__ float acc[8][32];
    const float* src = blockIdx.y == 0 ? part : part_b;
    float* dst = blockIdx.y == 0 ? dw : db;
    if (dst == nullptr) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (col < D)
        for (int k = warp; k < parts; k += 8) s += src[(long long)k * D + col];
    acc[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && col < D) {
        for (int w = 1; w < 8; ++w) s += acc[w][lane];
        dst[col] = accumulate ? dst[col] + s : s;
    }
}

// Most partial rows of a weight gradient; sizes the workspace.
constexpr int kMaxParts = 1024;

static int row_grid(long long T) { return (int)(T < 148 * 8 ? T : 148 * 8); }

static rlf_status check_norm(int64_t T, int32_t D, rlf_dtype dt, rlf_dtype w_dt, int kind) {
    if ((dt != RLF_BF16 && dt != RLF_F32) || (w_dt != RLF_BF16 && w_dt != RLF_F32)) return RLF_ERR_DTYPE;
    if (T < 0 || D < 1) return RLF_ERR_SHAPE;
    if (kind != RLF_NORM_LAYER && kind != RLF_NORM_RMS) return RLF_ERR_UNSUPPORTED;
    return RLF_OK;
}

}  // namespace nm

size_t norm_bwd_workspace_bytes(int64_t T, int32_t D) {
    if (D < 1) return 0;
    const size_t parts = (size_t)(T < 1 ? 1 : T < nm::kMaxParts ? T : nm::kMaxParts);
    return 2 * parts * (size_t)D * sizeof(float) + 256;
}

}  // namespace rlf

extern "C" rlf_status rlf_norm_fwd(const void* x, const void* residual, rlf_dtype dt, int64_t T, int32_t D,
                                   int64_t x_stride, const void* weight, const void* bias, rlf_dtype w_dt, int kind,
                                   float eps, void* sum_out, void* y_out, float* mean_out, float* rstd_out,
                                   rlf_stream_t stream) {
    using namespace rlf;
    using namespace rlf::nm;
    rlf_status st = check_norm(T, D, dt, w_dt, kind);
    if (st != RLF_OK) return st;
    if (x_stride < D) return RLF_ERR_SHAPE;
    if (!(eps > 0.0f) || !(eps < INFINITY)) return RLF_ERR_UNSUPPORTED;
    if (T == 0) return RLF_OK;
    if (!x || !weight || !y_out) return RLF_ERR_NULL;
    const size_t esz = dt == RLF_BF16 ? 2 : 4, wsz = w_dt == RLF_BF16 ? 2 : 4;
    if (!aligned(x, esz) || !aligned(residual, esz) || !aligned(sum_out, esz) || !aligned(y_out, esz) ||
        !aligned(weight, wsz) || !aligned(bias, wsz) || !aligned(mean_out, 4) || !aligned(rstd_out, 4))
        return RLF_ERR_ALIGN;
    st = check_arch();
    if (st != RLF_OK) return st;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    FwdParams p;
    p.x = x; p.res = residual; p.x_stride = x_stride; p.w = weight; p.b = bias; p.w_bf16 = w_dt == RLF_BF16;
    p.layer = kind == RLF_NORM_LAYER; p.sum = sum_out; p.y = y_out; p.mean = mean_out; p.rstd = rstd_out;
    p.T = T; p.D = D; p.eps = eps;
    if (dt == RLF_BF16) norm_fwd_general_kernel<__nv_bfloat16><<<row_grid(T), kGenThreads, 0, s>>>(p);
    else norm_fwd_general_kernel<float><<<row_grid(T), kGenThreads, 0, s>>>(p);
    count_launch();
    return cuda_ok(cudaGetLastError());
}

extern "C" rlf_status rlf_norm_bwd(const void* grad_y, int64_t grad_y_stride, const void* x, int64_t x_stride, rlf_dtype dt,
                                   int64_t T, int32_t D, const void* weight, rlf_dtype w_dt, int kind, const float* mean,
                                   const float* rstd, const void* grad_skip, void* grad_x, float* grad_weight,
                                   float* grad_bias, int accumulate, void* workspace, size_t workspace_bytes,
                                   rlf_stream_t stream) {
    using namespace rlf;
    using namespace rlf::nm;
    rlf_status st = check_norm(T, D, dt, w_dt, kind);
    if (st != RLF_OK) return st;
    if (x_stride < D || grad_y_stride < D) return RLF_ERR_SHAPE;
    const bool layer = kind == RLF_NORM_LAYER, want_w = grad_weight || grad_bias;
    if (T > 0 && (!grad_y || !x || !weight || !rstd || (layer && !mean))) return RLF_ERR_NULL;
    const size_t esz = dt == RLF_BF16 ? 2 : 4, wsz = w_dt == RLF_BF16 ? 2 : 4;
    if (!aligned(grad_y, esz) || !aligned(x, esz) || !aligned(grad_skip, esz) || !aligned(grad_x, esz) ||
        !aligned(weight, wsz) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(grad_weight, 4) || !aligned(grad_bias, 4))
        return RLF_ERR_ALIGN;
    if (want_w && (!workspace || !aligned(workspace, 256) || workspace_bytes < norm_bwd_workspace_bytes(T, D)))
        return RLF_ERR_WORKSPACE;
    st = check_arch();
    if (st != RLF_OK) return st;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    BwdParams p;
    p.dy = grad_y; p.dy_stride = grad_y_stride; p.x = x; p.x_stride = x_stride; p.w = weight; p.w_bf16 = w_dt == RLF_BF16;
    p.layer = layer; p.mean = mean; p.rstd = rstd; p.skip = grad_skip; p.dx = grad_x; p.T = T; p.D = D;
    p.part = p.part_b = nullptr;
    int parts = 0;
    if (T > 0) {
        if (want_w) {
            const long long rows = T < kMaxParts ? 1 : (T + 127) / 128;      // per slice: at most 128 slices of a long batch
            parts = (int)((T + rows - 1) / rows);
            p.part = grad_weight ? static_cast<float*>(workspace) : nullptr;
            p.part_b = grad_bias ? static_cast<float*>(workspace) + (size_t)parts * D : nullptr;
            const dim3 grid((unsigned)((D + 31) / 32), (unsigned)parts);
            if (dt == RLF_BF16) norm_dw_general_kernel<__nv_bfloat16><<<grid, 256, 0, s>>>(p, rows);
            else norm_dw_general_kernel<float><<<grid, 256, 0, s>>>(p, rows);
            count_launch();
            if (cudaGetLastError() != cudaSuccess) return RLF_ERR_CUDA;
        }
        // last: grad_x may be the buffer of x or grad_y
        if (grad_x) {
            if (dt == RLF_BF16) norm_bwd_general_kernel<__nv_bfloat16><<<row_grid(T), kGenThreads, 0, s>>>(p);
            else norm_bwd_general_kernel<float><<<row_grid(T), kGenThreads, 0, s>>>(p);
            count_launch();
            if (cudaGetLastError() != cudaSuccess) return RLF_ERR_CUDA;
        }
    }
    if (!want_w) return RLF_OK;
    // with no rows the gradient is zero (or what was accumulated before)
    const float* part = static_cast<const float*>(workspace);
    norm_dw_reduce_kernel<<<dim3((unsigned)((D + 31) / 32), 2), 256, 0, s>>>(
        part, part + (size_t)parts * D, parts, D, accumulate, grad_weight, grad_bias);
    count_launch();
    return cuda_ok(cudaGetLastError());
}
