// The norms after a block and before the next, with the block's gate and the residual's scale, in one pass over the rows:
//
//   n = norm_post(x);   h = alpha residual + beta gate n;   y = norm_pre(h)            (either norm may be absent)
// norms as in norm.cu (RMS, or layer with mean and bias); the gate is a vector over the columns, one number per row, or absent.
// Backward, from dy (gradient of y) and dh (gradient that reaches h along the residual stream), with u = (h - m2) r2, v = (x - m1) r1:
//   gh = dh + r2 (q - [layer] mean(q) - u mean(q u)),  q = dy w_pre;                     d residual = alpha gh
//   with s = beta gate:   dx = r1 (g - [layer] mean(g) - v mean(g v)),  g = s gh w_post   (no norm: dx = s gh)
//   dw_pre = sum_t dy u,  db_pre = sum_t dy,  dw_post = sum_t s gh v,  db_post = sum_t s gh,  dgate = beta sum gh n  (over t, or the row)
//
// Bound by HBM: forward reads two rows and writes two, backward reads four and writes two.  Statistics and sums are fp32 and no
// intermediate is rounded: y comes from the unrounded h, dx from the unrounded gh.
// A column gate is a factor of the post norm's sums over tokens, S1 = sum_t [row gate] gh v and S2 = sum_t [row gate] gh, so that
// the gradients of gate, weight and bias all come from these two (finish kernel).
#include "norm_rows.cuh"

namespace rlf {
namespace bn {

using namespace nm;

struct BlockParams {
    const void* x;
    long long x_stride;
    const void* res;                // forward
    const void* w1;                 // post norm's weight and bias, pre norm's weight and bias, [D] each
    const void* b1;
    const void* w2;
    const void* b2;
    const void* gate;
    int w_bf16;
    int post, pre;                  // RLF_NORM_*
    int gate_form;                  // RLF_GATE_*
    float alpha, beta, eps;
    void* h;                        // forward: output; backward: input
    void* y;
    float* stats;                   // [4][T]: post mean, post rstd, pre mean, pre rstd
    const void* dy;                 // backward
    const void* dh;                 // nullable
    void* dx;                       // nullable
    void* dres;                     // nullable
    float* dgate_row;               // [T], nullable
    float* part;                    // partial sums [4][parts][D] (dw_pre, db_pre, S1, S2); NULL: none wanted
    int want;                       // bit i: sum i is wanted
    long long part_stride;          // floats from one sum's partial rows to the next's
    float2* row_sums;               // general form: mean(q u), mean(q) of each row
    long long T;
    int D;
    int period, x_shift;            // fast forms: see below
};

__device__ __forceinline__ bool has_norm(int kind) { return kind != RLF_NORM_NONE; }
// factor of column c (weight, column gate and branch scale) and the same of the bias
__device__ __forceinline__ float col_scale(const BlockParams& p, int c) {
    return p.beta * (p.gate_form == RLF_GATE_COLUMN ? ld_w(p.gate, p.w_bf16, c) : 1.0f);
}
__device__ __forceinline__ float post_w(const BlockParams& p, int c) { return p.w1 ? ld_w(p.w1, p.w_bf16, c) : 1.0f; }
__device__ __forceinline__ float row_gate(const BlockParams& p, long long t) {
    return p.gate_form == RLF_GATE_ROW ? static_cast<const float*>(p.gate)[t] : 1.0f;
}

constexpr int kGenThreads = 256;

// ---- any width, stride and alignment: one CTA per row, the row read once per pass (later passes are served by L2) ----------
template <typename T>
__global__ void __launch_bounds__(kGenThreads)
block_fwd_general_kernel(const BlockParams p) {
    __shared__ float red[kGenThreads / 32];
    const float inv_d = 1.0f / (float)p.D;
    for (long long t = blockIdx.x; t < p.T; t += gridDim.x) {
        const T* x = static_cast<const T*>(p.x) + t * p.x_stride;
        const T* res = static_cast<const T*>(p.res) + t * p.D;
        float m1 = 0.0f, r1 = 1.0f, m2 = 0.0f, r2 = 1.0f;
        const float g = row_gate(p, t);
        auto stats = [&](auto value, int kind, float& m, float& r) {
            if (kind == RLF_NORM_LAYER) {
                float s = 0.0f;
                for (int i = threadIdx.x; i < p.D; i += kGenThreads) s += value(i);
                m = cta_sum(s, red) * inv_d;
            }
            float q = 0.0f;
            for (int i = threadIdx.x; i < p.D; i += kGenThreads) {
                const float c = value(i) - m;
                q = fmaf(c, c, q);
            }
            r = rsqrtf(cta_sum(q, red) * inv_d + p.eps);
        };
        if (has_norm(p.post)) stats([&](int i) { return to_f<T>(x[i]); }, p.post, m1, r1);
        auto h = [&](int i) {
            float n = (to_f<T>(x[i]) - m1) * r1 * post_w(p, i);
            if (p.b1) n += ld_w(p.b1, p.w_bf16, i);
            return fmaf(p.alpha, to_f<T>(res[i]), g * col_scale(p, i) * n);
        };
        if (has_norm(p.pre)) stats(h, p.pre, m2, r2);
        for (int i = threadIdx.x; i < p.D; i += kGenThreads) {
            const float v = h(i);                        // (reads residual before h, which may be the same buffer, is written)
            static_cast<T*>(p.h)[t * p.D + i] = from_f<T>(v);
            if (has_norm(p.pre)) {
                float o = (v - m2) * r2 * ld_w(p.w2, p.w_bf16, i);
                if (p.b2) o += ld_w(p.b2, p.w_bf16, i);
                static_cast<T*>(p.y)[t * p.D + i] = from_f<T>(o);
            }
        }
        if (threadIdx.x == 0 && p.stats) {
            p.stats[t] = m1;
            p.stats[p.T + t] = r1;
            p.stats[2 * p.T + t] = m2;
            p.stats[3 * p.T + t] = r2;
        }
    }
}

// gradient of h in one element, from the row's means over q u and q
template <typename T>
__device__ __forceinline__ float grad_h_at(const BlockParams& p, long long t, int i, float m2, float r2, float a, float b) {
    const long long at = t * p.D + i;
    float g = p.dh ? to_f<T>(static_cast<const T*>(p.dh)[at]) : 0.0f;
    if (has_norm(p.pre)) {
        const float q = to_f<T>(static_cast<const T*>(p.dy)[at]) * ld_w(p.w2, p.w_bf16, i);
        g += r2 * (q - b - (to_f<T>(static_cast<const T*>(p.h)[at]) - m2) * r2 * a);
    }
    return g;
}

template <typename T>
__global__ void __launch_bounds__(kGenThreads)
block_bwd_general_kernel(const BlockParams p) {
    __shared__ float red[kGenThreads / 32];
    const float inv_d = 1.0f / (float)p.D;
    for (long long t = blockIdx.x; t < p.T; t += gridDim.x) {
        const T* x = static_cast<const T*>(p.x) + t * p.x_stride;
        const float m1 = p.stats[t], r1 = p.stats[p.T + t], m2 = p.stats[2 * p.T + t], r2 = p.stats[3 * p.T + t];
        float a1 = 0.0f, b1 = 0.0f;
        if (has_norm(p.pre)) {
            for (int i = threadIdx.x; i < p.D; i += kGenThreads) {
                const long long at = t * p.D + i;
                const float q = to_f<T>(static_cast<const T*>(p.dy)[at]) * ld_w(p.w2, p.w_bf16, i);
                a1 = fmaf(q, (to_f<T>(static_cast<const T*>(p.h)[at]) - m2) * r2, a1);
                b1 += q;
            }
            a1 = cta_sum(a1, red) * inv_d;
            b1 = p.pre == RLF_NORM_LAYER ? cta_sum(b1, red) * inv_d : 0.0f;
        }
        if (threadIdx.x == 0 && p.row_sums) p.row_sums[t] = make_float2(a1, b1);
        const float g = row_gate(p, t);
        float a2 = 0.0f, b2 = 0.0f, c2 = 0.0f;               // over gh w v, gh w, gh b (w and b with the column gate and beta)
        if (has_norm(p.post) || p.dgate_row) {
            for (int i = threadIdx.x; i < p.D; i += kGenThreads) {
                const float gh = grad_h_at<T>(p, t, i, m2, r2, a1, b1) * col_scale(p, i), w = gh * post_w(p, i);
                a2 = fmaf(w, (to_f<T>(x[i]) - m1) * r1, a2);
                b2 += w;
                if (p.b1) c2 = fmaf(gh, ld_w(p.b1, p.w_bf16, i), c2);
            }
            a2 = cta_sum(a2, red);
            b2 = p.post == RLF_NORM_LAYER ? cta_sum(b2, red) * inv_d : 0.0f;
            c2 = p.b1 ? cta_sum(c2, red) : 0.0f;
        }
        if (threadIdx.x == 0 && p.dgate_row) p.dgate_row[t] = a2 + c2;
        a2 = has_norm(p.post) ? a2 * inv_d : 0.0f;
        for (int i = threadIdx.x; i < p.D; i += kGenThreads) {
            const float gh = grad_h_at<T>(p, t, i, m2, r2, a1, b1);
            if (p.dres) static_cast<T*>(p.dres)[t * p.D + i] = from_f<T>(p.alpha * gh);
            if (p.dx) {
                const float w = gh * col_scale(p, i) * post_w(p, i);
                static_cast<T*>(p.dx)[t * p.D + i] = from_f<T>(g * r1 * (w - b2 - (to_f<T>(x[i]) - m1) * r1 * a2));
            }
        }
    }
}

// Sums over tokens for any width: a CTA covers 32 columns of one slice of rows, 8 rows at a time.
template <typename T>
__global__ void __launch_bounds__(256)
block_sums_general_kernel(const BlockParams p, long long rows_per_slice) {
    __shared__ float acc[4][8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + lane;
    const long long t0 = (long long)blockIdx.y * rows_per_slice, t1 = min(p.T, t0 + rows_per_slice);
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (col < p.D)
        for (long long t = t0 + warp; t < t1; t += 8) {
            const float m1 = p.stats[t], r1 = p.stats[p.T + t], m2 = p.stats[2 * p.T + t], r2 = p.stats[3 * p.T + t];
            float2 q = make_float2(0.0f, 0.0f);
            if (has_norm(p.pre)) {
                q = p.row_sums[t];
                const float dy = to_f<T>(static_cast<const T*>(p.dy)[t * p.D + col]);
                s[0] = fmaf(dy, (to_f<T>(static_cast<const T*>(p.h)[t * p.D + col]) - m2) * r2, s[0]);
                s[1] += dy;
            }
            const float gh = row_gate(p, t) * grad_h_at<T>(p, t, col, m2, r2, q.x, q.y);
            s[2] = fmaf(gh, (to_f<T>(static_cast<const T*>(p.x)[t * p.x_stride + col]) - m1) * r1, s[2]);
            s[3] += gh;
        }
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[k][warp][lane] = s[k];
    __syncthreads();
    if (warp < 4 && col < p.D && ((p.want >> warp) & 1)) {
        float v = 0.0f;
        for (int w = 0; w < 8; ++w) v += acc[warp][w][lane];
        p.part[warp * p.part_stride + (long long)blockIdx.y * p.D + col] = v;
    }
}

struct Finish {
    const float* part;
    long long part_stride;
    int parts, D, want, accumulate;
    const void* w1;
    const void* b1;
    const void* gate;
    int w_bf16, gate_form;
    float beta;
    float* dw2;
    float* db2;
    float* dw1;
    float* db1;
    float* dgate;                   // [D], nullable
};
// partial rows -> gradients, added in a fixed order: a CTA covers 32 columns of the pre (blockIdx.y = 0) or post norm's two
// sums; warp w adds the partial rows w, w + 32, ... and the 32 sums are added in order.
__global__ void __launch_bounds__(1024)
block_finish_kernel(const Finish f) {
    __shared__ float acc[2][32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + lane, first = 2 * blockIdx.y;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if (col < f.D && ((f.want >> (first + k)) & 1)) {
            const float* src = f.part + (first + k) * f.part_stride + col;
#pragma unroll 4
            for (int r = warp; r < f.parts; r += 32) s[k] += src[(long long)r * f.D];
        }
        acc[k][warp][lane] = s[k];
    }
    __syncthreads();
    if (warp != 0 || col >= f.D) return;
    for (int w = 1; w < 32; ++w) {
        s[0] += acc[0][w][lane];
        s[1] += acc[1][w][lane];
    }
    auto leave = [&](float* d, float v) {
        if (d) d[col] = f.accumulate ? d[col] + v : v;
    };
    if (blockIdx.y == 0) {
        leave(f.dw2, s[0]);
        leave(f.db2, s[1]);
    } else {
        const float scale = f.beta * (f.gate_form == RLF_GATE_COLUMN ? ld_w(f.gate, f.w_bf16, col) : 1.0f);
        leave(f.dw1, scale * s[0]);
        leave(f.db1, scale * s[1]);
        float v = s[0] * (f.w1 ? ld_w(f.w1, f.w_bf16, col) : 1.0f);
        if (f.b1) v = fmaf(s[1], ld_w(f.b1, f.w_bf16, col), v);
        leave(f.dgate, f.beta * v);
    }
}

// ---- host side ----------------------------------------------------------------------------------
// Most partial rows of a sum over tokens (sizes the workspace): enough for one per resident CTA.
static long long max_parts(long long T, int D) {
    long long n = (1ll << 21) / D;
    if (n < 1024) n = 1024;
    if (n > 4096) n = 4096;
    if (n > T) n = T;
    return n < 1 ? 1 : n;
}
static long long part_stride(long long parts, int D) { return (parts * D + 63) & ~63ll; }
static size_t sums_offset(long long T, int D) { return 4 * (size_t)part_stride(max_parts(T, D), D) * sizeof(float); }

static int row_grid(long long T) { return (int)(T < 148 * 8 ? T : 148 * 8); }

static bool kind_ok(int k) { return k == RLF_NORM_RMS || k == RLF_NORM_LAYER || k == RLF_NORM_NONE; }
static rlf_status check_block(int64_t T, int32_t D, rlf_dtype dt, rlf_dtype w_dt, int post, int pre, int gate_form, float alpha, float beta) {
    if ((dt != RLF_BF16 && dt != RLF_F32) || (w_dt != RLF_BF16 && w_dt != RLF_F32)) return RLF_ERR_DTYPE;
    if (T < 0 || D < 1) return RLF_ERR_SHAPE;
    if (D >= (1 << 30)) return RLF_ERR_UNSUPPORTED;    // the kernels count columns in 32 bits
    if (!kind_ok(post) || !kind_ok(pre) || (post == RLF_NORM_NONE && pre == RLF_NORM_NONE)) return RLF_ERR_UNSUPPORTED;
    if (gate_form < RLF_GATE_NONE || gate_form > RLF_GATE_ROW) return RLF_ERR_UNSUPPORTED;
    if (!(alpha - alpha == 0.0f) || !(beta - beta == 0.0f)) return RLF_ERR_UNSUPPORTED;      // finite
    return RLF_OK;
}

static rlf_status launch_finish(const Finish& f, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    cfg.gridDim = dim3((unsigned)((f.D + 31) / 32), 2);
    cfg.blockDim = dim3(1024);
    cfg.stream = s;
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, block_finish_kernel, f) != cudaSuccess) {
        cudaGetLastError();
        return RLF_ERR_CUDA;
    }
    count_launch();
    return RLF_OK;
}

}  // namespace bn

size_t block_norm_bwd_workspace_bytes(int64_t T, int32_t D) {
    if (T < 0 || D < 1) return 0;
    return bn::sums_offset(T, D) + (size_t)T * sizeof(float2);
}

}  // namespace rlf

extern "C" rlf_status rlf_block_norm_fwd(const void* x, int64_t x_stride, const void* residual, rlf_dtype dt, int64_t T, int32_t D,
                                         const void* post_weight, const void* post_bias, int post_kind, const void* pre_weight,
                                         const void* pre_bias, int pre_kind, rlf_dtype w_dt, const void* gate, int gate_form, float alpha,
                                         float beta, float eps, void* h_out, void* y_out, float* stats_out, rlf_stream_t stream) {
    using namespace rlf;
    using namespace rlf::bn;
    rlf_status st = check_block(T, D, dt, w_dt, post_kind, pre_kind, gate_form, alpha, beta);
    if (st != RLF_OK) return st;
    if (x_stride < D) return RLF_ERR_SHAPE;
    if (!(eps > 0.0f) || !(eps < INFINITY)) return RLF_ERR_UNSUPPORTED;
    if (T == 0) return RLF_OK;
    const bool post = post_kind != RLF_NORM_NONE, pre = pre_kind != RLF_NORM_NONE;
    if (!x || !residual || !h_out || (post && !post_weight) || (pre && (!pre_weight || !y_out)) || (gate_form != RLF_GATE_NONE && !gate))
        return RLF_ERR_NULL;
    const size_t esz = dt == RLF_BF16 ? 2 : 4, wsz = w_dt == RLF_BF16 ? 2 : 4;
    if (!aligned(x, esz) || !aligned(residual, esz) || !aligned(h_out, esz) || !aligned(y_out, esz) || !aligned(post_weight, wsz) ||
        !aligned(post_bias, wsz) || !aligned(pre_weight, wsz) || !aligned(pre_bias, wsz) ||
        !aligned(gate, gate_form == RLF_GATE_ROW ? 4 : wsz) || !aligned(stats_out, 4))
        return RLF_ERR_ALIGN;
    st = check_arch();
    if (st != RLF_OK) return st;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    BlockParams p = {};
    p.x = x; p.x_stride = x_stride; p.res = residual;
    p.w1 = post ? post_weight : nullptr; p.b1 = post ? post_bias : nullptr; p.w2 = pre ? pre_weight : nullptr; p.b2 = pre ? pre_bias : nullptr;
    p.gate = gate; p.w_bf16 = w_dt == RLF_BF16; p.post = post_kind; p.pre = pre_kind; p.gate_form = gate_form;
    p.alpha = alpha; p.beta = beta; p.eps = eps; p.h = h_out; p.y = y_out; p.stats = stats_out; p.T = T; p.D = D;
    if (dt == RLF_BF16) block_fwd_general_kernel<__nv_bfloat16><<<row_grid(T), kGenThreads, 0, s>>>(p);
    else block_fwd_general_kernel<float><<<row_grid(T), kGenThreads, 0, s>>>(p);
    count_launch();
    return cuda_ok(cudaGetLastError());
}

extern "C" rlf_status rlf_block_norm_bwd(const void* grad_y, const void* grad_h, const void* x, int64_t x_stride, const void* h, rlf_dtype dt,
                                         int64_t T, int32_t D, const void* post_weight, const void* post_bias, int post_kind,
                                         const void* pre_weight, int pre_kind, rlf_dtype w_dt, const void* gate, int gate_form, float alpha,
                                         float beta, const float* stats, void* grad_x, void* grad_residual, float* grad_gate,
                                         float* grad_post_weight, float* grad_post_bias, float* grad_pre_weight, float* grad_pre_bias,
                                         int accumulate, void* workspace, size_t workspace_bytes, rlf_stream_t stream) {
    using namespace rlf;
    using namespace rlf::bn;
    rlf_status st = check_block(T, D, dt, w_dt, post_kind, pre_kind, gate_form, alpha, beta);
    if (st != RLF_OK) return st;
    if (x_stride < D) return RLF_ERR_SHAPE;
    const bool post = post_kind != RLF_NORM_NONE, pre = pre_kind != RLF_NORM_NONE;
    if ((!post && (grad_post_weight || grad_post_bias)) || (!pre && (grad_pre_weight || grad_pre_bias)) ||
        (gate_form == RLF_GATE_NONE && grad_gate))
        return RLF_ERR_UNSUPPORTED;
    const bool col_gate = gate_form == RLF_GATE_COLUMN;
    const int want = (grad_pre_weight ? 1 : 0) | (grad_pre_bias ? 2 : 0) | (grad_post_weight || (col_gate && grad_gate) ? 4 : 0) |
                     (grad_post_bias || (col_gate && grad_gate && post && post_bias) ? 8 : 0);
    if (T > 0 && (!x || !stats || (post && !post_weight) || (pre && (!pre_weight || !grad_y || !h)) || (!pre && !grad_h)))
        return RLF_ERR_NULL;
    if (gate_form != RLF_GATE_NONE && !gate) return RLF_ERR_NULL;      // (read by the sums' last step even without tokens)
    const size_t esz = dt == RLF_BF16 ? 2 : 4, wsz = w_dt == RLF_BF16 ? 2 : 4;
    if (!aligned(grad_y, esz) || !aligned(grad_h, esz) || !aligned(x, esz) || !aligned(h, esz) || !aligned(grad_x, esz) ||
        !aligned(grad_residual, esz) || !aligned(post_weight, wsz) || !aligned(post_bias, wsz) || !aligned(pre_weight, wsz) ||
        !aligned(gate, gate_form == RLF_GATE_ROW ? 4 : wsz) || !aligned(stats, 4) || !aligned(grad_gate, 4) || !aligned(grad_post_weight, 4) ||
        !aligned(grad_post_bias, 4) || !aligned(grad_pre_weight, 4) || !aligned(grad_pre_bias, 4))
        return RLF_ERR_ALIGN;
    if (want && (!workspace || !aligned(workspace, 256) || workspace_bytes < block_norm_bwd_workspace_bytes(T, D))) return RLF_ERR_WORKSPACE;
    st = check_arch();
    if (st != RLF_OK) return st;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    BlockParams p = {};
    p.x = x; p.x_stride = x_stride; p.h = const_cast<void*>(h);
    p.w1 = post ? post_weight : nullptr; p.b1 = post ? post_bias : nullptr; p.w2 = pre ? pre_weight : nullptr;
    p.gate = gate; p.w_bf16 = w_dt == RLF_BF16; p.post = post_kind; p.pre = pre_kind; p.gate_form = gate_form;
    p.alpha = alpha; p.beta = beta; p.stats = const_cast<float*>(stats); p.dy = grad_y; p.dh = grad_h; p.dx = grad_x; p.dres = grad_residual;
    p.dgate_row = gate_form == RLF_GATE_ROW ? grad_gate : nullptr;
    p.want = want; p.T = T; p.D = D;
    float* part = static_cast<float*>(workspace);
    int parts = 0;
    const bool bf16 = dt == RLF_BF16;
    if (T > 0 && (grad_x || grad_residual || p.dgate_row || want)) {
        if (want) p.row_sums = reinterpret_cast<float2*>(static_cast<char*>(workspace) + sums_offset(T, D));
        if (bf16) block_bwd_general_kernel<__nv_bfloat16><<<row_grid(T), kGenThreads, 0, s>>>(p);
        else block_bwd_general_kernel<float><<<row_grid(T), kGenThreads, 0, s>>>(p);
        count_launch();
        if (cudaGetLastError() != cudaSuccess) return RLF_ERR_CUDA;
        if (want) {
            const long long rows = T < 1024 ? 1 : (T + 127) / 128;       // per slice: at most 128 slices of a long batch
            parts = (int)((T + rows - 1) / rows);
            p.part = part;
            p.part_stride = part_stride(parts, D);
            const dim3 grid((unsigned)((D + 31) / 32), (unsigned)parts);
            if (bf16) block_sums_general_kernel<__nv_bfloat16><<<grid, 256, 0, s>>>(p, rows);
            else block_sums_general_kernel<float><<<grid, 256, 0, s>>>(p, rows);
            count_launch();
            if (cudaGetLastError() != cudaSuccess) return RLF_ERR_CUDA;
        }
    }
    if (!want) return RLF_OK;
    Finish f = {};
    f.part = part; f.part_stride = part_stride(parts, D); f.parts = parts; f.D = D; f.want = want; f.accumulate = accumulate;
    f.w1 = p.w1; f.b1 = p.b1; f.gate = gate; f.w_bf16 = p.w_bf16; f.gate_form = gate_form; f.beta = beta;
    f.dw2 = grad_pre_weight; f.db2 = grad_pre_bias; f.dw1 = grad_post_weight; f.db1 = grad_post_bias; f.dgate = col_gate ? grad_gate : nullptr;
    return launch_finish(f, s);
}
