// The norms after a block and before the next, with the block's gate and the residual's scale, in one pass over the rows:
//
//   n = norm_post(x);   h = alpha residual + beta gate n;   y = norm_pre(h)            (either norm may be absent)
// norms as in norm.cu (RMS, or layer with mean and bias); the gate is a vector over the columns, one number per row, or absent.
// Backward, from dy (gradient of y) and dh (gradient that reaches h along the residual stream), with u = (h - m2) r2, v = (x - m1) r1:
//   gh = dh + r2 (q - [layer] mean(q) - u mean(q u)),  q = dy w_pre;                     d residual = alpha gh
//   with s = beta gate:   dx = r1 (g - [layer] mean(g) - v mean(g v)),  g = s gh w_post   (no norm: dx = s gh)
//   dw_pre = sum_t dy u,  db_pre = sum_t dy,  dw_post = sum_t s gh v,  db_post = sum_t s gh,  dgate = beta sum gh n  (over t, or the row)
//
// Bound by HBM: forward reads two rows and writes two, backward reads four and writes two (32768 x 2560 bf16 RMS: 108 us, 6.2 TB/s, and
// 162 us, 6.2; as calls 109 - 113 and 168 - 175; the layer forms with biases by latency, 8191 x 4096: 55 us, 4.9 TB/s, and 88, 4.6).  Statistics and sums are fp32 and no
// intermediate is rounded: y comes from the unrounded h, dx from the unrounded gh.
// A column gate is a factor of the post norm's sums over tokens, S1 = sum_t [row gate] gh v and S2 = sum_t [row gate] gh, so that
// the gradients of gate, weight and bias all come from these two (finish kernel).
#include "norm_rows.cuh"
#include "row.cuh"

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
constexpr int kSmemLimit = 200 * 1024;           // most dynamic shared memory that a fast form asks for

// ---- any width, stride and alignment: one CTA per row, the row read once per pass (later passes are served by L2): rows shorter than a
// vector, longer than 8192 elements, or of tensors that sit apart in their vectors (4096 x 16384 bf16 470 us forward, 1021 backward, where
// the bytes are 82 and 123) --------
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

// the same shared-memory float of CTA `rank` of this cluster
__device__ __forceinline__ float ld_cluster_f32(const float* p, uint32_t rank) {
    uint32_t at;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
    return v;
}
struct Finish {
    const float* part;
    long long part_stride;
    int parts, D, want, accumulate, split;
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
// partial rows -> gradients, added in a fixed order: a cluster of `split` CTAs covers 32 columns of the pre (blockIdx.y = 0) or
// post norm's two sums.  Warp w of all of them adds the partial rows w, w + 32 split, ..., and the 32 sums are added in order,
// then the CTAs' (with one CTA the many partial rows of narrow rows were this kernel's whole time: backward of 5768 x 128 fp32,
// 2960 partial rows, 32 us, so 11).
__global__ void __launch_bounds__(1024)
block_finish_kernel(const Finish f) {
    __shared__ float acc[2][32][33];
    __shared__ float total[2][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t block;
    asm volatile("mov.u32 %0, %%clusterid.x;" : "=r"(block));
    const int rank = (int)cluster_ctarank(), col0 = (int)block * 32, first = 2 * blockIdx.y, step = 32 * f.split;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int col = col0 + lane;
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if (col < f.D && ((f.want >> (first + k)) & 1)) {
            const float* src = f.part + (first + k) * f.part_stride + col;
#pragma unroll 8
            for (int r = rank * 32 + warp; r < f.parts; r += step) s[k] += src[(long long)r * f.D];
        }
        acc[k][warp][lane] = s[k];
    }
    __syncthreads();
    if (warp == 0) {
        for (int w = 1; w < 32; ++w) {
            s[0] += acc[0][w][lane];
            s[1] += acc[1][w][lane];
        }
    }
    if (f.split > 1) {
        if (warp == 0) {
            total[0][lane] = s[0];
            total[1][lane] = s[1];
        }
        cluster_sync_all();
        if (warp == 0 && rank == 0)
            for (int q = 1; q < f.split; ++q) {
                s[0] += ld_cluster_f32(&total[0][lane], (uint32_t)q);
                s[1] += ld_cluster_f32(&total[1][lane], (uint32_t)q);
            }
        cluster_sync_all();                                // the others' sums have been read
    }
    if (warp != 0 || rank != 0 || col >= f.D) return;
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

// ---- fast forms ---------------------------------------------------------------------------------
// A CTA works on R rows at a time, with the next R rows on their way into the other half of a shared-memory buffer (cp.async);
// a thread owns NV 16-byte vectors of each row.  EDGE: rows on no boundary, all dense tensors' rows alike; a CTA then takes
// every period-th row, whose places in their vectors are the same, and a row's first and last vector are masked.  The rows of
// x, whose stride is its own, may sit otherwise (x_shift): they are copied as the aligned chunks that cover them and read by
// element.
__host__ __device__ constexpr int shifted_pitch(int D, int esz) { return staged_pitch(D, esz) + 48; }     // (read from 16 before to 32 behind)
template <typename T, int NV, int R, bool EDGE, int BUFS = 2>
struct Stage {
    static constexpr int P = Vec<T>::P, N = Vec<T>::N;
    const BlockParams& p;
    const Rows<T, EDGE> rows;
    uint4* slots;                   // [BUFS][R][arrays][NV][threads], a slot is its thread's own
    char* shifted;                  // [BUFS][R] rows of x
    int arrays, pitch, th, tid;
    bool shift;
    unsigned keep[NV];              // which elements of a vector are the row's
    __device__ __forceinline__ Stage(const BlockParams& p_, uint4* smem, const void* dense, int arrays_)
        : p(p_), rows(dense, p_.D, p_.T, p_.D, p_.period, R), slots(smem), arrays(arrays_), th(blockDim.x), tid(threadIdx.x) {
        shift = EDGE && p.x_shift;
        pitch = shifted_pitch(p.D, (int)sizeof(T));
        shifted = reinterpret_cast<char*>(smem + BUFS * R * arrays * NV * th);
#pragma unroll
        for (int i = 0; i < NV; ++i) keep[i] = EDGE ? rows.bits(tid + i * th, p.D) : (1u << N) - 1u;
    }
    // a first or last vector that other elements than the row's are in
    __device__ __forceinline__ bool partial(int i) const { return EDGE && keep[i] != (1u << N) - 1u; }
    __device__ __forceinline__ uint4 masked(uint4 q, int i) const {
        auto word = [&](int k) {
            if (N == 4) return (keep[i] >> k) & 1u ? 0xffffffffu : 0u;
            return ((keep[i] >> (2 * k)) & 1u ? 0xffffu : 0u) | ((keep[i] >> (2 * k + 1)) & 1u ? 0xffff0000u : 0u);
        };
        return make_uint4(q.x & word(0), q.y & word(1), q.z & word(2), q.w & word(3));
    }
    // what lies outside the rows of a batch that has arrived becomes zero (in the few slots concerned)
    __device__ __forceinline__ void trim(int buf) const {
        if constexpr (EDGE) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (partial(i))
                    for (int q = 0; q < R * arrays; ++q) {
                        uint4* at = slot(buf, 0, q, i);
                        *at = masked(*at, i);
                    }
        }
    }
    __device__ __forceinline__ bool mine(int i) const { return tid + i * th < rows.nvec; }
    __device__ __forceinline__ uint4* slot(int buf, int k, int a, int i) const { return slots + (((buf * R + k) * arrays + a) * NV + i) * th + tid; }
    __device__ __forceinline__ void copy(int buf, int k, int a, const void* tensor, long long stride, long long t) const {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (mine(i)) rows.copy(slot(buf, k, a, i), static_cast<const T*>(tensor) + t * stride, tid + i * th, p.D, t == 0);
    }
    // Slots that no copy writes (of threads without a vector i, or of a tensor that is not there) hold zeros, so that the
    // arithmetic needs no conditions: under conditions the values carried from pass to pass cost more moves than arithmetic.
    __device__ __forceinline__ void clear(int a, bool all) const {
        for (int q = 0; q < BUFS * R; ++q)
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (all || !mine(i)) *slot(0, q, a, i) = make_uint4(0u, 0u, 0u, 0u);
    }
    // x goes into array a, or to its own place
    __device__ __forceinline__ void copy_x(int buf, int k, int a, long long t) const {
        if (shift) copy_row<T>(shifted + (buf * R + k) * pitch + 16, static_cast<const T*>(p.x) + t * p.x_stride, p.D, t == 0);
        else copy(buf, k, a, p.x, p.x_stride, t);
    }
    __device__ __forceinline__ void read(int buf, int k, int a, int i, f2 (&v)[P]) const { Vec<T>::unpack(*slot(buf, k, a, i), v); }
    // A vector of a row that lies otherwise: two aligned pieces of it, shifted by the same distance in every thread.
    __device__ __forceinline__ void read_x(int buf, int k, int a, int i, long long t, f2 (&v)[P]) const {
        if (!EDGE || !shift) {
            read(buf, k, a, i, v);
            return;
        }
        const int first = 16 + chunk_head(static_cast<const T*>(p.x) + t * p.x_stride) - rows.lead * (int)sizeof(T);
        const uint4* from = reinterpret_cast<const uint4*>(shifted + (buf * R + k) * pitch + (first & ~15)) + min(tid + i * th, rows.nvec - 1);
        const uint4 q0 = from[0], q1 = from[1];
        uint32_t w[8] = {q0.x, q0.y, q0.z, q0.w, q1.x, q1.y, q1.z, q1.w};
        const bool by8 = first & 8, by4 = first & 4;
#pragma unroll
        for (int e = 0; e < 6; ++e) w[e] = by8 ? w[e + 2] : w[e];
#pragma unroll
        for (int e = 0; e < 5; ++e) w[e] = by4 ? w[e + 1] : w[e];
        if constexpr (sizeof(T) == 2) {
            const unsigned bits = (first & 2) * 8;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = __funnelshift_r(w[e], w[e + 1], bits);
        }
        uint4 q = make_uint4(w[0], w[1], w[2], w[3]);
        if (partial(i)) q = masked(q, i);
        Vec<T>::unpack(q, v);
    }
    __device__ __forceinline__ void store(void* tensor, long long t, int i, const f2 (&v)[P]) const {
        rows.store(static_cast<T*>(tensor) + t * p.D, tid + i * th, Vec<T>::pack(v), keep[i]);
    }
    // zeros outside the row
    __device__ __forceinline__ void mask(int i, f2 (&v)[P]) const { mask_pairs<P>(v, keep[i]); }
    // this thread's columns of a [D] vector (0 outside the width); `none`: what stands for a vector that is not there
    __device__ __forceinline__ void columns(f2 (&f)[NV][P], const void* w, float none) const {
        const bool wide = !EDGE && (reinterpret_cast<uintptr_t>(w) & 15) == 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (tid + i * th) * N - rows.lead;
            if (wide && w != nullptr) {
                if (!mine(i)) {
#pragma unroll
                    for (int e = 0; e < P; ++e) f[i][e] = 0ull;
                } else if (p.w_bf16) {
#pragma unroll
                    for (int e = 0; e < P; e += 2) {
                        const uint2 q = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(w) + c + 2 * e);
                        f[i][e] = f2_make(__uint_as_float(q.x << 16), __uint_as_float(q.x & 0xffff0000u));
                        f[i][e + 1] = f2_make(__uint_as_float(q.y << 16), __uint_as_float(q.y & 0xffff0000u));
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < P; e += 2) {
                        const float4 q = *reinterpret_cast<const float4*>(static_cast<const float*>(w) + c + 2 * e);
                        f[i][e] = f2_make(q.x, q.y);
                        f[i][e + 1] = f2_make(q.z, q.w);
                    }
                }
                continue;
            }
            auto at = [&](int k) { return k < 0 || k >= p.D ? 0.0f : w ? ld_w(w, p.w_bf16, k) : none; };
#pragma unroll
            for (int e = 0; e < P; ++e) f[i][e] = f2_make(at(c + 2 * e), at(c + 2 * e + 1));
        }
    }
    // post norm's weight (and bias) times column gate and branch scale
    __device__ __forceinline__ void post_columns(f2 (&f)[NV][P], const void* w, float none) const {
        columns(f, w, none);
        if (p.gate_form == RLF_GATE_COLUMN) {
            f2 g[NV][P];
            columns(g, p.gate, 1.0f);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < P; ++e) f[i][e] = f2_mul(f[i][e], g[i][e]);
        }
        if (p.beta != 1.0f) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < P; ++e) f[i][e] = f2_mul(f[i][e], f2_make(p.beta, p.beta));
        }
    }
};
// K sums over the CTA of at most W warps, the same in every thread afterwards (one barrier; `red` holds two halves of [K][W]
// floats used in turn, zeros where a warp is missing).  W is known to the compiler: reading the warps' parts in a loop cost
// more instructions than the rest of a short row.
template <int K, int W>
__device__ __forceinline__ void row_sums(float (&v)[K], float* red, int& turn) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    if (blockDim.x == 32) return;
    float* r = red + turn * K * W;
    turn ^= 1;
    if (lane == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) r[k * W + warp] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        f2 a = 0ull;
#pragma unroll
        for (int q = 0; q < W / 4; ++q) {
            const ulonglong2 x = *reinterpret_cast<const ulonglong2*>(r + k * W + 4 * q);
            a = f2_add(a, f2_add(x.x, x.y));
        }
        v[k] = f2_sum(a);
    }
}
template <int N>
__device__ __forceinline__ void clear_sums(float (&red)[N]) {
    for (int i = threadIdx.x; i < N; i += blockDim.x) red[i] = 0.0f;
    __syncthreads();
}

__device__ __forceinline__ f2 f2_dup(float v) { return f2_make(v, v); }

// L: a mean or a bias is in it somewhere (the RMS norms without bias keep no registers for them)
template <typename T, int NV, int R, bool L, bool EDGE, int MAXT>
__global__ void __launch_bounds__(MAXT)
block_fwd_kernel(const BlockParams p) {
    using V = Vec<T>;
    constexpr int P = V::P;
    extern __shared__ __align__(16) uint4 smem[];       // residual, x (where it is like the others)
    __shared__ __align__(16) float red[2 * (MAXT / 32) * R];
    int turn = 0;
    clear_sums(red);
    const Stage<T, NV, R, EDGE> st(p, smem, p.res, EDGE && p.x_shift ? 1 : 2);
    const float inv_d = 1.0f / (float)p.D;
    const bool post = has_norm(p.post), pre = has_norm(p.pre);
    st.clear(0, false);
    if (!st.shift) st.clear(1, false);
    float gate_next[R];
    auto fetch = [&](long long j0, int buf) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            gate_next[k] = 1.0f;
            if (j0 + k < st.rows.n) {
                const long long t = st.rows.row(j0 + k);
                gate_next[k] = row_gate(p, t);
                st.copy(buf, k, 0, p.res, p.D, t);
                st.copy_x(buf, k, 1, t);
            }
        }
        nm::cp_async_commit();
    };
    long long j0 = st.rows.first;
    fetch(j0, 0);
    f2 w1[NV][P], w2[NV][P], b1[L ? NV : 1][P], b2[L ? NV : 1][P];
    st.post_columns(w1, p.w1, 1.0f);
    st.columns(w2, p.w2, 0.0f);
    if constexpr (L) {
        st.post_columns(b1, p.b1, 0.0f);
        st.columns(b2, p.b2, 0.0f);
    }
    const f2 alpha = f2_dup(p.alpha);
    for (int buf = 0; j0 < st.rows.n; j0 += st.rows.step, buf ^= 1) {
        float gate[R];
#pragma unroll
        for (int k = 0; k < R; ++k) gate[k] = gate_next[k];
        if (st.shift) __syncthreads();                  // the other half has been read by everyone
        fetch(j0 + st.rows.step, buf ^ 1);
        cp_async_wait1();
        if (st.shift) __syncthreads();                  // everyone's chunks of this half are here
        st.trim(buf);
        f2 v[R][NV][P];
        float m1[R], r1[R], m2[R], r2[R], s[R];
        // mean and 1 / spread of the rows held in v
        auto stats = [&](bool layer, float (&m)[R], float (&r)[R]) {
            if (L && layer) {
#pragma unroll
                for (int k = 0; k < R; ++k) {
                    f2 q = 0ull;
#pragma unroll
                    for (int i = 0; i < NV; ++i)
#pragma unroll
                        for (int e = 0; e < P; ++e) q = f2_add(q, v[k][i][e]);
                    s[k] = f2_sum(q);
                }
                row_sums<R, MAXT / 32>(s, red, turn);
            }
#pragma unroll
            for (int k = 0; k < R; ++k) {
                m[k] = L && layer ? s[k] * inv_d : 0.0f;
                const f2 c = f2_dup(-m[k]);
                f2 q = 0ull;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    // (a thread without a vector i holds zeros, which stay it)
                    const f2 here = st.mine(i) ? c : 0ull;
                    f2 part = 0ull;
#pragma unroll
                    for (int e = 0; e < P; ++e) {
                        const f2 d = L ? f2_add(v[k][i][e], here) : v[k][i][e];
                        part = f2_fma(d, d, part);
                    }
                    if (L && st.partial(i)) {
                        f2 d[P];
#pragma unroll
                        for (int e = 0; e < P; ++e) d[e] = f2_add(v[k][i][e], c);
                        st.mask(i, d);
                        part = 0ull;
#pragma unroll
                        for (int e = 0; e < P; ++e) part = f2_fma(d[e], d[e], part);
                    }
                    q = f2_add(q, part);
                }
                s[k] = f2_sum(q);
            }
            row_sums<R, MAXT / 32>(s, red, turn);
#pragma unroll
            for (int k = 0; k < R; ++k) r[k] = rsqrtf(s[k] * inv_d + p.eps);
        };
#pragma unroll
        for (int k = 0; k < R; ++k) {
            m1[k] = m2[k] = 0.0f;
            r1[k] = r2[k] = 1.0f;
            const long long t = st.rows.row(min(j0 + k, st.rows.n - 1));
#pragma unroll
            for (int i = 0; i < NV; ++i) st.read_x(buf, k, 1, i, t, v[k][i]);
        }
        if (post) stats(p.post == RLF_NORM_LAYER, m1, r1);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const f2 c = f2_dup(-m1[k]), r = f2_dup(r1[k] * gate[k]), g = f2_dup(gate[k]);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                f2 res[P];
                st.read(buf, k, 0, i, res);
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    f2 n = f2_mul(f2_mul(L ? f2_add(v[k][i][e], c) : v[k][i][e], r), w1[i][e]);
                    if (L) n = f2_fma(g, b1[L ? i : 0][e], n);
                    v[k][i][e] = f2_fma(alpha, res[e], n);
                }
            }
        }
        if (pre) stats(p.pre == RLF_NORM_LAYER, m2, r2);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            if (j0 + k >= st.rows.n) continue;
            const long long t = st.rows.row(j0 + k);
            const f2 c = f2_dup(-m2[k]), r = f2_dup(r2[k]);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                f2 o[P];
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    o[e] = f2_mul(f2_mul(L ? f2_add(v[k][i][e], c) : v[k][i][e], r), w2[i][e]);
                    if (L) o[e] = f2_add(o[e], b2[L ? i : 0][e]);
                }
                if (st.mine(i)) {
                    st.store(p.h, t, i, v[k][i]);
                    if (pre) st.store(p.y, t, i, o);
                }
            }
            if (st.tid == 0 && p.stats) {
                p.stats[t] = m1[k];
                p.stats[p.T + t] = r1[k];
                p.stats[2 * p.T + t] = m2[k];
                p.stats[3 * p.T + t] = r2[k];
            }
        }
    }
    cp_async_wait0();
}

// Backward, one row at a time: two sums per row one after the other (the second needs gh, which needs the first); what the later
// passes need is held in registers, so that each element is unpacked once.  The sums over tokens are added up row after row in
// registers and leave as one partial row per CTA.
// Rows too long for two buffers (ONE: fp32, wider than 5000 to 6200 columns) take one, and a slot is filled again as soon as it has been read
// (8949 x 7104 fp32 layer form 277 us; by the general form 1200).
template <typename T, int NV, bool L, bool EDGE, int MAXT, bool ONE>
__global__ void __launch_bounds__(MAXT, !L && !EDGE ? 0 : NV * Vec<T>::N <= 16 && MAXT <= 256 ? 512 / MAXT : 1)
block_bwd_kernel(const BlockParams p) {
    using V = Vec<T>;
    constexpr int P = V::P, N = V::N, K = L ? 2 : 1, W = MAXT / 32;
    constexpr bool WS = L || EDGE;                              // the weights live in shared memory (a thread's own columns), not in registers
    extern __shared__ __align__(16) uint4 smem[];       // dh, dy, h (zeros for what is not there), x (where it is like the others)
    __shared__ __align__(16) float red[2 * W * K];
    int turn = 0;
    clear_sums(red);
    const bool post = has_norm(p.post), pre = has_norm(p.pre);
    const Stage<T, NV, 1, EDGE, ONE ? 1 : 2> st(p, smem, pre ? p.h : p.dh, EDGE && p.x_shift ? 3 : 4);
    const float inv_d = 1.0f / (float)p.D;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    st.clear(0, p.dh == nullptr);
    st.clear(1, !pre);
    st.clear(2, !pre);
    if (!st.shift) st.clear(3, false);
    float next[5];                                      // the row's statistics and gate
    auto fetch = [&](long long j, int buf) {
        if (j < st.rows.n) {
            const long long t = st.rows.row(j);
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (L || (q & 1)) next[q] = p.stats[q * p.T + t];
            next[4] = row_gate(p, t);
            if (p.dh) st.copy(buf, 0, 0, p.dh, p.D, t);
            if (pre) {
                st.copy(buf, 0, 1, p.dy, p.D, t);
                st.copy(buf, 0, 2, p.h, p.D, t);
            }
            if (!ONE) st.copy_x(buf, 0, 3, t);
        }
        nm::cp_async_commit();
    };
    auto fetch_x = [&](long long j) {                   // (ONE)
        if (j < st.rows.n) st.copy_x(0, 0, 3, st.rows.row(j));
        nm::cp_async_commit();
    };
    long long j = st.rows.first;
    fetch(j, 0);
    if constexpr (ONE) fetch_x(j);
    f2 w1[WS ? 1 : NV][P], w2[WS ? 1 : NV][P], sum_dyu[NV][P], sum_ghv[NV][P], sum_dy[L ? NV : 1][P], sum_gh[L ? NV : 1][P];
    ulonglong2* const w_s = reinterpret_cast<ulonglong2*>(st.shifted + (st.shift ? (ONE ? 1 : 2) * st.pitch : 0)) + st.tid;    // [2][NV][P / 2][threads]
    if constexpr (WS) {
        f2 w[NV][P];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (k == 0) st.post_columns(w, p.w1, 1.0f);
            else st.columns(w, p.w2, 0.0f);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < P / 2; ++e) w_s[((k * NV + i) * (P / 2) + e) * st.th] = make_ulonglong2(w[i][2 * e], w[i][2 * e + 1]);
        }
    } else {
        st.post_columns(w1, p.w1, 1.0f);
        st.columns(w2, p.w2, 0.0f);
    }
    auto weights = [&](int k, int i, f2 (&w)[P]) {
        if constexpr (WS) {
#pragma unroll
            for (int e = 0; e < P / 2; ++e) {
                const ulonglong2 q = w_s[((k * NV + i) * (P / 2) + e) * st.th];
                w[2 * e] = q.x;
                w[2 * e + 1] = q.y;
            }
        } else {
#pragma unroll
            for (int e = 0; e < P; ++e) w[e] = k == 0 ? w1[WS ? 0 : i][e] : w2[WS ? 0 : i][e];
        }
    };
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < P; ++e) {
            sum_dyu[i][e] = sum_ghv[i][e] = 0ull;
            if (L) sum_dy[L ? i : 0][e] = sum_gh[L ? i : 0][e] = 0ull;
        }
    for (int buf = 0; j < st.rows.n; j += st.rows.step, buf ^= ONE ? 0 : 1) {
        const long long t = st.rows.row(j);
        const float m1 = next[0], r1 = next[1], m2 = next[2], r2 = next[3], gate = next[4];
        if constexpr (ONE) {
            cp_async_wait0();
        } else {
            if (st.shift) __syncthreads();
            fetch(j + st.rows.step, buf ^ 1);
            cp_async_wait1();
        }
        if (st.shift) __syncthreads();
        st.trim(buf);
        auto unit = [&](const f2& v, const f2& c, const f2& r) { return f2_mul(L ? f2_add(v, c) : v, r); };
        // gh: at first dh + r2 dy w2;  uv: u, then v
        f2 gh[NV][P], uv[NV][P];
        float s[K];
        {
            f2 a = 0ull, b = 0ull;
            const f2 c = f2_dup(-m2), r = f2_dup(r2);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                f2 dy[P], w[P];
                weights(1, i, w);
                st.read(buf, 0, 0, i, gh[i]);
                st.read(buf, 0, 1, i, dy);
                st.read(buf, 0, 2, i, uv[i]);
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    const f2 u = unit(uv[i][e], c, r), q = f2_mul(dy[e], w[e]);
                    uv[i][e] = u;
                    a = f2_fma(q, u, a);
                    gh[i][e] = f2_fma(q, r, gh[i][e]);
                    sum_dyu[i][e] = f2_fma(dy[e], u, sum_dyu[i][e]);
                    if (L) {
                        b = f2_add(b, q);
                        sum_dy[L ? i : 0][e] = f2_add(sum_dy[L ? i : 0][e], dy[e]);
                    }
                }
            }
            s[0] = f2_sum(a);
            if (L) s[K - 1] = f2_sum(b);
        }
        if constexpr (ONE) fetch(j + st.rows.step, 0);
        if (pre) row_sums<K, W>(s, red, turn);
        float bias_sum = 0.0f;
        {
            f2 a = 0ull, b = 0ull;
            const f2 ra = f2_dup(-r2 * (s[0] * inv_d)), rb = f2_dup(L && p.pre == RLF_NORM_LAYER ? -r2 * (s[K - 1] * inv_d) : 0.0f);
            const f2 c = f2_dup(-m1), r = f2_dup(r1), g = f2_dup(gate), al = f2_dup(p.alpha);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                f2 x[P], d[P], o[P], w[P];
                weights(0, i, w);
                st.read_x(buf, 0, 3, i, t, x);
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    d[e] = f2_fma(uv[i][e], ra, gh[i][e]);
                    if (L) d[e] = f2_add(d[e], rb);
                    const f2 v = unit(x[e], c, r), q = f2_mul(d[e], w[e]), sg = f2_mul(d[e], g);
                    gh[i][e] = q;                       // (all that is left to do needs gh w)
                    uv[i][e] = v;
                    o[e] = f2_mul(d[e], al);
                    a = f2_fma(q, v, a);
                    sum_ghv[i][e] = f2_fma(sg, v, sum_ghv[i][e]);
                    if (L) {
                        b = f2_add(b, q);
                        sum_gh[L ? i : 0][e] = f2_add(sum_gh[L ? i : 0][e], sg);
                    }
                }
                if (p.dres && st.mine(i)) st.store(p.dres, t, i, o);
                if (L && p.dgate_row && p.b1) {
#pragma unroll
                    for (int e = 0; e < P; ++e) {
                        const int col = (st.tid + i * st.th) * N + 2 * e - st.rows.lead;
                        float lo, hi;
                        f2_split(d[e], lo, hi);
                        if (col >= 0 && col < p.D) bias_sum = fmaf(lo, ld_w(p.b1, p.w_bf16, col), bias_sum);
                        if (col + 1 >= 0 && col + 1 < p.D) bias_sum = fmaf(hi, ld_w(p.b1, p.w_bf16, col + 1), bias_sum);
                    }
                }
            }
            s[0] = f2_sum(a);
            if (L) s[K - 1] = f2_sum(b);
        }
        if constexpr (ONE) {
            if (st.shift) __syncthreads();              // the row of x has been read by everyone
            fetch_x(j + st.rows.step);
        }
        if (post || p.dgate_row) row_sums<K, W>(s, red, turn);
        if (p.dgate_row) {
            if (L && p.b1) {
                float c[K] = {bias_sum};
                row_sums<K, W>(c, red, turn);
                bias_sum = c[0];
            }
            if (st.tid == 0) p.dgate_row[t] = fmaf(p.beta, bias_sum, s[0]);
        }
        if (p.dx == nullptr) continue;
        // gate r1 (gh w1 - b - v a)
        const float gr = gate * r1, a = post ? s[0] * inv_d : 0.0f, b = L && p.post == RLF_NORM_LAYER ? s[K - 1] * inv_d : 0.0f;
        const f2 r = f2_dup(gr), ra = f2_dup(-gr * a), rb = f2_dup(-gr * b);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            f2 o[P];
#pragma unroll
            for (int e = 0; e < P; ++e) o[e] = f2_fma(uv[i][e], ra, L ? f2_fma(gh[i][e], r, rb) : f2_mul(gh[i][e], r));
            if (st.mine(i)) st.store(p.dx, t, i, o);
        }
    }
    cp_async_wait0();
    auto leave = [&](int which, const f2 (&g)[P], int i) {
        if (!((p.want >> which) & 1) || !st.mine(i)) return;
        float* d = p.part + which * p.part_stride + (long long)blockIdx.x * p.D + (st.tid + i * st.th) * N - st.rows.lead;
        float v[N];
#pragma unroll
        for (int e = 0; e < P; ++e) f2_split(g[e], v[2 * e], v[2 * e + 1]);
        // whole vectors where rows fill them (as single floats these stores are partial sectors: 8191 x 4096 bf16, layer form: 102 us, so 87)
        if constexpr (!EDGE) {
#pragma unroll
            for (int e = 0; e < N; e += 4) *reinterpret_cast<float4*>(d + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if ((st.keep[i] >> e) & 1u) d[e] = v[e];
        }
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        leave(0, sum_dyu[i], i);
        leave(2, sum_ghv[i], i);
        if (L) {
            leave(1, sum_dy[L ? i : 0], i);
            leave(3, sum_gh[L ? i : 0], i);
        }
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

// how rows are cut: nv vectors per thread, `threads` threads, `rows` rows at a time in each of `buffers`, bytes of shared memory
struct Cut { int nv, threads, rows, smem, max_threads, buffers; };

// false: no fast form holds the rows (rows shorter than a vector, or longer than 8192 elements).  `arrays` rows are read per
// row besides a shifted x.  Up to 128 threads of one vector, then of two (fp32: four) vectors each; the backward of long bf16 rows
// four vectors on up to 256 threads (10240 x 8192 RMS 178 us with two on 512, 167 with four).  Forward two rows at a time
// where a CTA has up to 256 threads (8191 x 4096 layer form 61 us with one, 53 with two).
static bool pick_cut(bool bf16, bool edge, bool shift, bool fwd, bool full, long long T, int D, int arrays, Cut* c) {
    const int esz = bf16 ? 2 : 4, v = 16 / esz;
    if (D < v || D > 8192) return false;
    const int nvec = edge ? (D + 2 * v - 2) / v : D / v;
    const int most_nv = bf16 && (fwd || nvec <= 512) ? 2 : 4;
    c->nv = 1;
    while ((nvec + c->nv - 1) / c->nv > 128 && c->nv < most_nv) c->nv *= 2;
    c->threads = ((nvec + c->nv - 1) / c->nv + 31) / 32 * 32;
    if (c->threads > 512) return false;                    // (rows of 8192 on no boundary)
    c->max_threads = c->threads <= 128 ? 128 : c->threads <= 256 ? 256 : 512;
    if (!fwd && bf16 && c->max_threads == 512) return false;
    c->rows = !fwd || c->max_threads == 512 ? 1 : 2;
    while (c->rows > 1 && T < 148ll * 4 * c->rows) c->rows /= 2;      // too few rows to put several on a CTA
    c->buffers = 2;
    for (;;) {
        c->smem = c->buffers * c->rows * (arrays * c->nv * c->threads * 16 + (shift ? shifted_pitch(D, esz) : 0));
        if (!fwd && (full || edge)) c->smem += 2 * c->nv * c->threads * v * 4;         // the weights
        if (c->smem <= (c->rows > 1 ? kSmemLimit / 2 : kSmemLimit)) return true;
        if (c->rows > 1) c->rows /= 2;
        else if (!fwd && c->max_threads == 512 && c->buffers == 2) c->buffers = 1;
        else return false;
    }
}

typedef void (*BlockKernel)(const BlockParams);
template <typename T, int NV, bool L, bool EDGE, int MAXT>
static BlockKernel fwd_form(const Cut& c) {
    if constexpr (MAXT < 512) {
        if (c.rows == 2) return block_fwd_kernel<T, NV, 2, L, EDGE, MAXT>;
    }
    return block_fwd_kernel<T, NV, 1, L, EDGE, MAXT>;
}
template <bool FWD, typename T, int NV, bool L, bool EDGE, int MAXT>
static BlockKernel form(const Cut& c) {
    if constexpr (FWD) return fwd_form<T, NV, L, EDGE, MAXT>(c);
    if constexpr (!FWD && MAXT == 512) {
        if (c.buffers == 1) return block_bwd_kernel<T, NV, L, EDGE, MAXT, true>;
    }
    if constexpr (!FWD) return block_bwd_kernel<T, NV, L, EDGE, MAXT, false>;
}
template <bool FWD, typename T, bool L, bool EDGE>
static BlockKernel kernel_form(const Cut& c) {
    if (c.nv == 1) return form<FWD, T, 1, L, EDGE, 128>(c);
    if (c.nv == 2 && c.max_threads == 128) return form<FWD, T, 2, L, EDGE, 128>(c);
    if constexpr (sizeof(T) == 2) {
        if (c.nv == 2) return FWD && c.max_threads == 512 ? form<true, T, 2, L, EDGE, 512>(c) : form<FWD, T, 2, L, EDGE, 256>(c);
        if constexpr (!FWD) return form<false, T, 4, L, EDGE, 256>(c);
    } else {
        if (c.max_threads == 128) return form<FWD, T, 4, L, EDGE, 128>(c);
        return c.max_threads == 256 ? form<FWD, T, 4, L, EDGE, 256>(c) : form<FWD, T, 4, L, EDGE, 512>(c);
    }
    return nullptr;
}
template <bool FWD>
static BlockKernel kernel_of(bool bf16, bool full, bool edge, const Cut& c) {
    if (bf16) {
        if (full) return edge ? kernel_form<FWD, __nv_bfloat16, true, true>(c) : kernel_form<FWD, __nv_bfloat16, true, false>(c);
        return edge ? kernel_form<FWD, __nv_bfloat16, false, true>(c) : kernel_form<FWD, __nv_bfloat16, false, false>(c);
    }
    if (full) return edge ? kernel_form<FWD, float, true, true>(c) : kernel_form<FWD, float, true, false>(c);
    return edge ? kernel_form<FWD, float, false, true>(c) : kernel_form<FWD, float, false, false>(c);
}

// CTAs of this kernel that are resident at once (0: none fits); opts the kernel in to its shared memory on the way
static int resident_ctas(const void* k, const Cut& c) {
    static ResidentTable table;
    return table.get(k, c.threads, c.smem, [&](int dev) {
        int per_sm = 0, sms = 0;
        if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit) != cudaSuccess ||
            cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, k, c.threads, c.smem) != cudaSuccess) {
            cudaGetLastError();
            per_sm = 0;
        }
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
        return per_sm * (sms > 0 ? sms : 148);
    });
}

// Which fast form fits the tensors' rows (the first of `at` is dense): sets period and x_shift.
static bool fast_form(bool bf16, long long T, int D, const void* const* at, int n, const void* x, long long x_stride, BlockParams* p, bool* edge) {
    int period = 1;
    const Form form = row_form(bf16, T, D, at, n, D, D, &period);
    if (form == kStaged) return false;
    const int v = bf16 ? 8 : 4;
    const bool alike = (reinterpret_cast<uintptr_t>(x) - reinterpret_cast<uintptr_t>(at[0])) % 16 == 0 && (T <= 1 || x_stride % v == D % v);
    p->period = period;
    p->x_shift = !alike;
    *edge = form == kEdge || !alike;
    return true;
}
static long long batches(long long T, const Cut& c, int period) {
    const long long rows = (T + period - 1) / period;
    return (rows + c.rows - 1) / c.rows * period;
}

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
    cudaLaunchAttribute at[2];
    cfg.gridDim = dim3((unsigned)((f.D + 31) / 32 * f.split), 2);
    cfg.blockDim = dim3(1024);
    cfg.stream = s;
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = f.split;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = f.split > 1 ? 2 : 1;
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
    const bool bf16 = dt == RLF_BF16, full = post_kind == RLF_NORM_LAYER || pre_kind == RLF_NORM_LAYER || p.b1 || p.b2;
    const void* const at[] = {residual, h_out, pre ? y_out : nullptr};
    bool edge;
    Cut c;
    if (fast_form(bf16, T, D, at, 3, x, x_stride, &p, &edge) && pick_cut(bf16, edge, p.x_shift, true, full, T, D, p.x_shift ? 1 : 2, &c)) {
        const BlockKernel k = kernel_of<true>(bf16, full, edge, c);
        const int resident = k ? resident_ctas((const void*)k, c) : 0;
        if (resident > 0) {
            long long grid = batches(T, c, p.period);
            // RMS: CTAs that retire early, up to eight generations of them, keep the loads of some under the stores of others (32768 x 2560
            // bf16: 125 us as one generation, 111 as four, 104 as eight); with means and biases, or rows on no boundary, a CTA's start
            // costs more than that gains (8191 x 4096 layer form 53 us as one, 61 as four; 20000 x 2603 RMS 106 and 129)
            long long gens = full || edge ? 1 : grid / (4ll * resident);
            gens = gens < 1 ? 1 : gens > 8 ? 8 : gens;
            if (grid > gens * resident) grid = gens * resident / p.period * p.period;
            k<<<(unsigned)grid, c.threads, c.smem, s>>>(p);
            count_launch();
            return cuda_ok(cudaGetLastError());
        }
    }
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
    const bool any = T > 0 && (grad_x || grad_residual || p.dgate_row || want);
    const bool full = post_kind == RLF_NORM_LAYER || pre_kind == RLF_NORM_LAYER || (want & 10) || (p.b1 && p.dgate_row);
    const void* const at[] = {pre ? h : grad_h, grad_h, pre ? grad_y : nullptr, grad_x, grad_residual};
    bool edge, done = false;
    Cut c;
    if (any && fast_form(bf16, T, D, at, 5, x, x_stride, &p, &edge) &&
        pick_cut(bf16, edge, p.x_shift, false, full, T, D, p.x_shift ? 3 : 4, &c)) {
        const BlockKernel k = kernel_of<false>(bf16, full, edge, c);
        const int resident = k ? resident_ctas((const void*)k, c) : 0;
        if (resident > 0) {
            long long grid = batches(T, c, p.period), most = max_parts(T, D);
            if (most > resident) most = resident;
            if (grid > most) grid = most / p.period * p.period;
            parts = (int)grid;
            p.part = part;
            p.part_stride = part_stride(parts, D);
            k<<<(unsigned)grid, c.threads, c.smem, s>>>(p);
            count_launch();
            if (cudaGetLastError() != cudaSuccess) return RLF_ERR_CUDA;
            done = true;
        }
    }
    if (any && !done) {
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
    // CTAs for a column block: while a warp has more than one batch of loads and the GPU has room for them
    f.split = 1;
    while (f.split < 8 && parts > 32 * 8 * f.split && (D + 31) / 32 * 2 * f.split * 2 <= 296) f.split *= 2;
    return launch_finish(f, s);
}
