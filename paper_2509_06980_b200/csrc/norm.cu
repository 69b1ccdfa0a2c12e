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
#include "norm_rows.cuh"

namespace rlf {
namespace nm {

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
    int period;                 // edge form: rows t and t + period sit alike in their 16-byte vectors
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
    int period;                 // as in FwdParams
};

constexpr int kGenThreads = 256;

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

// partial rows -> gradient, added in a fixed order (results are run-to-run identical).  A CTA covers 32 columns; warp w
// adds the partials w, w + 32, ... and the 32 sums are added in order.  It may be set up while the kernel before it
// still runs (programmatic dependent launch) and waits for that kernel's results here.
__global__ void __launch_bounds__(1024)
norm_dw_reduce_kernel(const float* __restrict__ part, const float* __restrict__ part_b, int parts, int D, int accumulate,
                      float* __restrict__ dw, float* __restrict__ db) {
    __shared__ float acc[32][33];
    const float* src = blockIdx.y == 0 ? part : part_b;
    float* dst = blockIdx.y == 0 ? dw : db;
    if (dst == nullptr) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + lane;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    float s = 0.0f;
    if (col < D) {
#pragma unroll 4
        for (int k = warp; k < parts; k += 32) s += src[(long long)k * D + col];
    }
    acc[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && col < D) {
        for (int w = 1; w < 32; ++w) s += acc[w][lane];
        dst[col] = accumulate ? dst[col] + s : s;
    }
}

// ---- fast forms -----------------------------------------------------------------------------
// A CTA works on R rows at a time, with the next R rows on their way into the other half of a shared-memory buffer
// (cp.async), so that HBM is kept busy through the sums' exchanges; the rows stay in shared memory between the pass that
// sums and the pass that writes.  One exchange (one barrier) serves the R rows' sums.
//   wide    every row starts on 16 bytes and the width fills its 16-byte vectors: a thread owns NV vectors of each row, copies
//           them itself and reads back only those; its columns' weights and weight gradients live in registers;
//   edge    (wide kernels with EDGE) rows on no boundary, all tensors' rows alike: with a stride that is no multiple of a vector
//           the row's place in its vectors repeats after 2, 4 or 8 rows, so a CTA takes every 2nd, 4th or 8th row and its
//           threads keep fixed columns all the same; only a row's first and last vector are masked and stored by element.  Forward
//           (backward) of 20000 x 2603 bf16, layer form with residual: 114 us (125), the staged form 151 (198); 4999 x 1021
//           fp32: 17 (23), staged 23 (29);
//   staged  any width, stride and base: a row is copied as the aligned 16-byte chunks that cover it, by whichever thread, and a
//           thread owns every blockDim-th column; weights and weight gradients live in shared memory.
constexpr int kShortRow = 96;                    // vectors of a row that the backward takes four rows at a time, a thread each
constexpr int kSmemLimit = 200 * 1024;           // most dynamic shared memory that a fast form asks for

// Forward.  The rows' elements (x + residual) are held unpacked in registers through the passes.
// fp32 rows, two vectors and two rows per thread: asking for three CTAs of 256 threads per SM keeps the compiler at 68 registers
// (32768 x 1024 layer form 49.7 -> 45.7 us, 4999 x 1021 19.1 -> 17.6); the bf16 form would spill (124 -> 136 us at 32768 x 4096).
// 0 asks for nothing; even 1 changes the bf16 code for the worse (32768 x 2560 RMS 58 -> 66 us).
template <typename T, int NV, int R, bool LAYER, bool EDGE>
__global__ void __launch_bounds__(sizeof(T) == 4 && R == 2 ? 256 : kMaxThreads, sizeof(T) == 4 && R == 2 && NV == 2 ? 3 : 0)
norm_fwd_wide_kernel(const FwdParams p) {
    using V = Vec<T>;
    constexpr int P = V::P, N = V::N;
    extern __shared__ __align__(16) uint4 stage[];      // [2][R][arrays][NV][blockDim], a slot is its thread's own
    __shared__ __align__(16) float red[2 * (kMaxThreads / 32) * R];
    int turn = 0;
    const int th = blockDim.x, tid = threadIdx.x;
    const int arrays = p.res ? 2 : 1;
    const Rows<T, EDGE> rows(p.x, p.x_stride, p.T, p.D, p.period, R);
    const int nvec = rows.nvec;
    const float inv_d = 1.0f / (float)p.D;
    auto slot = [&](int buf, int k, int a, int i) -> uint4* { return stage + (((buf * R + k) * arrays + a) * NV + i) * th + tid; };
    unsigned keep[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) keep[i] = EDGE ? rows.bits(tid + i * th, p.D) : (1u << N) - 1u;
    auto masked = [&](int i) { return EDGE && keep[i] != (1u << N) - 1u; };
    auto fetch = [&](long long j0, int buf) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const long long t = rows.row(j0 + k);
            if (j0 + k < rows.n) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int c = tid + i * th;
                    if (c < nvec) {
                        rows.copy(slot(buf, k, 0, i), static_cast<const T*>(p.x) + t * p.x_stride, c, p.D, t == 0);
                        if (p.res) rows.copy(slot(buf, k, 1, i), static_cast<const T*>(p.res) + t * p.x_stride, c, p.D, t == 0);
                    }
                }
            }
        }
        cp_async_commit();
    };
    long long j0 = rows.first;
    fetch(j0, 0);
    f2 w[NV][P], b[LAYER ? NV : 1][P];                  // (the RMS form's bias, rare, is fetched where it is used)
    load_w<P, NV>(p.w, p.w_bf16, p.D, rows.lead, w);
    if constexpr (LAYER) load_w<P, NV>(p.b, p.w_bf16, p.D, rows.lead, b);
    for (int buf = 0; j0 < rows.n; j0 += rows.step, buf ^= 1) {
        fetch(j0 + rows.step, buf ^ 1);
        cp_async_wait1();
        f2 h[R][NV][P];
        float s[R], mu[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            f2 q = 0ull;
            mu[k] = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (tid + i * th < nvec) {
                    V::unpack(*slot(buf, k, 0, i), h[k][i]);
                    if (p.res) {
                        f2 z[P];
                        V::unpack(*slot(buf, k, 1, i), z);
#pragma unroll
                        for (int e = 0; e < P; ++e) h[k][i][e] = f2_add(h[k][i][e], z[e]);
                    }
                    if (masked(i)) mask_pairs<P>(h[k][i], keep[i]);
#pragma unroll
                    for (int e = 0; e < P; ++e) q = LAYER ? f2_add(q, h[k][i][e]) : f2_fma(h[k][i][e], h[k][i][e], q);
                }
            s[k] = f2_sum(q);
        }
        cta_sums<R>(s, red, turn);
        if (LAYER) {
#pragma unroll
            for (int k = 0; k < R; ++k) {
                mu[k] = s[k] * inv_d;
                const f2 m2 = f2_make(-mu[k], -mu[k]);
                f2 q = 0ull;
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (tid + i * th < nvec) {
                        f2 d[P];
#pragma unroll
                        for (int e = 0; e < P; ++e) d[e] = f2_add(h[k][i][e], m2);
                        if (masked(i)) mask_pairs<P>(d, keep[i]);
#pragma unroll
                        for (int e = 0; e < P; ++e) q = f2_fma(d[e], d[e], q);
                    }
                s[k] = f2_sum(q);
            }
            cta_sums<R>(s, red, turn);
        }
#pragma unroll
        for (int k = 0; k < R; ++k) {
            if (j0 + k >= rows.n) continue;
            const long long t = rows.row(j0 + k);
            const float r = rsqrtf(s[k] * inv_d + p.eps);
            const f2 r2 = f2_make(r, r), m2 = f2_make(-mu[k], -mu[k]);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = tid + i * th;
                if (c >= nvec) continue;
                f2 o[P];
                if (p.sum) rows.store(static_cast<T*>(p.sum) + t * p.D, c, V::pack(h[k][i]), keep[i]);
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    o[e] = f2_mul(f2_mul(LAYER ? f2_add(h[k][i][e], m2) : h[k][i][e], r2), w[i][e]);
                    if (LAYER) o[e] = f2_add(o[e], b[LAYER ? i : 0][e]);
                    else if (p.b) o[e] = f2_add(o[e], f2_make(ld_w_in(p.b, p.w_bf16, p.D, c * N + 2 * e - rows.lead), ld_w_in(p.b, p.w_bf16, p.D, c * N + 2 * e + 1 - rows.lead)));
                }
                rows.store(static_cast<T*>(p.y) + t * p.D, c, V::pack(o), keep[i]);
            }
            if (tid == 0) {
                if (p.mean) p.mean[t] = mu[k];
                if (p.rstd) p.rstd[t] = r;
            }
        }
    }
    cp_async_wait0();
}

// Backward: a CTA owns the row.  One sum per row, mean(g xh), and with FULL (layer form, or a bias gradient asked for) also
// mean(g) and the bias gradient; a CTA's weight gradients are added up row after row and leave as one partial row per CTA.
// Short rows (four at a time) are compiled for CTAs of up to kShortRow threads, six or more per SM: left at 512 threads the
// compiler chose 50 - 64 registers and overlapped the four rows less (65536 x 512 bf16 RMS 50 -> 42 us, layer form 54 -> 51).
template <typename T, int NV, int R, bool FULL, bool EDGE>
__global__ void __launch_bounds__(R == 4 ? kShortRow : kMaxThreads, R == 4 ? 6 : 0)
norm_bwd_wide_kernel(const BwdParams p) {
    using V = Vec<T>;
    constexpr int P = V::P, N = V::N, K = FULL ? 2 * R : R;
    extern __shared__ __align__(16) uint4 stage[];      // [2][R][dy, x (, skip)][NV][blockDim]
    __shared__ __align__(16) float red[2 * (kMaxThreads / 32) * K];
    int turn = 0;
    const int th = blockDim.x, tid = threadIdx.x;
    const int arrays = p.skip ? 3 : 2;
    const Rows<T, EDGE> rows(p.x, p.x_stride, p.T, p.D, p.period, R);
    const int nvec = rows.nvec;
    const float inv_d = 1.0f / (float)p.D;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    auto slot = [&](int buf, int k, int a, int i) -> uint4* { return stage + (((buf * R + k) * arrays + a) * NV + i) * th + tid; };
    float mu_next[R], r_next[R];
    unsigned keep[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) keep[i] = EDGE ? rows.bits(tid + i * th, p.D) : (1u << N) - 1u;
    auto masked = [&](int i) { return EDGE && keep[i] != (1u << N) - 1u; };
    auto fetch = [&](long long j0, int buf) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const long long t = rows.row(j0 + k);
            mu_next[k] = r_next[k] = 0.0f;
            if (j0 + k < rows.n) {
                if (FULL && p.layer) mu_next[k] = p.mean[t];
                r_next[k] = p.rstd[t];
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int c = tid + i * th;
                    if (c < nvec) {
                        rows.copy(slot(buf, k, 0, i), static_cast<const T*>(p.dy) + t * p.dy_stride, c, p.D, t == 0);
                        rows.copy(slot(buf, k, 1, i), static_cast<const T*>(p.x) + t * p.x_stride, c, p.D, t == 0);
                        if (p.skip) rows.copy(slot(buf, k, 2, i), static_cast<const T*>(p.skip) + t * p.D, c, p.D, t == 0);
                    }
                }
            }
        }
        cp_async_commit();
    };
    long long j0 = rows.first;
    fetch(j0, 0);
    f2 w[NV][P], dw[NV][P], db[FULL ? NV : 1][P];
    load_w<P, NV>(p.w, p.w_bf16, p.D, rows.lead, w);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < P; ++e) {
            dw[i][e] = 0ull;
            if (FULL) db[FULL ? i : 0][e] = 0ull;
        }
    for (int buf = 0; j0 < rows.n; j0 += rows.step, buf ^= 1) {
        float mu[R], r[R], s[K];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            mu[k] = mu_next[k];
            r[k] = r_next[k];
        }
        fetch(j0 + rows.step, buf ^ 1);
        cp_async_wait1();
#pragma unroll
        for (int k = 0; k < R; ++k) {
            f2 a = 0ull, b = 0ull;
            if (j0 + k < rows.n) {
                const f2 m2 = f2_make(-mu[k], -mu[k]), r2 = f2_make(r[k], r[k]);
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (tid + i * th < nvec) {
                        f2 x[P], dy[P];
                        V::unpack(*slot(buf, k, 0, i), dy);
                        V::unpack(*slot(buf, k, 1, i), x);
                        if (masked(i)) {
                            mask_pairs<P>(dy, keep[i]);
                            mask_pairs<P>(x, keep[i]);
                        }
#pragma unroll
                        for (int e = 0; e < P; ++e) {
                            const f2 xh = f2_mul(FULL ? f2_add(x[e], m2) : x[e], r2), q = f2_mul(dy[e], xh);
                            a = f2_fma(q, w[i][e], a);
                            dw[i][e] = f2_add(dw[i][e], q);
                            if (FULL) {
                                b = f2_fma(dy[e], w[i][e], b);
                                db[FULL ? i : 0][e] = f2_add(db[FULL ? i : 0][e], dy[e]);
                            }
                        }
                    }
            }
            s[k] = f2_sum(a);
            if (FULL) s[FULL ? R + k : 0] = f2_sum(b);
        }
        if (p.dx == nullptr) continue;
        cta_sums<K>(s, red, turn);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            if (j0 + k >= rows.n) continue;
            const long long t = rows.row(j0 + k);
            // r (g - b - (x - mu) r a) = r g + x (- r^2 a) + (mu r^2 a - r b)
            const float a = s[k] * inv_d * r[k] * r[k];
            const float b = (FULL && p.layer) ? r[k] * (s[FULL ? R + k : 0] * inv_d) : 0.0f;
            const f2 r2 = f2_make(r[k], r[k]), a2 = f2_make(-a, -a), b2 = f2_make(-b, -b), m2 = f2_make(-mu[k], -mu[k]);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = tid + i * th;
                if (c >= nvec) continue;
                f2 x[P], dy[P], o[P];
                V::unpack(*slot(buf, k, 0, i), dy);
                V::unpack(*slot(buf, k, 1, i), x);
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    o[e] = f2_mul(f2_mul(dy[e], w[i][e]), r2);
                    if (FULL) o[e] = f2_add(o[e], b2);
                    o[e] = f2_fma(FULL ? f2_add(x[e], m2) : x[e], a2, o[e]);
                }
                if (p.skip) {
                    f2 q[P];
                    V::unpack(*slot(buf, k, 2, i), q);
#pragma unroll
                    for (int e = 0; e < P; ++e) o[e] = f2_add(o[e], q[e]);
                }
                rows.store(static_cast<T*>(p.dx) + t * p.D, c, V::pack(o), keep[i]);
            }
        }
    }
    cp_async_wait0();
    auto leave = [&](float* part, const f2 (&g)[P], int i) {
        const int c = (tid + i * th) * N;
        if (part == nullptr || tid + i * th >= nvec) return;
        if constexpr (EDGE) {
            float* d = part + (long long)blockIdx.x * p.D - rows.lead + c;
#pragma unroll
            for (int e = 0; e < P; ++e) {
                float lo, hi;
                f2_split(g[e], lo, hi);
                if ((keep[i] >> (2 * e)) & 1u) d[2 * e] = lo;
                if ((keep[i] >> (2 * e + 1)) & 1u) d[2 * e + 1] = hi;
            }
            return;
        }
        ulonglong2* d = reinterpret_cast<ulonglong2*>(part + (long long)blockIdx.x * p.D + c);
#pragma unroll
        for (int e = 0; e < P; e += 2) d[e / 2] = make_ulonglong2(g[e], g[e + 1]);
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        leave(p.part, dw[i], i);
        if (FULL) leave(p.part_b, db[FULL ? i : 0], i);
    }
}

template <typename T, int R, bool LAYER>
__global__ void __launch_bounds__(kMaxThreads)
norm_fwd_staged_kernel(const FwdParams p) {
    extern __shared__ __align__(16) char smem[];        // [2][R][arrays] rows, then the weights (and biases) in fp32
    __shared__ __align__(16) float red[2 * (kMaxThreads / 32) * R];
    int turn = 0;
    const int th = blockDim.x, tid = threadIdx.x, D = p.D;
    const int arrays = p.res ? 2 : 1, pitch = staged_pitch(D, (int)sizeof(T));
    const float inv_d = 1.0f / (float)D;
    float* w_s = reinterpret_cast<float*>(smem + 2 * R * arrays * pitch);
    float* b_s = w_s + D;
    auto at = [&](int buf, int k, int a) -> char* { return smem + ((buf * R + k) * arrays + a) * pitch; };
    auto fetch = [&](long long t0, int buf) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const long long t = t0 + k;
            if (t < p.T) {
                copy_row(at(buf, k, 0), static_cast<const T*>(p.x) + t * p.x_stride, D, t == 0);
                if (p.res) copy_row(at(buf, k, 1), static_cast<const T*>(p.res) + t * p.x_stride, D, t == 0);
            }
        }
        cp_async_commit();
    };
    const long long step = (long long)gridDim.x * R;
    long long t0 = (long long)blockIdx.x * R;
    fetch(t0, 0);
    for (int c = tid; c < D; c += th) {
        w_s[c] = ld_w(p.w, p.w_bf16, c);
        if (p.b) b_s[c] = ld_w(p.b, p.w_bf16, c);
    }
    for (int buf = 0; t0 < p.T; t0 += step, buf ^= 1) {
        __syncthreads();                                // the other half has been read by everyone
        fetch(t0 + step, buf ^ 1);
        cp_async_wait1();
        __syncthreads();                                // everyone's chunks of this half are here
        const T* x[R];
        const T* res[R];
        float s[R], mu[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const long long t = min(t0 + k, p.T - 1);
            x[k] = reinterpret_cast<const T*>(at(buf, k, 0) + chunk_head(static_cast<const T*>(p.x) + t * p.x_stride));
            res[k] = p.res ? reinterpret_cast<const T*>(at(buf, k, 1) + chunk_head(static_cast<const T*>(p.res) + t * p.x_stride)) : x[k];
            s[k] = mu[k] = 0.0f;
        }
        auto h = [&](int k, int c) -> float { return to_f<T>(x[k][c]) + (p.res ? to_f<T>(res[k][c]) : 0.0f); };
#pragma unroll 2
        for (int c = tid; c < D; c += th)
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const float v = h(k, c);
                s[k] = LAYER ? s[k] + v : fmaf(v, v, s[k]);
            }
        cta_sums<R>(s, red, turn);
        if (LAYER) {
#pragma unroll
            for (int k = 0; k < R; ++k) {
                mu[k] = s[k] * inv_d;
                s[k] = 0.0f;
            }
#pragma unroll 2
            for (int c = tid; c < D; c += th)
#pragma unroll
                for (int k = 0; k < R; ++k) {
                    const float v = h(k, c) - mu[k];
                    s[k] = fmaf(v, v, s[k]);
                }
            cta_sums<R>(s, red, turn);
        }
        float r[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            r[k] = rsqrtf(s[k] * inv_d + p.eps);
            if (tid == 0 && t0 + k < p.T) {
                if (p.mean) p.mean[t0 + k] = mu[k];
                if (p.rstd) p.rstd[t0 + k] = r[k];
            }
        }
#pragma unroll 2
        for (int c = tid; c < D; c += th) {
            const float wc = w_s[c], bc = p.b ? b_s[c] : 0.0f;
#pragma unroll
            for (int k = 0; k < R; ++k) {
                if (t0 + k >= p.T) continue;
                const float v = h(k, c);
                if (p.sum) static_cast<T*>(p.sum)[(t0 + k) * D + c] = from_f<T>(v);
                static_cast<T*>(p.y)[(t0 + k) * D + c] = from_f<T>((v - mu[k]) * r[k] * wc + bc);
            }
        }
    }
    cp_async_wait0();
}

template <typename T, int R, bool FULL>
__global__ void __launch_bounds__(kMaxThreads)
norm_bwd_staged_kernel(const BwdParams p) {
    extern __shared__ __align__(16) char smem[];        // [2][R][dy, x (, skip)] rows, then w, dw (and db) in fp32
    __shared__ __align__(16) float red[2 * (kMaxThreads / 32) * 2 * R];
    int turn = 0;
    const int th = blockDim.x, tid = threadIdx.x, D = p.D;
    const int arrays = p.skip ? 3 : 2, pitch = staged_pitch(D, (int)sizeof(T));
    const float inv_d = 1.0f / (float)D;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    float* w_s = reinterpret_cast<float*>(smem + 2 * R * arrays * pitch);
    float* dw_s = w_s + D;
    float* db_s = dw_s + D;
    auto at = [&](int buf, int k, int a) -> char* { return smem + ((buf * R + k) * arrays + a) * pitch; };
    auto fetch = [&](long long t0, int buf) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const long long t = t0 + k;
            if (t < p.T) {
                copy_row(at(buf, k, 0), static_cast<const T*>(p.dy) + t * p.dy_stride, D, t == 0);
                copy_row(at(buf, k, 1), static_cast<const T*>(p.x) + t * p.x_stride, D, t == 0);
                if (p.skip) copy_row(at(buf, k, 2), static_cast<const T*>(p.skip) + t * D, D, t == 0);
            }
        }
        cp_async_commit();
    };
    const long long step = (long long)gridDim.x * R;
    long long t0 = (long long)blockIdx.x * R;
    fetch(t0, 0);
    for (int c = tid; c < D; c += th) {
        w_s[c] = ld_w(p.w, p.w_bf16, c);
        dw_s[c] = 0.0f;
        if (FULL && p.part_b) db_s[c] = 0.0f;
    }
    for (int buf = 0; t0 < p.T; t0 += step, buf ^= 1) {
        __syncthreads();
        fetch(t0 + step, buf ^ 1);
        const T* dy[R];
        const T* x[R];
        const T* skip[R];
        float mu[R], r[R], s[2 * R];
        bool row[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            row[k] = t0 + k < p.T;
            const long long t = min(t0 + k, p.T - 1);
            dy[k] = reinterpret_cast<const T*>(at(buf, k, 0) + chunk_head(static_cast<const T*>(p.dy) + t * p.dy_stride));
            x[k] = reinterpret_cast<const T*>(at(buf, k, 1) + chunk_head(static_cast<const T*>(p.x) + t * p.x_stride));
            skip[k] = p.skip ? reinterpret_cast<const T*>(at(buf, k, 2) + chunk_head(static_cast<const T*>(p.skip) + t * D)) : x[k];
            mu[k] = p.layer ? p.mean[t] : 0.0f;
            r[k] = p.rstd[t];
            s[2 * k] = s[2 * k + 1] = 0.0f;
        }
        cp_async_wait1();
        __syncthreads();
#pragma unroll 2
        for (int c = tid; c < D; c += th) {
            const float wc = w_s[c];
            float qs = 0.0f, ds = 0.0f;
#pragma unroll
            for (int k = 0; k < R; ++k) {
                if (!row[k]) continue;
                const float d = to_f<T>(dy[k][c]), q = d * ((to_f<T>(x[k][c]) - mu[k]) * r[k]);
                s[2 * k] = fmaf(q, wc, s[2 * k]);
                if (FULL) s[2 * k + 1] = fmaf(d, wc, s[2 * k + 1]);
                qs += q;
                ds += d;
            }
            dw_s[c] += qs;
            if (FULL && p.part_b) db_s[c] += ds;
        }
        if (p.dx == nullptr) continue;
        cta_sums<2 * R>(s, red, turn);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            s[2 * k] *= inv_d;
            s[2 * k + 1] = p.layer ? s[2 * k + 1] * inv_d : 0.0f;
        }
#pragma unroll 2
        for (int c = tid; c < D; c += th) {
            const float wc = w_s[c];
#pragma unroll
            for (int k = 0; k < R; ++k) {
                if (!row[k]) continue;
                float o = r[k] * (fmaf(to_f<T>(dy[k][c]), wc, -s[2 * k + 1]) - (to_f<T>(x[k][c]) - mu[k]) * r[k] * s[2 * k]);
                if (p.skip) o += to_f<T>(skip[k][c]);
                static_cast<T*>(p.dx)[(t0 + k) * D + c] = from_f<T>(o);
            }
        }
    }
    cp_async_wait0();
    for (int c = tid; c < D; c += th) {                 // (a thread's own columns)
        if (p.part) p.part[(long long)blockIdx.x * D + c] = dw_s[c];
        if (FULL && p.part_b) p.part_b[(long long)blockIdx.x * D + c] = db_s[c];
    }
}

// ---- host side --------------------------------------------------------------------------------
// Most partial rows of a weight gradient (sizes the workspace): enough for one per resident CTA.
static long long max_parts(long long T, int D) {
    long long n = (1ll << 21) / D;
    if (n < 1024) n = 1024;
    if (n > 4096) n = 4096;
    if (n > T) n = T;
    return n < 1 ? 1 : n;
}

// floats from one gradient's partial rows to the other's (keeps 16-byte alignment)
static size_t part_stride(int parts, int D) { return ((size_t)parts * (size_t)D + 63) & ~(size_t)63; }

// how rows are cut: wide (nv vectors per thread) or staged, `threads` threads, `rows` rows at a time, bytes of shared memory
struct Cut { Form form; int nv, threads, rows, smem; };

// false: no fast form holds the rows (the general kernels do: rows beyond 512 threads x 4 vectors, or that do not fit shared
// memory when staged; and rows shorter than a vector, several of which may start in the vector that their tensor starts in: a
// test for them in the copies costs the others 3 - 8 %, 20000 x 2603 bf16 with a stride of 2606 142 -> 152 us).  `arrays` rows are read per row; the staged form keeps `vectors` fp32 vectors of the width.
//   Forward: CTAs of up to 256 threads, two rows at a time.  32768 x 2560 bf16, no residual: 58.7 us with 256 threads and two
//   rows, 63.7 with one row, 66 with 512 threads; with the residual 106 - 108 us whichever.
//   Rows of up to 256 vectors without a residual, or off their vectors: 128 threads (32768 rows, 256 threads -> 128: 2048 bf16
//   68 -> 62 us layer, 52 -> 48 RMS; 1024 fp32 layer 57 -> 50; 1531 bf16 with residual 132 -> 96); with one they cost 1 - 4 %.
//   bf16 rows of more than 512 vectors, layer form, either direction: up to 512 threads, one row at a time (16384 x 8192: 140 ->
//   130 us forward, 175 -> 167 backward; 16384 x 5120 with residual 125 -> 116, 139 -> 115).
//   Backward: bf16 rows without the second sum (RMS form, no bias) four vectors per thread, one row at a time: 32768 x 2560
//   bf16 110 us against 117 - 122 with one or two vectors; else up to 512 threads of two vectors, two rows at a time:
//   8191 x 4096 bf16 layer form 49 us against 54 with four vectors, 32768 x 2560 fp32 162 against 190.  The layer form takes
//   two vectors per thread at shorter rows too (32768 rows, one vector -> two: 2048 bf16 99 -> 81 us, 1024 bf16
//   54 -> 47, 1024 fp32 81 -> 71); rows of up to 96 vectors keep one, four rows at a time (65536 rows,
//   two rows -> four: 768 bf16 layer form 79 -> 72 us, 384 fp32 72 -> 57; 128 vectors gained nothing more and lost 12 % at 1013 bf16).
static bool pick_cut(bool bf16, Form form, bool fwd, bool layer, bool full, long long T, int D, int arrays, int vectors, Cut* c) {
    const int esz = bf16 ? 2 : 4;
    if (D > kSmemLimit / esz) return false;            // (before any product of D)
    const int v = 16 / esz, nvec = form == kEdge ? (D + 2 * v - 2) / v : D / v;
    if (D < v) return false;
    const bool wide = form != kStaged;
    c->form = form;
    c->nv = 1;
    if (wide) {
        int most = fwd ? (nvec <= 256 && (arrays == 1 || form == kEdge) ? 128 : 256) : (bf16 && !full && nvec <= 512) ? 128 : bf16 ? 256 : 512;
        if (!fwd && layer && nvec > kShortRow && nvec <= 2 * most) most = nvec <= 128 ? 64 : (nvec + 63) / 64 * 32;
        const bool long_layer = bf16 && layer && nvec > 512;
        if (long_layer) most = 512;
        while ((nvec + c->nv - 1) / c->nv > most && c->nv < 4) c->nv *= 2;
        c->threads = ((nvec + c->nv - 1) / c->nv + 31) / 32 * 32;
        if (c->threads > kMaxThreads) return false;
        c->rows = c->nv == 4 || long_layer ? 1 : (!fwd && nvec <= kShortRow) ? 4 : 2;
    } else {
        c->threads = D <= 512 ? 128 : 256;
        c->rows = 2;
    }
    // too few rows to put several on a CTA
    while (c->rows > 1 && T < 148ll * 4 * c->rows) c->rows /= 2;
    for (;; c->rows /= 2) {
        const int batch = 2 * c->rows * arrays;
        c->smem = wide ? batch * c->nv * c->threads * 16 : batch * staged_pitch(D, esz) + 4 * vectors * D;
        if (c->smem <= (c->rows > 1 ? kSmemLimit / 2 : kSmemLimit)) return true;
        if (c->rows == 1) return false;
    }
}

typedef void (*FwdKernel)(const FwdParams);
typedef void (*BwdKernel)(const BwdParams);
template <typename T, int R, bool F, bool E>
static FwdKernel fwd_wide_form(const Cut& c) {
    if (c.nv == 1) return norm_fwd_wide_kernel<T, 1, R, F, E>;
    if (c.nv == 2) return norm_fwd_wide_kernel<T, 2, R, F, E>;
    return R == 1 ? norm_fwd_wide_kernel<T, 4, 1, F, E> : nullptr;
}
template <typename T, int R, bool F>
static FwdKernel fwd_kernel_form(const Cut& c) {
    if (c.form == kStaged) return norm_fwd_staged_kernel<T, R, F>;
    return c.form == kEdge ? fwd_wide_form<T, R, F, true>(c) : fwd_wide_form<T, R, F, false>(c);
}
template <typename T, int R, bool F, bool E>
static BwdKernel bwd_wide_form(const Cut& c) {
    if (c.nv == 1) return norm_bwd_wide_kernel<T, 1, R, F, E>;
    if (R == 4) return nullptr;                  // (narrow rows only)
    if (c.nv == 2) return norm_bwd_wide_kernel<T, 2, (R < 4 ? R : 1), F, E>;
    return R == 1 ? norm_bwd_wide_kernel<T, 4, 1, F, E> : nullptr;
}
template <typename T, int R, bool F>
static BwdKernel bwd_kernel_form(const Cut& c) {
    if (c.form == kStaged) return R == 4 ? nullptr : norm_bwd_staged_kernel<T, (R < 4 ? R : 1), F>;
    return c.form == kEdge ? bwd_wide_form<T, R, F, true>(c) : bwd_wide_form<T, R, F, false>(c);
}
template <bool F>
static FwdKernel fwd_kernel(bool bf16, const Cut& c) {
    if (c.rows == 1) return bf16 ? fwd_kernel_form<__nv_bfloat16, 1, F>(c) : fwd_kernel_form<float, 1, F>(c);
    return bf16 ? fwd_kernel_form<__nv_bfloat16, 2, F>(c) : fwd_kernel_form<float, 2, F>(c);
}
template <bool F>
static BwdKernel bwd_kernel(bool bf16, const Cut& c) {
    if (c.rows == 1) return bf16 ? bwd_kernel_form<__nv_bfloat16, 1, F>(c) : bwd_kernel_form<float, 1, F>(c);
    if (c.rows == 2) return bf16 ? bwd_kernel_form<__nv_bfloat16, 2, F>(c) : bwd_kernel_form<float, 2, F>(c);
    return bf16 ? bwd_kernel_form<__nv_bfloat16, 4, F>(c) : bwd_kernel_form<float, 4, F>(c);
}

// CTAs of this kernel that are resident at once (0: none fits); cached per device, kernel, width and shared memory, and opts
// the kernel in to its shared memory on the way
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

static rlf_status launch_reduce(const float* part, const float* part_b, int parts, int D, int accumulate, float* dw, float* db,
                                cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    cfg.gridDim = dim3((unsigned)((D + 31) / 32), db ? 2 : 1);
    cfg.blockDim = dim3(1024);
    cfg.stream = s;
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, norm_dw_reduce_kernel, part, part_b, parts, D, accumulate, dw, db) != cudaSuccess) {
        cudaGetLastError();
        return RLF_ERR_CUDA;
    }
    count_launch();
    return RLF_OK;
}

// CTAs that give each one batch: whole multiples of the period in the edge form
static long long batches(long long T, const Cut& c, int period) {
    if (c.form != kEdge) return (T + c.rows - 1) / c.rows;
    const long long rows = (T + period - 1) / period;
    return (rows + c.rows - 1) / c.rows * period;
}

static int row_grid(long long T) { return (int)(T < 148 * 8 ? T : 148 * 8); }

static rlf_status check_norm(int64_t T, int32_t D, rlf_dtype dt, rlf_dtype w_dt, int kind) {
    if ((dt != RLF_BF16 && dt != RLF_F32) || (w_dt != RLF_BF16 && w_dt != RLF_F32)) return RLF_ERR_DTYPE;
    if (T < 0 || D < 1) return RLF_ERR_SHAPE;
    if (D >= (1 << 30)) return RLF_ERR_UNSUPPORTED;    // the kernels count columns in 32 bits
    if (kind != RLF_NORM_LAYER && kind != RLF_NORM_RMS) return RLF_ERR_UNSUPPORTED;
    return RLF_OK;
}

}  // namespace nm

size_t norm_bwd_workspace_bytes(int64_t T, int32_t D) {
    if (D < 1) return 0;
    return 2 * nm::part_stride((int)nm::max_parts(T, D), D) * sizeof(float);
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
    const bool bf16 = dt == RLF_BF16;
    const void* const at[] = {x, residual, sum_out, y_out};
    const Form form = row_form(bf16, T, D, at, 4, x_stride, x_stride, &p.period);
    Cut c;
    auto cut = [&](Form f) { return pick_cut(bf16, f, true, p.layer, p.layer, T, D, residual ? 2 : 1, bias ? 2 : 1, &c); };
    if (cut(form) || (form == kEdge && cut(kStaged))) {
        const FwdKernel k = p.layer ? fwd_kernel<true>(bf16, c) : fwd_kernel<false>(bf16, c);
        const int resident = k ? resident_ctas((const void*)k, c) : 0;
        if (resident > 0) {
            // CTAs that retire after a quarter of a resident generation's rows: in step for the whole launch, all of them
            // load, then all store (32768 x 2560 bf16 with residual: 130 us as one generation, 109 as four)
            long long grid = batches(T, c, p.period);
            if (grid > 4ll * resident) grid = 4ll * resident / p.period * p.period;
            k<<<(unsigned)grid, c.threads, c.smem, s>>>(p);
            count_launch();
            return cuda_ok(cudaGetLastError());
        }
    }
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
    // with no rows the weight gradient is zero (or what was accumulated before)
    int parts = 0;
    float* part = static_cast<float*>(workspace);
    if (T > 0) {
        const bool bf16 = dt == RLF_BF16;
        const void* const at[] = {x, grad_y, grad_skip, grad_x};
        const Form form = row_form(bf16, T, D, at, 4, x_stride, grad_y_stride, &p.period);
        const bool full = layer || grad_bias;
        Cut c;
        BwdKernel k = nullptr;
        long long resident = 0;
        auto cut = [&](Form f) { return pick_cut(bf16, f, false, layer, full, T, D, grad_skip ? 3 : 2, grad_bias ? 3 : 2, &c); };
        if (cut(form) || (form == kEdge && cut(kStaged))) {
            k = full ? bwd_kernel<true>(bf16, c) : bwd_kernel<false>(bf16, c);
            resident = k ? resident_ctas((const void*)k, c) : 0;
        }
        if (resident > 0) {
            long long grid = batches(T, c, p.period), most = max_parts(T, D);
            if (most > resident) most = resident;        // (more CTAs would mean more partial rows: 110 -> 117 us at twice as many)
            if (grid > most) grid = c.form == kEdge ? most / p.period * p.period : most;
            parts = (int)grid;
            p.part = grad_weight ? part : nullptr;
            p.part_b = grad_bias ? part + part_stride(parts, D) : nullptr;
            if (grad_x || want_w) {
                k<<<(unsigned)grid, c.threads, c.smem, s>>>(p);
                count_launch();
            }
        } else {
            if (want_w) {
                const long long rows = T < 1024 ? 1 : (T + 127) / 128;       // per slice: at most 128 slices of a long batch
                parts = (int)((T + rows - 1) / rows);
                p.part = grad_weight ? part : nullptr;
                p.part_b = grad_bias ? part + part_stride(parts, D) : nullptr;
                const dim3 grid((unsigned)((D + 31) / 32), (unsigned)parts);
                if (bf16) norm_dw_general_kernel<__nv_bfloat16><<<grid, 256, 0, s>>>(p, rows);
                else norm_dw_general_kernel<float><<<grid, 256, 0, s>>>(p, rows);
                count_launch();
                if (cudaGetLastError() != cudaSuccess) return RLF_ERR_CUDA;
            }
            // last: grad_x may be the buffer of x or grad_y
            if (grad_x) {
                if (bf16) norm_bwd_general_kernel<__nv_bfloat16><<<row_grid(T), kGenThreads, 0, s>>>(p);
                else norm_bwd_general_kernel<float><<<row_grid(T), kGenThreads, 0, s>>>(p);
                count_launch();
            }
        }
        if (cudaGetLastError() != cudaSuccess) return RLF_ERR_CUDA;
    }
    if (!want_w) return RLF_OK;
    return launch_reduce(part, part + part_stride(parts, D), parts, D, accumulate, grad_weight, grad_bias, s);
}
