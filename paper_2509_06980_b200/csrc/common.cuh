// Shared host/device helpers of the CUDA library (status codes, launch accounting, small
// device utilities).  Nothing here is used by, or shared with, the CPU oracle.
#pragma once
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <stdint.h>

#include <mutex>

#include "../../include/rlf.h"

namespace rlf {

// counts kernels launched by this library (host side, relaxed)
void count_launch(int n = 1);

// RLF_OK iff the current device is compute capability 10.x
rlf_status check_arch();

// token-record and scalar-loss stages (logits_loss.cu), also used by the fused LM-head path
rlf_status launch_token_prep(const int32_t* ids, const int32_t* seq_id, const float* adv, const float* old_logp,
                             const float* ref_logp, const uint8_t* mask, int64_t T, int32_t V, int32_t B,
                             void* rec, long long* n_count_or_null, int32_t* dev_status, cudaStream_t s);
rlf_status launch_token_loss(const float* logp, const void* rec, int64_t T, float eps_clip, float beta,
                             double* partial, const long long* denom, double* loss_out, cudaStream_t s);
size_t token_loss_partial_bytes();
// the same with an asymmetric clip range and optional per-token weights (weighted sums are already means)
rlf_status launch_token_loss_w(const float* logp, const void* rec, int64_t T, float eps_lo, float eps_hi, float beta,
                               const float* wtok, double* partial, const long long* denom, double* loss_out,
                               cudaStream_t s);
// sequence-mean aggregation: wtok[t] = live_t / (n_b * S); cnt [B] ints and s_slot [1] are scratch
rlf_status launch_seq_weights(const void* rec, const int32_t* seq_id, int64_t T, int32_t B,
                              const long long* denom_or_null, int* cnt, long long* s_slot, float* wtok,
                              cudaStream_t s);

// cross-entropy stages (cross_entropy.cu), also used by the fused LM-head form: the work list (int2 {row, target id} of
// the live rows in order, then {row, -1} of the others, last row first), the loss scalars from per-token terms
// {-logp, smooth, lse, counts} (float4), argument check.  The plan also zeroes zero_words (at most 1024) words at `zero`.
rlf_status ce_launch_plan(const int32_t* ids, const uint8_t* mask, int64_t T, int32_t V, void* list, int* n_live,
                          long long* n_mask, int* zero, int zero_words, int32_t* dev_status, cudaStream_t s);
rlf_status ce_launch_loss(const void* terms, int64_t T, const long long* denom, float eps, float zeta, double* loss_out,
                          cudaStream_t s);
rlf_status ce_check_objective(float label_smoothing, float z_coef);

inline rlf_status cuda_ok(cudaError_t e) { return e == cudaSuccess ? RLF_OK : RLF_ERR_CUDA; }

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// What fits on a device at once, remembered per (device, kernel, launch shape); a shape beyond the table's size replaces the
// oldest.  Nothing here allocates, so nothing can throw through a C entry.
struct ResidentTable {
    struct Entry { int dev; const void* kernel; int a, b, n; };
    std::mutex mu;
    Entry entry[256];
    int count = 0;
    template <typename Ask> int get(const void* kernel, int a, int b, Ask ask) {
        int dev = 0;
        cudaGetDevice(&dev);
        std::lock_guard<std::mutex> lock(mu);
        const int have = count < 256 ? count : 256;
        for (int i = 0; i < have; ++i) {
            const Entry& e = entry[i];
            if (e.dev == dev && e.kernel == kernel && e.a == a && e.b == b) return e.n;
        }
        const int n = ask(dev);
        entry[count & 255] = {dev, kernel, a, b, n};
        count = count == 511 ? 256 : count + 1;
        return n;
    }
};

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Exponents formed as one multiply-add from a rounded offset, x log2 e - (m log2 e rounded), all lack the same r = (m log2 e rounded) -
// m log2 e, which is known exactly: the exponentials, and their sums, are put right by the factor 2^r = 1 + r ln 2 (|r| <= 2^-13 up
// to |m| = 2048, so that the next term is below 2^-27).  Returns r ln 2.
__device__ __forceinline__ float offset_error(float m) {
    return fmaf(-m, kLog2e, __fmul_rn(m, kLog2e)) * kLn2;
}

__device__ __forceinline__ float ex2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float lg2_approx(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Pairs of fp32 values in one register pair: one instruction for two additions, products or multiply-adds (at one each the
// norms and the forward-only cross entropy are bound by instruction issue before HBM).
typedef unsigned long long f2;
__device__ __forceinline__ f2 f2_make(float lo, float hi) {
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void f2_split(f2 v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ f2 f2_add(f2 a, f2 b) {
    f2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 f2_mul(f2 a, f2 b) {
    f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 f2_fma(f2 a, f2 b, f2 c) {
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float f2_sum(f2 v) {
    float a, b;
    f2_split(v, a, b);
    return a + b;
}

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

}  // namespace rlf
