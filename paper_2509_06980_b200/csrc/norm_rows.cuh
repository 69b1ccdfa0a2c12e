// Device helpers of the kernels that own whole rows of activations (the norms): 16-byte vectors of either type as pairs of
// fp32, sums over a CTA, rows of any width, stride and alignment on their way into shared memory and back.
#pragma once
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

constexpr int kMaxThreads = 512;
__device__ __forceinline__ void cp_async16(uint32_t smem_dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(smem_dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async16_part(uint32_t smem_dst, const void* src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(smem_dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void cp_async_wait1() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }
__device__ __forceinline__ void cp_async_wait0() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// 16-byte vectors of either type as pairs
template <typename T> struct Vec;
template <> struct Vec<__nv_bfloat16> {
    static constexpr int N = 8, P = 4;
    static __device__ __forceinline__ void unpack(const uint4& r, f2 (&f)[4]) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] = f2_make(__uint_as_float(w[k] << 16), __uint_as_float(w[k] & 0xffff0000u));
    }
    static __device__ __forceinline__ uint4 pack(const f2 (&f)[4]) {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float lo, hi;
            f2_split(f[k], lo, hi);
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[k]) : "f"(hi), "f"(lo));
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <> struct Vec<float> {
    static constexpr int N = 4, P = 2;
    static __device__ __forceinline__ void unpack(const uint4& r, f2 (&f)[2]) {
        f[0] = f2_make(__uint_as_float(r.x), __uint_as_float(r.y));
        f[1] = f2_make(__uint_as_float(r.z), __uint_as_float(r.w));
    }
    static __device__ __forceinline__ uint4 pack(const f2 (&f)[2]) {
        float a, b, c, d;
        f2_split(f[0], a, b);
        f2_split(f[1], c, d);
        return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
    }
};

// K sums over the CTA at once, each the same in every thread afterwards.  Inside a warp the K values are halved with every
// exchange (a lane passes on the half that its partner keeps), K - 1 + 5 - log2 K shuffles instead of 5 K; across warps they
// go through `red` (two halves of [16][K] floats used in turn: one barrier per call).
template <int K>
__device__ __forceinline__ void cta_sums(float (&v)[K], float* red, int& turn) {
    static_assert(K == 1 || K == 2 || K == 4 || K == 8, "power of two");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    int o = 16;
    float w[K];
#pragma unroll
    for (int k = 0; k < K; ++k) w[k] = v[k];
#pragma unroll
    for (int n = K; n > 1; n >>= 1, o >>= 1) {
        const bool up = (lane & o) != 0;
#pragma unroll
        for (int k = 0; k < n / 2; ++k) {
            const float keep = up ? w[k + n / 2] : w[k], give = up ? w[k] : w[k + n / 2];
            w[k] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
    }
    float t = w[0];
#pragma unroll
    for (; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    // a lane now holds the sum whose number its top log2 K bits spell
    constexpr int kShift = K == 1 ? 5 : K == 2 ? 4 : K == 4 ? 3 : 2;
    if (warps == 1) {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = __shfl_sync(0xffffffffu, t, k << kShift);
        return;
    }
    float* r = red + turn * (kMaxThreads / 32) * K;
    turn ^= 1;
    if ((lane & ((1 << kShift) - 1)) == 0) r[warp * K + (lane >> kShift)] = t;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = 0.0f;
    for (int q = 0; q < warps; ++q) {
        if constexpr (K >= 4) {
#pragma unroll
            for (int k = 0; k < K; k += 4) {
                const float4 x = *reinterpret_cast<const float4*>(r + q * K + k);
                v[k] += x.x; v[k + 1] += x.y; v[k + 2] += x.z; v[k + 3] += x.w;
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) v[k] += r[q * K + k];
        }
    }
}

// Where a CTA's rows lie.  EDGE: rows q, q + period, ... with q = blockIdx.x mod period; `lead` elements of a row's first vector
// belong to what lies before the row.
template <typename T, bool EDGE>
struct Rows {
    long long q = 0, n;         // first row, number of rows
    int lead = 0, nvec, period = 1;
    long long first, step;      // this CTA's first batch and the way to the next, in rows of its class
    __device__ __forceinline__ Rows(const void* x, long long stride, long long T_, int D, int period_, int R) {
        constexpr int N = Vec<T>::N;
        if constexpr (EDGE) {
            period = period_;
            q = blockIdx.x & (period - 1);
            n = (T_ - q + period - 1) / period;
            lead = (int)(reinterpret_cast<uintptr_t>(static_cast<const T*>(x) + q * stride) & 15) / (int)sizeof(T);
            nvec = (lead + D + N - 1) / N;
            first = (long long)(blockIdx.x / period) * R;
            step = (long long)(gridDim.x / period) * R;
        } else {
            n = T_;
            nvec = D / N;
            first = (long long)blockIdx.x * R;
            step = (long long)gridDim.x * R;
        }
    }
    __device__ __forceinline__ long long row(long long j) const { return EDGE ? q + j * period : j; }
    // vector c of the row that starts at src, on its way to dst; a tensor's very first vector is not read before its start (only
    // row 0, `top`, can start in it: rows are as long as a vector or longer)
    __device__ __forceinline__ void copy(uint4* dst, const T* src, int c, int D, bool top) const {
        constexpr int N = Vec<T>::N;
        const uint4* from = reinterpret_cast<const uint4*>(src - lead) + c;
        if constexpr (!EDGE) {
            cp_async16(smem_at(dst), from);
        } else if (top && c == 0 && lead > 0) {
            for (int e = lead; e < N && e < lead + D; ++e) reinterpret_cast<T*>(dst)[e] = src[e - lead];
        } else {
            cp_async16_part(smem_at(dst), from, min(16, (lead + D - c * N) * (int)sizeof(T)));
        }
    }
    // which elements of vector c are the row's
    __device__ __forceinline__ unsigned bits(int c, int D) const {
        constexpr int N = Vec<T>::N;
        const int lo = max(0, lead - c * N), hi = min(N, lead + D - c * N);
        return hi > lo ? ((1u << hi) - 1u) & ~((1u << lo) - 1u) : 0u;
    }
    __device__ __forceinline__ void store(T* row_start, int c, const uint4& v, unsigned keep) const {
        constexpr int N = Vec<T>::N;
        T* d = row_start - lead;
        if (!EDGE || keep == (1u << N) - 1u) {
            reinterpret_cast<uint4*>(d)[c] = v;
        } else {
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < N; ++e)
                if ((keep >> e) & 1u) {
                    if constexpr (N == 4) reinterpret_cast<uint32_t*>(d)[c * N + e] = w[e];
                    else reinterpret_cast<uint16_t*>(d)[c * N + e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
                }
        }
    }
};
// what a first or last vector holds of other rows becomes zero
template <int P>
__device__ __forceinline__ void mask_pairs(f2 (&v)[P], unsigned keep) {
#pragma unroll
    for (int e = 0; e < P; ++e) {
        float lo, hi;
        f2_split(v[e], lo, hi);
        v[e] = f2_make((keep >> (2 * e)) & 1u ? lo : 0.0f, (keep >> (2 * e + 1)) & 1u ? hi : 0.0f);
    }
}
__device__ __forceinline__ float ld_w_in(const void* w, int w_bf16, int D, int c) {
    return c >= 0 && c < D ? ld_w(w, w_bf16, c) : 0.0f;
}

// weights of a thread's columns, widened (0 outside the width or without a vector)
template <int P, int NV>
__device__ __forceinline__ void load_w(const void* w, int w_bf16, int D, int lead, f2 (&f)[NV][P]) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < P; ++e) {
            const int c = ((i * (int)blockDim.x + (int)threadIdx.x) * P + e) * 2 - lead;
            f[i][e] = w != nullptr ? f2_make(ld_w_in(w, w_bf16, D, c), ld_w_in(w, w_bf16, D, c + 1)) : 0ull;
        }
}

// A row of any alignment into shared memory, by the whole CTA: the aligned 16-byte chunks that cover it.  Returns where its
// element 0 then lies.  Only the row's own bytes and, before them, bytes of the chunk it starts in are read; a tensor's first
// row, before which there may be nothing, has the elements of that chunk copied one by one (rows are as long as a chunk or
// longer, so that no other row starts in the tensor's first).
__device__ __forceinline__ int chunk_head(const void* src) { return (int)(reinterpret_cast<uintptr_t>(src) & 15); }
template <typename T>
__device__ __forceinline__ void copy_row(char* dst, const T* src, int D, bool first) {
    const int head = chunk_head(src), bytes = head + D * (int)sizeof(T);
    const char* from = reinterpret_cast<const char*>(src) - head;
    for (int o = 16 * threadIdx.x; o < bytes; o += 16 * blockDim.x) {
        if (first && o < head) {
            for (int e = head; e < 16 && e < bytes; e += (int)sizeof(T)) *reinterpret_cast<T*>(dst + e) = *reinterpret_cast<const T*>(from + e);
        } else {
            cp_async16_part(smem_at(dst + o), from + o, min(16, bytes - o));
        }
    }
}
__host__ __device__ constexpr int staged_pitch(int D, int esz) { return (D * esz + 15 + 16) / 16 * 16; }

// how rows are cut: in vectors (wide), in vectors with ragged ends (edge), or staged through shared memory
enum Form { kStaged, kWide, kEdge };
// Which of the forms fits rows at these addresses (NULL: not there) with these strides; `period` for the edge form: rows of all
// tensors must sit alike in their vectors, and a CTA takes every period-th row.
static Form row_form(bool bf16, long long T, int D, const void* const* at, int n, long long stride_a, long long stride_b, int* period) {
    const int v = bf16 ? 8 : 4;
    const uintptr_t base = reinterpret_cast<uintptr_t>(at[0]);
    *period = 1;
    for (int i = 1; i < n; ++i)
        if (at[i] && (reinterpret_cast<uintptr_t>(at[i]) - base) % 16 != 0) return kStaged;
    if (T > 1 && (stride_a % v != D % v || stride_b % v != D % v)) return kStaged;
    if (base % 16 == 0 && D % v == 0) return kWide;
    while (T > 1 && *period * (long long)D % v != 0) *period *= 2;
    return T < *period ? kStaged : kEdge;
}

}  // namespace nm
}  // namespace rlf
