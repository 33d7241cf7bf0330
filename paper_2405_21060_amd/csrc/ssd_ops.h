// Internal interface and device helpers of the operators around the layer: the
// short convolution (ssd_conv.hip), the selective scan (ssd_scan.hip,
// ssd_scan_bwd.hip) and the residual addition with norm (ssd_norm.hip).
// Host validation: ssd_ops_api.cpp.
#pragma once

#include <cfloat>

#include "ssd_device.h"

namespace ssd {

// ---- parameters ------------------------------------------------------------

struct ConvParams {
    int64_t b, T, C, nseq;
    int W, silu, nparts;
    int64_t off[4];         // first channel of each part, then C
    const void* x;
    int64_t xb, xt;         // element strides of batch rows and tokens
    const float* weight;    // (C, W)
    const float* bias;      // (C) or null
    const void* init;       // (units, W - 1, C) or null
    const int32_t* seq_idx; // (T) or null
    void* y[3];             // step: y[0]
    void* fin;              // (units, W - 1, C) or null; step: the state
    // gradients
    const void* dy[3];
    const void* dfin;
    void* dx;
    void* dinit;
    float* dweight;
    float* dbias;
    float* partial;         // workspace: (strips, W + 1, C)
};

// Tokens per strip of the gradient kernel, and its workspace.
int64_t conv_bwd_strip(int64_t b, int64_t T, int64_t C);
hipError_t launch_conv_forward(const ConvParams& p, bool bf16, hipStream_t stream);
hipError_t launch_conv_backward(const ConvParams& p, bool bf16, hipStream_t stream);
hipError_t launch_conv_step(const ConvParams& p, bool bf16, hipStream_t stream);

struct ScanParams {
    int64_t b, T, E, N, G, nseq;
    const void *x, *dt, *z, *B, *C;      // z may be null
    int64_t xb, xt, db, dtt, zb, zt, bb, bt, cb, ct;   // element strides: batch row, token
    const float *A_log, *D, *dt_bias;    // D, dt_bias may be null
    const float* init;                   // (units, E, N) or null
    const int32_t* seq_idx;
    void* y;
    float* fin;                          // or null; step: the state
    int softplus;
    // time split: S chunks of L tokens (S == 1: none), a workspace of chunk
    // states (b, S, N, E) and of each chunk's sum of dt (b, S, E)
    int64_t S, L;
    float* states;
    float* sums;
    float* steps;                        // time steps (b, T, E) (forward)
    // gradients
    const void* dy;
    const float* dfin;
    void *dx, *ddt, *dB, *dC, *dz;
    float *dA_log, *dD, *ddt_bias, *dinit;
    float* rstates;                      // (b, S, N, E) reverse chunk states
    float* marks;                        // states at every tile of tokens (b, tiles, N, E), and
    float* marksums;                     // sums of dt (b, tiles, E), both from the chunk's start
    float* pA;                           // (b S, N, E) partial sums of dA
    float* pD;                           // (b S, 2, E) of dD, ddt_bias
    float* pBC;                          // (channel blocks, b, T, 2, N) of dB, dC
};

struct ScanPlan {
    int64_t S, L;
    size_t states, sums, steps, rstates, marks, marksums, pA, pD, pBC, total;   // byte offsets
    int64_t cblocks;   // channel blocks of the gradients
};

ScanPlan scan_plan(int64_t b, int64_t T, int64_t E, int64_t N, int64_t G, bool backward);
hipError_t launch_scan_forward(const ScanParams& p, bool bf16, hipStream_t stream);
hipError_t launch_scan_backward(const ScanParams& p, bool bf16, hipStream_t stream);
hipError_t launch_scan_step(const ScanParams& p, bool bf16, hipStream_t stream);

struct NormParams {
    int64_t rows, C;
    float eps;
    const void* x;         // gradients: dy
    const void* res;       // or null; gradients: r
    const float* weight;   // or null
    void* y;               // gradients: dx
    float* scale;
    void* res_out;         // or null; gradients: dresidual
    const void* dres;      // gradients: dresidual_out, or null
    float* dweight;
    float* partial;
};

enum NormOut { kNormSame = 0, kNormI8, kNormE4M3 };
// Workgroups' partial rows of dweight in the gradient kernel.
int64_t norm_bwd_partials(int64_t rows, int64_t C);
hipError_t launch_add_norm(const NormParams& p, bool bf16, bool res_bf16, NormOut out, hipStream_t stream);
hipError_t launch_add_norm_backward(const NormParams& p, bool bf16, bool res_bf16, hipStream_t stream);

// Whether so many workgroups of so many threads fit one launch (32 bits of threads).
constexpr bool fits(int64_t groups, int64_t threads) { return groups <= 0xffffffffLL / threads; }

#if defined(__HIP_DEVICE_COMPILE__) || defined(__HIPCC__)

// ---- device helpers ----------------------------------------------------------

// Loads through the scalar cache: a uniform address of memory that the kernel
// does not write.
template <typename T>
__device__ __forceinline__ T scalar_load(const T* p)
{
    return *reinterpret_cast<const __attribute__((address_space(4))) T*>(reinterpret_cast<uintptr_t>(p));
}

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// A sequence id held to the states' range.
__device__ __forceinline__ int64_t held(int32_t id, int64_t nseq)
{
    const int64_t v = id < 0 ? 0 : id;
    return v < nseq ? v : nseq - 1;
}

// exp(v) of v in [-104, 88]: 2^t (1 + r), t = v log2(e) rounded and r what the rounding
// left over (where 2^t alone is off by |v| 6e-8); relative error near 2e-7.
__device__ __forceinline__ float exp_of(float v)
{
    const float t = v * kLog2e, e = __builtin_amdgcn_exp2f(t);
    return fmaf(e, fmaf(t, -0.69314718f, v), e);
}

// exp(-v), likewise.  v is held to +-104, beyond which the result is infinite or 0; a
// NaN counts as one of the two.  2^t is infinite from v < -88.7 on and r of either sign,
// so r is taken of the largest finite number there: infinity times an r of 0 or below
// would be a NaN, or make one.  LARGE: v may be that small (false: a v of 0 and more
// needs no such care).
template <bool LARGE = true>
__device__ __forceinline__ float exp_neg(float v)
{
    v = __builtin_amdgcn_fmed3f(v, -104.f, 104.f);
    const float t = v * -kLog2e, e = __builtin_amdgcn_exp2f(t);
    return fmaf(LARGE ? fminf(e, FLT_MAX) : e, fmaf(t, -0.69314718f, -v), e);
}

__device__ __forceinline__ float sigmoid_hw(float v) { return __builtin_amdgcn_rcpf(1.f + exp_neg(v)); }

// softplus(v) = max(v, 0) + log(1 + u), u = exp(-|v|) in (0, 1]: log(1 + u) =
// 2 atanh(s), s = u / (2 + u) <= 1/3, and atanh(s) / s as a polynomial in s^2 of
// degree 4, the interpolant of its power series at Chebyshev points of [0, 1/9]
// (1e-8 off).  Relative error near 2e-7 also where the result is as small as u, as a
// time step is.  -infinity gives 0, a NaN a NaN.
constexpr float kAtanh0 = 2.f, kAtanh1 = 0.666663229f, kAtanh2 = 0.400245965f, kAtanh3 = 0.279651582f, kAtanh4 = 0.281577796f;   // times 2

__device__ __forceinline__ float softplus_hw(float v, float u)   // u = exp_neg<false>(|v|)
{
    const float s = u * __builtin_amdgcn_rcpf(2.f + u), q = s * s;
    float r = fmaf(q, kAtanh4, kAtanh3);
    r = fmaf(r, q, kAtanh2);
    r = fmaf(r, q, kAtanh1);
    r = fmaf(r, q, kAtanh0);
    return fmaf(s, r, __builtin_elementwise_maximum(v, 0.f));
}

__device__ __forceinline__ float softplus_hw(float v) { return softplus_hw(v, exp_neg<false>(fabsf(v))); }

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); }

template <typename T>
__device__ __forceinline__ T narrow(float v);
template <>
__device__ __forceinline__ float narrow<float>(float v) { return v; }
template <>
__device__ __forceinline__ uint16_t narrow<uint16_t>(float v)   // round to nearest even
{
    return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
}

// V consecutive values of T at any alignment that T itself has (the hardware
// reads and writes vectors at any).
template <typename T, int V>
struct Pack {
    typedef T vec __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    vec v;
    __device__ __forceinline__ float operator[](int i) const { return widen(static_cast<T>(v[i])); }
    __device__ __forceinline__ void set(int i, float f) { v[i] = narrow<T>(f); }
    static __device__ __forceinline__ Pack load(const T* p) { return Pack{*reinterpret_cast<const vec*>(p)}; }
    __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<vec*>(p) = v; }
};

template <typename T>
struct Pack<T, 1> {
    T v;
    __device__ __forceinline__ float operator[](int) const { return widen(v); }
    __device__ __forceinline__ void set(int, float f) { v = narrow<T>(f); }
    static __device__ __forceinline__ Pack load(const T* p) { return Pack{*p}; }
    __device__ __forceinline__ void store(T* p) const { *p = v; }
};

// The sum of a column of partial sums, `rows` values `step` apart: kSumLanes
// threads take every kSumLanes-th value, in four sums of their own, and join in
// order.  Four loads at a time, without a branch between them (8 and 16 are no
// faster for many rows and read in vain where rows are few).  A workgroup takes
// kSumCols columns; the sum is thread (lane 0, col)'s.
constexpr int kSumLanes = 64, kSumCols = 16, kSumBatch = 4;

__device__ __forceinline__ float column_sum(const float* from, int64_t rows, int64_t step, bool real)
{
    __shared__ float part[kSumLanes][kSumCols + 1];
    const int col = threadIdx.x % kSumCols, lane = threadIdx.x / kSumCols;
    float v[kSumBatch] = {};
    if (real)
        for (int64_t k = lane; k < rows; k += kSumBatch * kSumLanes) {
            float f[kSumBatch];
#pragma unroll
            for (int u = 0; u < kSumBatch; ++u) {   // (behind the last row, that row again)
                const int64_t at = k + u * kSumLanes;
                f[u] = from[(at < rows ? at : rows - 1) * step];
            }
#pragma unroll
            for (int u = 0; u < kSumBatch; ++u) v[u] += k + u * kSumLanes < rows ? f[u] : 0.f;
        }
    part[lane][col] = (v[0] + v[1]) + (v[2] + v[3]);
    __syncthreads();
    float sum = 0.f;
    if (lane == 0) {
#pragma unroll 8
        for (int k = 0; k < kSumLanes; ++k) sum += part[k][col];
    }
    return sum;
}

#endif

}  // namespace ssd
