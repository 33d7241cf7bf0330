// Residual addition and RMS norm between blocks, with the output in the
// activations' type or in 8 bits with a scale per row; and its gradients.
//
//     r = x + residual,  rstd = 1 / sqrt(mean(r^2) + eps),  y = r rstd w
//     t = r w, m = max |t|:  q = round(t / m top),  scale = m rstd / top
//     n = r rstd, g = dy w:  dr = rstd (g - n mean(g n)) + dresidual,  dw = sum dy n
//
// Bound by HBM: every tensor is read or written once.  `LANES` lanes share a row
// and keep it in registers (NV vectors of 8 values a lane) between the row's
// sums and the stores.  Where there are enough rows to fill the device a row is a
// wavefront's (sums in registers, no barrier); fewer rows take a workgroup each.
//
// q needs no rstd: t / m is the same for a row however it is scaled, so the
// rounding is of the exact quotient of two float32 products and does not depend
// on the order of the row's sum.
#include "ssd_internal.h"
#include "ssd_ops.h"

namespace ssd {
namespace {

constexpr int kV = 8;

template <typename T>
__device__ __forceinline__ void load8(const T* row, int64_t c, int64_t C, float (&v)[kV])
{
    if (c + kV <= C) {
        const auto a = Pack<T, 4>::load(row + c), b = Pack<T, 4>::load(row + c + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = a[e];
            v[4 + e] = b[e];
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < kV; ++e) v[e] = c + e < C ? widen(row[c + e]) : 0.f;
}

template <>
__device__ __forceinline__ void load8<uint16_t>(const uint16_t* row, int64_t c, int64_t C, float (&v)[kV])
{
    if (c + kV <= C) {
        const auto a = Pack<uint16_t, 8>::load(row + c);
#pragma unroll
        for (int e = 0; e < kV; ++e) v[e] = a[e];
        return;
    }
#pragma unroll
    for (int e = 0; e < kV; ++e) v[e] = c + e < C ? widen(row[c + e]) : 0.f;
}

template <typename T>
__device__ __forceinline__ void store8(T* row, int64_t c, int64_t C, const float (&v)[kV])
{
    if (c + kV <= C) {
        constexpr int N = sizeof(T) == 2 ? 8 : 4;
#pragma unroll
        for (int k = 0; k < kV; k += N) {
            Pack<T, N> o;
#pragma unroll
            for (int e = 0; e < N; ++e) o.set(e, v[k + e]);
            o.store(row + c + k);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < kV; ++e)
        if (c + e < C) row[c + e] = narrow<T>(v[e]);
}

// Eight bytes, packed low to high.
__device__ __forceinline__ void store8b(uint8_t* row, int64_t c, int64_t C, uint32_t lo, uint32_t hi)
{
    if (c + kV <= C) {
        typedef uint32_t u2 __attribute__((ext_vector_type(2), aligned(1)));
        *reinterpret_cast<u2*>(row + c) = u2{lo, hi};
        return;
    }
#pragma unroll
    for (int e = 0; e < kV; ++e)
        if (c + e < C) row[c + e] = static_cast<uint8_t>((e < 4 ? lo >> (8 * e) : hi >> (8 * (e - 4))) & 0xFF);
}

template <int CTRL>
__device__ __forceinline__ float dpp_max(float v)
{
    return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, false)));
}

// Largest over the wavefront's lanes (of values >= 0).
__device__ __forceinline__ float wave_max(float v)
{
    v = dpp_max<0x128>(v);
    v = dpp_max<0x124>(v);
    v = dpp_max<0x122>(v);
    v = dpp_max<0x121>(v);
    uint32_t u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    u = __float_as_uint(v);
    const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// A row's sum and maximum over its LANES lanes.
template <int LANES>
__device__ __forceinline__ void row_reduce(float& sum, float& most)
{
    sum = wave_sum(sum);
    most = wave_max(most);
    if constexpr (LANES > 64) {
        constexpr int W = LANES / 64;
        __shared__ float s[2][W];
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
            s[0][wave] = sum;
            s[1][wave] = most;
        }
        __syncthreads();
        sum = 0.f;
        most = 0.f;
#pragma unroll
        for (int k = 0; k < W; ++k) {
            sum += s[0][k];
            most = fmaxf(most, s[1][k]);
        }
    }
}

// LANES lanes a row; workgroups of at least 256 threads (4 rows of one wavefront).
template <int LANES>
constexpr int kBlock = LANES > 256 ? LANES : 256;

template <typename T, typename R, NormOut OUT, int LANES, int NV>
__global__ __launch_bounds__(kBlock<LANES>) void k_add_norm(NormParams p)
{
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (kBlock<LANES> / LANES) + uniform(threadIdx.x / LANES);
    if (row >= p.rows) return;   // (whole wavefronts; with a workgroup a row, never)
    const int lane = threadIdx.x % LANES;
    const T* x = static_cast<const T*>(p.x) + row * p.C;
    const R* res = p.res ? static_cast<const R*>(p.res) + row * p.C : nullptr;
    float r[NV][kV], sum = 0.f, most = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int64_t c = (static_cast<int64_t>(k) * LANES + lane) * kV;
        if (c < p.C) {
            load8(x, c, p.C, r[k]);
            if (res) {
                float a[kV];
                load8(res, c, p.C, a);
#pragma unroll
                for (int e = 0; e < kV; ++e) r[k][e] += a[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < kV; ++e) r[k][e] = 0.f;
        }
    }
    if (p.res_out) {
        R* out = static_cast<R*>(p.res_out) + row * p.C;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int64_t c = (static_cast<int64_t>(k) * LANES + lane) * kV;
            if (c < p.C) store8(out, c, p.C, r[k]);
        }
    }
    // r becomes t = r w
    bool odd = false;   // some t is infinite or a NaN
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int64_t c = (static_cast<int64_t>(k) * LANES + lane) * kV;
        float w[kV];
        if (p.weight && c < p.C) {
            load8(p.weight, c, p.C, w);
        } else {
#pragma unroll
            for (int e = 0; e < kV; ++e) w[e] = 1.f;
        }
#pragma unroll
        for (int e = 0; e < kV; ++e) {
            sum = fmaf(r[k][e], r[k][e], sum);
            r[k][e] *= w[e];
            if (OUT != kNormSame) {
                const float m = fabsf(r[k][e]);
                odd |= !(m < INFINITY);
                most = fmaxf(most, m);
            }
        }
    }
    if (odd) most = INFINITY;
    row_reduce<LANES>(sum, most);
    const float rstd = 1.f / sqrtf(sum / static_cast<float>(p.C) + p.eps);
    if constexpr (OUT == kNormSame) {
        T* y = static_cast<T*>(p.y) + row * p.C;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int64_t c = (static_cast<int64_t>(k) * LANES + lane) * kV;
#pragma unroll
            for (int e = 0; e < kV; ++e) r[k][e] *= rstd;
            if (c < p.C) store8(y, c, p.C, r[k]);
        }
    } else {
        constexpr float kTop = OUT == kNormI8 ? 127.f : 448.f;
        uint8_t* q = static_cast<uint8_t*>(p.y) + row * p.C;
        const bool bad = !(sum < INFINITY) || !(most < INFINITY);
        if (lane == 0) p.scale[row] = bad ? __uint_as_float(0x7FC00000u) : most * rstd / kTop;
        const bool none = bad || most == 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int64_t c = (static_cast<int64_t>(k) * LANES + lane) * kV;
            if (c >= p.C) continue;
            uint32_t out[2] = {0, 0};
            if (!none) {
                float v[kV];
#pragma unroll
                for (int e = 0; e < kV; ++e) v[e] = r[k][e] / most * kTop;
                if constexpr (OUT == kNormI8) {
#pragma unroll
                    for (int e = 0; e < kV; ++e)
                        out[e / 4] |= (static_cast<uint32_t>(static_cast<int>(rintf(v[e]))) & 0xFFu) << (8 * (e % 4));
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h], v[4 * h + 1], 0, false);
                        out[h] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2], v[4 * h + 3], w, true);
                    }
                }
            }
            store8b(q, c, p.C, out[0], out[1]);
        }
    }
}

// Gradients: a wavefront (or workgroup) takes every `step`-th row, with its
// columns' sums of dweight in registers, one partial row of the workspace each.
template <typename T, typename R, int LANES, int NV>
__global__ __launch_bounds__(kBlock<LANES>) void k_add_norm_backward(NormParams p, int64_t step)
{
    const int64_t first = static_cast<int64_t>(blockIdx.x) * (kBlock<LANES> / LANES) + uniform(threadIdx.x / LANES);
    const int lane = threadIdx.x % LANES;
    float dw[NV][kV];
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < kV; ++e) dw[k][e] = 0.f;
    for (int64_t row = first; row < p.rows; row += step) {
        const T* dy = static_cast<const T*>(p.x) + row * p.C;
        const R* rp = static_cast<const R*>(p.res) + row * p.C;
        float r[NV][kV], g[NV][kV], ss = 0.f, gr = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int64_t c = (static_cast<int64_t>(k) * LANES + lane) * kV;
            if (c < p.C) {
                load8(rp, c, p.C, r[k]);
                load8(dy, c, p.C, g[k]);
            } else {
#pragma unroll
                for (int e = 0; e < kV; ++e) r[k][e] = g[k][e] = 0.f;
            }
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int64_t c = (static_cast<int64_t>(k) * LANES + lane) * kV;
            float w[kV];
            if (p.weight && c < p.C) {
                load8(p.weight, c, p.C, w);
            } else {
#pragma unroll
                for (int e = 0; e < kV; ++e) w[e] = 1.f;
            }
#pragma unroll
            for (int e = 0; e < kV; ++e) {
                ss = fmaf(r[k][e], r[k][e], ss);
                gr = fmaf(g[k][e] * w[e], r[k][e], gr);
            }
        }
        ss = wave_sum(ss);
        gr = wave_sum(gr);
        if constexpr (LANES > 64) {
            constexpr int W = LANES / 64;
            __shared__ float s[2][2][W];   // alternating, so that one barrier a row is enough
            const int wave = threadIdx.x >> 6, turn = static_cast<int>((row - first) / step) & 1;
            if ((threadIdx.x & 63) == 0) {
                s[turn][0][wave] = ss;
                s[turn][1][wave] = gr;
            }
            __syncthreads();
            ss = gr = 0.f;
#pragma unroll
            for (int k = 0; k < W; ++k) {
                ss += s[turn][0][k];
                gr += s[turn][1][k];
            }
        }
        const float n = static_cast<float>(p.C);
        const float rstd = 1.f / sqrtf(ss / n + p.eps);
        const float back = gr * rstd * rstd / n;   // mean(g n) rstd
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int64_t c = (static_cast<int64_t>(k) * LANES + lane) * kV;
            if (c >= p.C) continue;
            float w[kV], d[kV];
            if (p.weight) {
                load8(p.weight, c, p.C, w);
            } else {
#pragma unroll
                for (int e = 0; e < kV; ++e) w[e] = 1.f;
            }
            if (p.dres) {
                load8(static_cast<const R*>(p.dres) + row * p.C, c, p.C, d);
            } else {
#pragma unroll
                for (int e = 0; e < kV; ++e) d[e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < kV; ++e) {
                dw[k][e] = fmaf(g[k][e], r[k][e] * rstd, dw[k][e]);
                d[e] = fmaf(rstd, fmaf(g[k][e], w[e], -r[k][e] * back), d[e]);
            }
            if (p.y) store8(static_cast<T*>(p.y) + row * p.C, c, p.C, d);
            if (p.res_out) store8(static_cast<R*>(p.res_out) + row * p.C, c, p.C, d);
        }
    }
    if (p.partial && first < step) {
        float* out = p.partial + first * p.C;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int64_t c = (static_cast<int64_t>(k) * LANES + lane) * kV;
            if (c < p.C) store8(out, c, p.C, dw[k]);
        }
    }
}

__global__ __launch_bounds__(kSumLanes * kSumCols) void k_norm_dw(const float* partial, int64_t rows, int64_t C, float* dw)
{
    const int64_t c = static_cast<int64_t>(blockIdx.x) * kSumCols + threadIdx.x % kSumCols;
    const float v = column_sum(partial + c, rows, C, c < C);
    if (threadIdx.x < kSumCols && c < C) dw[c] = v;
}

// Lanes a row: a wavefront where rows are many and short enough for its
// registers, else a workgroup of 256 or (beyond 16,384 channels) 1,024.
int row_lanes(int64_t rows, int64_t C)
{
    if (C <= 64 * 8 * kV && rows >= 1024) return 64;
    return C <= 256 * 8 * kV ? 256 : 1024;
}

template <typename T, typename R, NormOut OUT, int LANES, int NV>
hipError_t forward(const NormParams& p, hipStream_t stream)
{
    constexpr int64_t per = kBlock<LANES> / LANES;
    const int64_t grid = (p.rows + per - 1) / per;
    if (!fits(grid, kBlock<LANES>)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((k_add_norm<T, R, OUT, LANES, NV>), dim3(static_cast<unsigned>(grid)), dim3(kBlock<LANES>), 0,
                       stream, p);
    return hipGetLastError();
}

template <typename T, typename R, int LANES, int NV>
hipError_t backward(const NormParams& p, hipStream_t stream)
{
    constexpr int64_t per = kBlock<LANES> / LANES;
    const int64_t partials = norm_bwd_partials(p.rows, p.C);   // a multiple of `per`
    hipLaunchKernelGGL((k_add_norm_backward<T, R, LANES, NV>), dim3(static_cast<unsigned>(partials / per)),
                       dim3(kBlock<LANES>), 0, stream, p, partials);
    return hipGetLastError();
}

template <int L, int V>
struct Row {
    static constexpr int lanes = L, vectors = V;
};

// f of the row's lanes and of the vectors that a lane holds.
template <typename F>
hipError_t by_row(const NormParams& p, F f)
{
    const int lanes = row_lanes(p.rows, p.C);
    const int64_t per = static_cast<int64_t>(lanes) * kV, n = (p.C + per - 1) / per;
    if (lanes == 1024) return n <= 3 ? f(Row<1024, 3>{}) : f(Row<1024, 4>{});
    const auto with = [&](auto l) {
        constexpr int L = decltype(l)::lanes;
        if (n <= 1) return f(Row<L, 1>{});
        if (n <= 2) return f(Row<L, 2>{});
        if (n <= 3) return f(Row<L, 3>{});
        if (n <= 5) return f(Row<L, 5>{});
        return f(Row<L, 8>{});
    };
    return lanes == 64 ? with(Row<64, 1>{}) : with(Row<256, 1>{});
}

template <typename T, typename R>
hipError_t by_out(const NormParams& p, NormOut out, hipStream_t stream)
{
    return by_row(p, [&](auto row) {
        constexpr int L = decltype(row)::lanes, V = decltype(row)::vectors;
        if (out == kNormSame) return forward<T, R, kNormSame, L, V>(p, stream);
        if (out == kNormI8) return forward<T, R, kNormI8, L, V>(p, stream);
        return forward<T, R, kNormE4M3, L, V>(p, stream);
    });
}

template <typename T, typename R>
hipError_t grads(const NormParams& p, hipStream_t stream)
{
    return by_row(p, [&](auto row) {
        return backward<T, R, decltype(row)::lanes, decltype(row)::vectors>(p, stream);
    });
}

}  // namespace

// Wavefronts (or workgroups) of the gradient kernel: eight wavefronts a compute
// unit; more would only write more partial rows of dweight.
int64_t norm_bwd_partials(int64_t rows, int64_t C)
{
    const int lanes = row_lanes(rows, C);
    const int64_t most = lanes == 64 ? 2048 : lanes == 256 ? 512 : 256, per = lanes == 64 ? 4 : 1;
    const int64_t n = rows < most ? rows : most;
    return (n + per - 1) / per * per;
}

hipError_t launch_add_norm(const NormParams& p, bool bf16, bool res_bf16, NormOut out, hipStream_t stream)
{
    if (!bf16) return by_out<float, float>(p, out, stream);
    return res_bf16 ? by_out<uint16_t, uint16_t>(p, out, stream) : by_out<uint16_t, float>(p, out, stream);
}

hipError_t launch_add_norm_backward(const NormParams& p, bool bf16, bool res_bf16, hipStream_t stream)
{
    hipError_t err = !bf16 ? grads<float, float>(p, stream)
                     : res_bf16 ? grads<uint16_t, uint16_t>(p, stream)
                                : grads<uint16_t, float>(p, stream);
    if (err != hipSuccess || !p.dweight) return err;
    hipLaunchKernelGGL(k_norm_dw, dim3(static_cast<unsigned>((p.C + kSumCols - 1) / kSumCols)),
                       dim3(kSumLanes * kSumCols), 0, stream, p.partial, norm_bwd_partials(p.rows, p.C), p.C, p.dweight);
    return hipGetLastError();
}

}  // namespace ssd
