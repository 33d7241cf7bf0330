// Residual addition and RMS norm between blocks, with the output in the
// activations' type or in 8 bits with a scale per row; and its gradients.
//
//     r = x + residual,  rstd = 1 / sqrt(mean(r^2) + eps),  y = r rstd w
//     t = r w, m = max |t|:  q = round(t / m top),  scale = m rstd / top
//     n = r rstd, g = dy w:  dr = rstd (g - n mean(g n)) + dresidual,  dw = sum dy n
//
// Bound by HBM: every tensor is read or written once.  A row is a workgroup's, as
// wide as the row is with 8 values a lane (up to 1,024 lanes, then 16 or 32 values),
// and stays in registers between the row's sums and the stores.  A wavefront a row,
// which needs no barrier, is slower or no faster in nearly every size: its 40 or 64
// values a lane leave few wavefronts (y of 16,384 x 2,560 bf16 60 us, 69; of 16,384 x
// 4,096 91, 156; with 8 values a lane 4,096 x 500 5.2, 4.8).
//
// Measured without a residual, 16,384 x 2,560 in bf16, repeated on the same tensors
// (in part from the cache): y 60 us, e4m3 53, gradients 51.  From HBM, with a
// float32 residual stream: 92 us (5.5 TB/s), e4m3 with a bf16 one 61, gradients 144.
//
// q needs no rstd: t / m is the same for a row however it is scaled, so the
// rounding is of the exact quotient of two float32 products and does not depend
// on the order of the row's sum.
#include <type_traits>

#include "ssd_internal.h"
#include "ssd_ops.h"

namespace ssd {
namespace {

constexpr int kV = 8;

// kV values of a row from column c on, as they lie in memory.  WHOLE: C is a
// multiple of kV, and where c is behind the row's end its last values stand in, so
// that no branch parts one load from the next (with the branches of the other case,
// zeros behind the end, each load waits for the one before: gradients of 16,384 x
// 2,560 bf16 51 us, of 16,384 x 2,561 62).
template <typename T, bool WHOLE>
struct Values {
    static constexpr int kWide = sizeof(T) == 2 ? 8 : 4;
    Pack<T, kWide> part[kV / kWide];
    __device__ __forceinline__ float operator[](int e) const { return part[e / kWide][e % kWide]; }
    __device__ __forceinline__ void load(const T* row, int c, int C)
    {
        if (WHOLE || c + kV <= C) {
            if (WHOLE) c = c < C ? c : C - kV;
#pragma unroll
            for (int k = 0; k < kV / kWide; ++k) part[k] = Pack<T, kWide>::load(row + c + k * kWide);
            return;
        }
#pragma unroll
        for (int e = 0; e < kV; ++e) part[e / kWide].v[e % kWide] = c + e < C ? row[c + e] : T{};
    }
};

template <bool WHOLE, typename T>
__device__ __forceinline__ void store8(T* row, int c, int C, const float (&v)[kV])
{
    if (WHOLE || c + kV <= C) {
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
template <bool WHOLE>
__device__ __forceinline__ void store8b(uint8_t* row, int c, int C, uint32_t lo, uint32_t hi)
{
    if (WHOLE || c + kV <= C) {
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

// Largest over 16 lanes, and over the wavefront's (of values >= 0).
__device__ __forceinline__ float row_max16(float v)
{
    v = dpp_max<0x128>(v);
    v = dpp_max<0x124>(v);
    v = dpp_max<0x122>(v);
    return dpp_max<0x121>(v);
}

__device__ __forceinline__ float wave_max(float v)
{
    v = row_max16(v);
    uint32_t u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    u = __float_as_uint(v);
    const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// The sums (or maxima) of a workgroup's wavefronts, one in every lane l % 16, joined.
__device__ __forceinline__ float waves_sum(const float* s)
{
    const int l = threadIdx.x & 15;
    return row_sum16(l < static_cast<int>(blockDim.x >> 6) ? s[l] : 0.f);
}

__device__ __forceinline__ float waves_max(const float* s)
{
    const int l = threadIdx.x & 15;
    return row_max16(l < static_cast<int>(blockDim.x >> 6) ? s[l] : 0.f);
}

constexpr int kWidest = 1024;

template <typename T, typename R, NormOut OUT, int NV, bool WHOLE>
__global__ __launch_bounds__(kWidest) void k_add_norm(NormParams p)
{
    const int64_t row = static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x;
    if (row >= p.rows) return;   // (whole workgroups)
    const int lane = threadIdx.x, lanes = blockDim.x, C = static_cast<int>(p.C);
    const T* x = static_cast<const T*>(p.x) + row * p.C;
    const R* res = p.res ? static_cast<const R*>(p.res) + row * p.C : nullptr;
    Values<T, WHOLE> in[NV];
    Values<R, WHOLE> more[NV] = {};
    Values<float, WHOLE> weight[NV];
    float r[NV][kV], sum = 0.f, most = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) in[k].load(x, (k * lanes + lane) * kV, C);
    if (res)
#pragma unroll
        for (int k = 0; k < NV; ++k) more[k].load(res, (k * lanes + lane) * kV, C);
    if (p.weight)
#pragma unroll
        for (int k = 0; k < NV; ++k) weight[k].load(p.weight, (k * lanes + lane) * kV, C);
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < kV; ++e) r[k][e] = res ? in[k][e] + more[k][e] : in[k][e];
    if (p.res_out) {
        R* out = static_cast<R*>(p.res_out) + row * p.C;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * lanes + lane) * kV;
            if (c < C) store8<WHOLE>(out, c, C, r[k]);
        }
    }
    // r becomes t = r w
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        float squares = 0.f, high = 0.f;
        bool odd = false;   // some t is infinite or a NaN
#pragma unroll
        for (int e = 0; e < kV; ++e) {
            squares = fmaf(r[k][e], r[k][e], squares);
            if (p.weight) r[k][e] *= weight[k][e];
            if (OUT != kNormSame) {
                const float m = fabsf(r[k][e]);
                odd |= !(m < INFINITY);
                high = fmaxf(high, m);
            }
        }
        if (odd) high = INFINITY;
        const bool live = (k * lanes + lane) * kV < C;
        sum += live ? squares : 0.f;
        most = fmaxf(most, live ? high : 0.f);
    }
    sum = wave_sum(sum);
    if (OUT != kNormSame) most = wave_max(most);
    __shared__ float s[2][kWidest / 64];
    if ((lane & 63) == 0) {
        s[0][lane >> 6] = sum;
        s[1][lane >> 6] = most;
    }
    __syncthreads();
    sum = waves_sum(s[0]);
    if (OUT != kNormSame) most = waves_max(s[1]);
    const float rstd = 1.f / sqrtf(sum / static_cast<float>(p.C) + p.eps);
    if constexpr (OUT == kNormSame) {
        T* y = static_cast<T*>(p.y) + row * p.C;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * lanes + lane) * kV;
#pragma unroll
            for (int e = 0; e < kV; ++e) r[k][e] *= rstd;
            if (c < C) store8<WHOLE>(y, c, C, r[k]);
        }
    } else {
        constexpr float kTop = OUT == kNormI8 ? 127.f : 448.f;
        uint8_t* q = static_cast<uint8_t*>(p.y) + row * p.C;
        const bool bad = !(sum < INFINITY) || !(most < INFINITY);
        const bool none = bad || most == 0.f;   // (without eps, rstd of a row of zeros is infinite)
        if (lane == 0) p.scale[row] = bad ? __uint_as_float(0x7FC00000u) : none ? 0.f : most * rstd / kTop;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * lanes + lane) * kV;
            if (c >= C) continue;
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
            store8b<WHOLE>(q, c, C, out[0], out[1]);
        }
    }
}

// c, made where it is used: the compiler would keep the addresses of all of a row's
// vectors in registers from one row to the next.
__device__ __forceinline__ int here(int c)
{
    asm volatile("" : "+v"(c));
    return c;
}

// Eight channels' operands of the gradients.
template <typename T, typename R, bool WHOLE>
struct GradValues {
    Values<R, WHOLE> r, d;
    Values<T, WHOLE> g;
    __device__ __forceinline__ void load(const NormParams& p, int64_t row, int c)
    {
        const int C = static_cast<int>(p.C);
        r.load(static_cast<const R*>(p.res) + row * p.C, c, C);
        g.load(static_cast<const T*>(p.x) + row * p.C, c, C);
        if (p.dres) d.load(static_cast<const R*>(p.dres) + row * p.C, c, C);
    }
};

// Gradients: a workgroup takes every `step`-th row, with its columns' sums of
// dweight in registers, one partial row of the workspace each.  With 8 channels a
// lane the weights stay in registers too, and the next row is loaded before the
// present one's sums are joined; a wider row has no registers for that and is read
// once more, from the cache, after its sums (16,384 x 20,000 bf16 637 us, kept in
// registers 1,590).  Above 16,384 channels, with 32 sums of dweight a lane, that still
// leaves 2 to 67 values of a lane in scratch memory.
template <typename T, typename R, int NV, bool WHOLE>
__global__ __launch_bounds__(kWidest) void k_add_norm_backward(NormParams p, int64_t step)
{
    constexpr bool kAhead = NV == 1;
    const int64_t first = blockIdx.x;   // < step <= rows
    const int lane = threadIdx.x, lanes = blockDim.x, C = static_cast<int>(p.C);
    float dw[NV][kV] = {};
    GradValues<T, R, WHOLE> now, next;
    Values<float, WHOLE> w;
    if constexpr (kAhead) {
        next.load(p, first, lane * kV);
        if (p.weight) w.load(p.weight, lane * kV, C);
    }
    int turn = 0;
    for (int64_t row = first; row < p.rows; row += step) {
        float ss = 0.f, gr = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if constexpr (kAhead) {
                now = next;
                if (row + step < p.rows) next.load(p, row + step, lane * kV);
            } else {
                const int c = here((k * lanes + lane) * kV);
                now.load(p, row, c);
                if (p.weight) w.load(p.weight, c, C);
            }
            float squares = 0.f, products = 0.f;
#pragma unroll
            for (int e = 0; e < kV; ++e) {
                const float r = now.r[e], g = now.g[e];
                squares = fmaf(r, r, squares);
                products = fmaf(p.weight ? g * w[e] : g, r, products);
            }
            const bool live = (k * lanes + lane) * kV < C;
            ss += live ? squares : 0.f;
            gr += live ? products : 0.f;
        }
        ss = wave_sum(ss);
        gr = wave_sum(gr);
        __shared__ float s[2][2][kWidest / 64];   // alternating, so that one barrier a row is enough
        if ((lane & 63) == 0) {
            s[turn][0][lane >> 6] = ss;
            s[turn][1][lane >> 6] = gr;
        }
        __syncthreads();
        ss = waves_sum(s[turn][0]);
        gr = waves_sum(s[turn][1]);
        turn ^= 1;
        const float n = static_cast<float>(p.C);
        const float rstd = 1.f / sqrtf(ss / n + p.eps);
        const float back = gr * rstd * rstd / n;   // mean(g n) rstd
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = kAhead ? lane * kV : here((k * lanes + lane) * kV);
            if constexpr (!kAhead) {
                now.load(p, row, c);
                if (p.weight) w.load(p.weight, c, C);
            }
            float out[kV];
#pragma unroll
            for (int e = 0; e < kV; ++e) {
                const float r = now.r[e], g = now.g[e], d = p.dres ? now.d[e] : 0.f;
                dw[k][e] = fmaf(g, r * rstd, dw[k][e]);
                out[e] = fmaf(rstd, (p.weight ? g * w[e] : g) - r * back, d);
            }
            if (c >= C) continue;
            if (p.y) store8<WHOLE>(static_cast<T*>(p.y) + row * p.C, c, C, out);
            if (p.res_out) store8<WHOLE>(static_cast<R*>(p.res_out) + row * p.C, c, C, out);
        }
    }
    if (p.partial) {
        float* out = p.partial + first * p.C;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * lanes + lane) * kV;
            if (c < C) store8<WHOLE>(out, c, C, dw[k]);
        }
    }
}

__global__ __launch_bounds__(kSumLanes * kSumCols) void k_norm_dw(const float* partial, int64_t rows, int64_t C, float* dw)
{
    const int64_t c = static_cast<int64_t>(blockIdx.x) * kSumCols + threadIdx.x % kSumCols;
    const float v = column_sum(partial + c, rows, C, c < C);
    if (threadIdx.x < kSumCols && c < C) dw[c] = v;
}

// Vectors a lane: one, as long as a workgroup is wide enough for the row.
int vectors(int64_t C) { return C <= kWidest * kV ? 1 : C <= 2 * kWidest * kV ? 2 : 4; }

int row_threads(int64_t C)
{
    const int64_t per = vectors(C) * kV * 64;
    return static_cast<int>((C + per - 1) / per) * 64;
}

template <typename T, typename R, NormOut OUT, int NV, bool WHOLE>
hipError_t forward(const NormParams& p, hipStream_t stream)
{
    // a dimension of a launch has 32 bits of threads; the rows go on in the second (of
    // the most elements that a tensor may have, 512 times)
    const int threads = row_threads(p.C);
    const int64_t most = 0xffffffffLL / threads, x = p.rows < most ? p.rows : most, y = (p.rows + x - 1) / x;
    hipLaunchKernelGGL((k_add_norm<T, R, OUT, NV, WHOLE>), dim3(static_cast<unsigned>(x), static_cast<unsigned>(y)),
                       dim3(threads), 0, stream, p);
    return hipGetLastError();
}

template <typename T, typename R, int NV, bool WHOLE>
hipError_t backward(const NormParams& p, hipStream_t stream)
{
    const int64_t partials = norm_bwd_partials(p.rows, p.C);
    hipLaunchKernelGGL((k_add_norm_backward<T, R, NV, WHOLE>), dim3(static_cast<unsigned>(partials)), dim3(row_threads(p.C)),
                       0, stream, p, partials);
    return hipGetLastError();
}

// f of the vectors that a lane holds and of whether C is a multiple of theirs.
template <typename F>
hipError_t by_row(const NormParams& p, F f)
{
    const auto with = [&](auto whole) {
        const int n = vectors(p.C);
        return n == 1   ? f(std::integral_constant<int, 1>{}, whole)
               : n == 2 ? f(std::integral_constant<int, 2>{}, whole)
                        : f(std::integral_constant<int, 4>{}, whole);
    };
    return p.C % kV == 0 ? with(std::true_type{}) : with(std::false_type{});
}

template <typename T, typename R>
hipError_t by_out(const NormParams& p, NormOut out, hipStream_t stream)
{
    return by_row(p, [&](auto n, auto whole) {
        constexpr int V = decltype(n)::value;
        constexpr bool W = decltype(whole)::value;
        if (out == kNormSame) return forward<T, R, kNormSame, V, W>(p, stream);
        if (out == kNormI8) return forward<T, R, kNormI8, V, W>(p, stream);
        return forward<T, R, kNormE4M3, V, W>(p, stream);
    });
}

template <typename T, typename R>
hipError_t grads(const NormParams& p, hipStream_t stream)
{
    return by_row(p, [&](auto n, auto whole) {
        return backward<T, R, decltype(n)::value, decltype(whole)::value>(p, stream);
    });
}

}  // namespace

// Workgroups of the gradient kernel: 4,096 wavefronts, four a SIMD (16,384 x 4,096
// bf16 79 us, 8,192 wavefronts 94; 16,384 x 8,192 150, 2,048 wavefronts 235), and at
// least two rows each: a partial row of dweight for every row costs more to add up
// than it saves (512 x 4,096 10.1 us, one row each 13.9).
int64_t norm_bwd_partials(int64_t rows, int64_t C)
{
    const int64_t most = 4096 / (row_threads(C) / 64), n = (rows + 1) / 2;
    return n < most ? n : most;
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
