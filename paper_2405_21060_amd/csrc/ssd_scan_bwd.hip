// Gradients of the selective scan (ssd_scan.hip).
//
// With g_t = dL/dh_t (of everything from token t on) and dy~ = dy silu(z):
//     g_t = dy~_t C_t + exp(dt_{t+1} A) g_{t+1}
//     dC_t = sum_e dy~_t h_t,        dB_t = sum_e dt_t x_t g_t,   du_t = g_t . B_t
//     q_t = exp(dt_t A) h_{t-1} g_t  (the gradient of the exponent dt_t A)
//     dx_t = dt_t du_t + D dy~_t,    d(dt_t) = x_t du_t + q_t . A,   dA = sum_t dt_t q_t
//     dz_t = dy_t (h_t . C_t + D x_t) silu'(z_t),   dD = sum_t dy~_t x_t
//
// Passes, each over chunks of tokens as in the forward: the chunks' states from
// zero in both directions, a scan over the chunks in each, the states in front of
// every tile of 16 tokens (the forward's kernel again), then k_scan_grad, which
// takes its chunk's tiles in reverse: four states at a time, a tile's states are
// computed again from its entering ones and kept, with the decays, in registers,
// and then walked back.  The sums over channels for dB and dC run across the
// lanes: 64 values, one after the other, are merged in a tree in which every
// level halves the lanes that a value is spread over, two instructions a value
// where a sum of its own would take seven.  Sums over channel tiles, chunks and
// rows are joined in a fixed order by k_scan_sums.
//
// Bound by vector arithmetic, like the forward.
#include <type_traits>

#include "ssd_internal.h"
#include "ssd_scan.h"

namespace ssd {
namespace {

__device__ __forceinline__ float silu_grad(float z, float s) { return s * fmaf(z, 1.f - s, 1.f); }

// dy~ of a token.
template <typename T>
__device__ __forceinline__ float gated(float dy, const T* z, int64_t at)
{
    if (!z) return dy;
    const float zv = widen(z[at]);
    return dy * zv * sigmoid_hw(zv);
}

// Each chunk's gradient of the state entering it, from a zero gradient behind it
// (from the final state's where a sequence ends).
template <typename T, bool PACKED>
__global__ void k_scan_rev(ScanParams p)
{
    const int slice = uniform(threadIdx.x >> 6), n0 = slice * kSlice;
    const ScanWork w = scan_work(p, blockIdx.x);
    const T* dt = static_cast<const T*>(p.dt) + w.row * p.db + w.e;
    const T* z = p.z ? static_cast<const T*>(p.z) + w.row * p.zb + w.e : nullptr;
    const T* C = static_cast<const T*>(p.C) + w.row * p.cb + w.g * p.N + n0;
    const T* dy = static_cast<const T*>(p.dy) + w.row * p.T * p.E + w.e;
    float A2[kSlice], g[kSlice];
    load_states(p.A_log, p, 0, w.e, n0, A2);
#pragma unroll
    for (int n = 0; n < kSlice; ++n) {
        A2[n] = decay_rate(A2[n]);
        g[n] = 0.f;
    }
    const float bias = p.dt_bias ? p.dt_bias[w.e] : 0.f;
    for (int64_t t = w.t1 - 1; t >= w.t0; t -= kTok) {
        T dr[kTok], yr[kTok], zr[kTok];
#pragma unroll
        for (int u = 0; u < kTok; ++u) {
            const int64_t at = t - u >= w.t0 ? t - u : w.t0;
            dr[u] = dt[at * p.dtt];
            yr[u] = dy[at * p.E];
            if (z) zr[u] = z[at * p.zt];
        }
#pragma unroll
        for (int u = 0; u < kTok; ++u) {
            const int64_t at = t - u;
            if (at < w.t0) break;
            if (scan_ends<PACKED>(p, at)) load_states(p.dfin, p, scan_unit<PACKED>(p, w.row, at), w.e, n0, g);
            const float d = time_step(p, widen(dr[u]) + bias), dyg = gated(widen(yr[u]), z ? zr : nullptr, u);
            float c[kSlice];
            uniform_row(C + at * p.ct, c);
#pragma unroll
            for (int n = 0; n < kSlice; ++n) g[n] = __builtin_amdgcn_exp2f(d * A2[n]) * fmaf(dyg, c[n], g[n]);
        }
    }
    if (!w.live) return;
    float* to = p.rstates + ((w.row * p.S + w.chunk) * p.N + n0) * p.E + w.e;
#pragma unroll
    for (int n = 0; n < kSlice; ++n) to[n * p.E] = g[n];
}

// The scan over chunks, backwards: each chunk's own gradient becomes the gradient
// behind it (of the state that it leaves to the next chunk).
__global__ __launch_bounds__(256) void k_scan_rev_pass(ScanParams p)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= p.b * p.N * p.E) return;
    const int64_t e = i % p.E, rn = i / p.E, n = rn % p.N, row = rn / p.N;
    const float A2 = decay_rate(p.A_log[e * p.N + n]);
    float* st = p.rstates + (row * p.S * p.N + n) * p.E + e;
    const int64_t step = p.N * p.E;
    float g = 0.f;
    for (int64_t c = p.S - 1; c >= 0; --c) {
        const float own = st[c * step];
        st[c * step] = g;
        if (c == 0) break;
        const float half = __builtin_amdgcn_exp2f(p.sums[(row * p.S + c) * p.E + e] * A2 * 0.5f);
        const float through = g * half * half;
        g = own;
        const int64_t t0 = c * p.L, t1 = t0 + p.L < p.T ? t0 + p.L : p.T;
        // (a sequence that ends in the chunk, its last token included, takes nothing from behind it)
        const bool joined = t1 < p.T && (!p.seq_idx || (p.seq_idx[t0] == p.seq_idx[t1 - 1] && p.seq_idx[t1 - 1] == p.seq_idx[t1]));
        if (joined) g += through;
    }
}

template <int CTRL>
__device__ __forceinline__ float moved(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, false));
}

// Merges two values that are each spread over groups of 2^(6 - LEVEL) lanes: lanes
// with the level's bit clear then hold a's halves added, those with it set b's.
template <int LEVEL>
__device__ __forceinline__ float merge(float a, float b, int lane)
{
    if constexpr (LEVEL == 0) {
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
        return __uint_as_float(s[0]) + __uint_as_float(s[1]);
    } else if constexpr (LEVEL == 1) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
        return __uint_as_float(s[0]) + __uint_as_float(s[1]);
    } else {
        const bool bit = lane & (32 >> LEVEL);
        const float keep = bit ? b : a, give = bit ? a : b;
        // row_ror:8, row_half_mirror, quad_perm [2,3,0,1] and [1,0,3,2]
        constexpr int ctrl = LEVEL == 2 ? 0x128 : LEVEL == 3 ? 0x141 : LEVEL == 4 ? 0x4E : 0xB1;
        return keep + moved<ctrl>(give);
    }
}

// The sums over the 64 lanes of 64 values put in one after the other (at
// compile-time places 0 .. 63): after the last, lane l holds the sum of value
// bitreverse6(l).  Holds at most a value per level in between.
struct LaneSums {
    float level[6];
    float out;
    template <int I, int LEVEL = 0>
    __device__ __forceinline__ void put(float v, int lane)
    {
        if constexpr (LEVEL == 6) {
            out = v;
        } else if constexpr ((I >> LEVEL) & 1) {
            put<I, LEVEL + 1>(merge<LEVEL>(level[LEVEL], v, lane), lane);
        } else {
            level[LEVEL] = v;
        }
    }
};

// k_scan_grad's tokens of a tile, from last to first: place I = 15 - token.
template <int I, typename F>
__device__ __forceinline__ void each(F&& f)
{
    if constexpr (I < kBwdTile) {
        f(std::integral_constant<int, I>{});
        each<I + 1>(f);
    }
}

constexpr int kQuad = 4;   // states taken at a time

// One wavefront: 64 channels of one chunk, its tiles from the last to the first.
// Shared memory: the states' running gradients g and sums of dA, [2][N][64].
template <typename T, bool PACKED>
__global__ __launch_bounds__(64) void k_scan_grad(ScanParams p)
{
    extern __shared__ float shared[];
    const int lane = threadIdx.x;
    const ScanWork w = scan_work(p, blockIdx.x);
    const int N = static_cast<int>(p.N);
    float* const gs = shared + lane;
    float* const as = shared + N * 64 + lane;
    const int64_t tiles = (p.T + kBwdTile - 1) / kBwdTile;
    const T* x = static_cast<const T*>(p.x) + w.row * p.xb + w.e;
    const T* dt = static_cast<const T*>(p.dt) + w.row * p.db + w.e;
    const T* z = p.z ? static_cast<const T*>(p.z) + w.row * p.zb + w.e : nullptr;
    const T* B = static_cast<const T*>(p.B) + w.row * p.bb + w.g * p.N;
    const T* C = static_cast<const T*>(p.C) + w.row * p.cb + w.g * p.N;
    const int64_t out = w.row * p.T * p.E + w.e;
    const T* dy = static_cast<const T*>(p.dy) + out;
    const float* A_log = p.A_log + w.e * p.N;
    const float bias = p.dt_bias ? p.dt_bias[w.e] : 0.f, D = p.D ? p.D[w.e] : 0.f;
    // the chunk's rows of dB and dC: [token][group][2][N] of this channel tile
    float* const bc = p.pBC + ((w.tile * p.b + w.row) * p.T * p.G + w.g) * 2 * p.N;
    float sumD = 0.f, sumBias = 0.f;
    {
        const float* from = p.rstates + (w.row * p.S + w.chunk) * p.N * p.E + w.e;
        for (int n = 0; n < N; ++n) {
            gs[n * 64] = w.live ? from[n * p.E] : 0.f;
            as[n * 64] = 0.f;
        }
    }
    const int place = static_cast<int>(__brev(static_cast<unsigned>(lane)) >> 26);   // the value this lane gets
    const int tok_of = kBwdTile - 1 - place / kQuad, n_of = place % kQuad;

    for (int64_t tile = (w.t1 - 1) / kBwdTile; tile * kBwdTile >= w.t0; --tile) {
        const int64_t t0 = tile * kBwdTile;
        const int count = static_cast<int>(w.t1 - t0 < kBwdTile ? w.t1 - t0 : kBwdTile);
        float d[kBwdTile], xv[kBwdTile], dyg[kBwdTile], du[kBwdTile], sa[kBwdTile], ys[kBwdTile];
        unsigned starts = 0, ends = 0;   // bits: the token starts / ends a sequence
#pragma unroll
        for (int u = 0; u < kBwdTile; ++u) {
            const int64_t at = u < count ? t0 + u : w.t1 - 1;
            xv[u] = widen(x[at * p.xt]);
            d[u] = widen(dt[at * p.dtt]);
            dyg[u] = w.live && u < count ? gated(widen(dy[at * p.E]), z, at * p.zt) : 0.f;
            du[u] = sa[u] = ys[u] = 0.f;
            if (u < count) {
                if (scan_starts<PACKED>(p, at)) starts |= 1u << u;
                if (scan_ends<PACKED>(p, at)) ends |= 1u << u;
            }
        }
#pragma unroll
        for (int u = 0; u < kBwdTile; ++u)   // (a token past the end: no decay, no input)
            d[u] = u < count ? time_step(p, d[u] + bias) : 0.f;

        for (int q = 0; q < N; q += kQuad) {
            float A2[kQuad], h[kQuad], g[kQuad], dA[kQuad];
            float hb[kBwdTile][kQuad], a[kBwdTile][kQuad];   // state before each token, its decay
            const float* m = p.marks + ((w.row * tiles + tile) * p.N + q) * p.E + w.e;
#pragma unroll
            for (int n = 0; n < kQuad; ++n) {
                A2[n] = decay_rate(A_log[q + n]);
                h[n] = m[n * p.E];
                g[n] = gs[(q + n) * 64];
                dA[n] = as[(q + n) * 64];
            }
#pragma unroll
            for (int u = 0; u < kBwdTile; ++u) {
                const int64_t at = u < count ? t0 + u : w.t1 - 1;
                if (starts >> u & 1) {
                    const int64_t unit = scan_unit<PACKED>(p, w.row, at);
#pragma unroll
                    for (int n = 0; n < kQuad; ++n) h[n] = p.init ? p.init[(unit * p.E + w.e) * p.N + q + n] : 0.f;
                }
                float b[kQuad], c[kQuad];
                uniform_row(B + at * p.bt + q, b);
                uniform_row(C + at * p.ct + q, c);
                const float in = u < count ? d[u] * xv[u] : 0.f;
#pragma unroll
                for (int n = 0; n < kQuad; ++n) {
                    a[u][n] = __builtin_amdgcn_exp2f(d[u] * A2[n]);
                    hb[u][n] = h[n];
                    h[n] = fmaf(a[u][n], h[n], in * b[n]);
                    if (p.dz) ys[u] = fmaf(h[n], c[n], ys[u]);
                }
            }
            LaneSums sB, sC;
            each<0>([&](auto i) {
                constexpr int I = decltype(i)::value, u = kBwdTile - 1 - I;
                const int64_t at = u < count ? t0 + u : w.t1 - 1;
                float b[kQuad], c[kQuad];
                uniform_row(B + at * p.bt + q, b);
                uniform_row(C + at * p.ct + q, c);
                const float in = u < count ? d[u] * xv[u] : 0.f;
                if (ends >> u & 1) {
                    const int64_t unit = scan_unit<PACKED>(p, w.row, at);
#pragma unroll
                    for (int n = 0; n < kQuad; ++n)
                        g[n] = p.dfin && w.live ? p.dfin[(unit * p.E + w.e) * p.N + q + n] : 0.f;
                }
                const auto one = [&](auto k) {
                    constexpr int n = decltype(k)::value;
                    const float hn = fmaf(a[u][n], hb[u][n], in * b[n]);   // the state after the token
                    g[n] = fmaf(dyg[u], c[n], g[n]);
                    sC.template put<I * kQuad + n>(dyg[u] * hn, lane);
                    sB.template put<I * kQuad + n>(w.live ? g[n] * in : 0.f, lane);
                    du[u] = fmaf(g[n], b[n], du[u]);
                    g[n] *= a[u][n];
                    const float e = g[n] * hb[u][n];
                    sa[u] = fmaf(e, A2[n], sa[u]);
                    dA[n] = fmaf(e, d[u], dA[n]);
                };
                one(std::integral_constant<int, 0>{});
                one(std::integral_constant<int, 1>{});
                one(std::integral_constant<int, 2>{});
                one(std::integral_constant<int, 3>{});
                if (starts >> u & 1) {
                    if (p.dinit && w.live) {
                        const int64_t unit = scan_unit<PACKED>(p, w.row, at);
#pragma unroll
                        for (int n = 0; n < kQuad; ++n) p.dinit[(unit * p.E + w.e) * p.N + q + n] = g[n];
                    }
                }
            });
            if (tok_of < count) {
                float* to = bc + (t0 + tok_of) * p.G * 2 * p.N + q + n_of;
                to[0] = sB.out;
                to[p.N] = sC.out;
            }
#pragma unroll
            for (int n = 0; n < kQuad; ++n) {
                gs[(q + n) * 64] = g[n];
                as[(q + n) * 64] = dA[n];
            }
        }
#pragma unroll
        for (int u = 0; u < kBwdTile; ++u) {
            const int64_t at = u < count ? t0 + u : w.t1 - 1, o = out + at * p.E;
            const float dx = fmaf(d[u], du[u], D * dyg[u]);
            float dd = fmaf(xv[u], du[u], sa[u] * 0.69314718f);   // (A2 is A log2(e))
            if (p.softplus) dd *= sigmoid_hw(widen(dt[at * p.dtt]) + bias);
            if (u < count) {
                sumD = fmaf(dyg[u], xv[u], sumD);
                sumBias += dd;
            }
            if (w.live && u < count) {
                static_cast<T*>(p.dx)[o] = narrow<T>(dx);
                static_cast<T*>(p.ddt)[o] = narrow<T>(dd);
                if (p.dz) {
                    const float zv = widen(z[at * p.zt]), s = sigmoid_hw(zv);
                    static_cast<T*>(p.dz)[o] = narrow<T>(widen(dy[at * p.E]) * fmaf(D, xv[u], ys[u]) * silu_grad(zv, s));
                }
            }
        }
    }
    if (!w.live) return;
    const int64_t rc = w.row * p.S + w.chunk;
    for (int n = 0; n < N; ++n) p.pA[(rc * p.N + n) * p.E + w.e] = as[n * 64];
    p.pD[rc * 2 * p.E + w.e] = sumD;
    p.pD[(rc * 2 + 1) * p.E + w.e] = sumBias;
}

// dA_log, dD and ddt_bias: sums over rows and chunks, in order.
__global__ __launch_bounds__(256) void k_scan_sum_params(ScanParams p)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, ne = p.N * p.E, parts = p.b * p.S;
    if (i < ne) {
        const int64_t n = i / p.E, e = i - n * p.E;
        float v = 0.f;
        for (int64_t k = 0; k < parts; ++k) v += p.pA[k * ne + i];
        p.dA_log[e * p.N + n] = v * -expf(p.A_log[e * p.N + n]);
        return;
    }
    const int64_t j = i - ne;
    if (j >= 2 * p.E) return;
    float* to = j < p.E ? p.dD : p.ddt_bias;
    if (!to) return;
    float v = 0.f;
    for (int64_t k = 0; k < parts; ++k) v += p.pD[k * 2 * p.E + j];
    to[j < p.E ? j : j - p.E] = v;
}

// dB and dC: sums over a group's channel tiles, in order.
template <typename T>
__global__ __launch_bounds__(256) void k_scan_sum_bc(ScanParams p, int64_t blocks)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, all = p.b * p.T * p.G * 2 * p.N;
    if (i >= all) return;
    float v = 0.f;
    for (int64_t k = 0; k < blocks; ++k) v += p.pBC[k * all + i];
    const int64_t tg = i / (2 * p.N), n = i - tg * 2 * p.N;
    T* to = static_cast<T*>(n < p.N ? p.dB : p.dC);
    to[tg * p.N + (n < p.N ? n : n - p.N)] = narrow<T>(v);
}

template <typename T, bool PACKED>
hipError_t run(const ScanParams& p, hipStream_t stream)
{
    const int64_t units = p.b * p.S * p.G * scan_tiles(p.E, p.G);
    const int64_t sums = (p.N * p.E + 2 * p.E + 255) / 256, bc = (p.b * p.T * p.G * 2 * p.N + 255) / 256;
    const int64_t pass = (p.b * p.N * p.E + 255) / 256;
    if (units > kMaxGrid || sums > kMaxGrid || bc > kMaxGrid || pass > kMaxGrid) return hipErrorInvalidConfiguration;
    const unsigned threads = 64 * static_cast<unsigned>(p.N / kSlice);
    if (p.S > 1) {
        if (hipError_t err = launch_scan_chunk_states(p, sizeof(T) == 2, false, stream); err != hipSuccess) return err;
        if (hipError_t err = launch_scan_pass(p, stream); err != hipSuccess) return err;
    }
    if (hipError_t err = launch_scan_chunk_states(p, sizeof(T) == 2, true, stream); err != hipSuccess) return err;
    hipLaunchKernelGGL((k_scan_rev<T, PACKED>), dim3(static_cast<unsigned>(units)), dim3(threads), 0, stream, p);
    hipLaunchKernelGGL(k_scan_rev_pass, dim3(static_cast<unsigned>(pass)), dim3(256), 0, stream, p);
    if (hipError_t err = hipGetLastError(); err != hipSuccess) return err;
    const size_t lds = 2 * static_cast<size_t>(p.N) * 64 * sizeof(float);
    if (lds > 65536) {   // (N > 128) beyond the default limit
        const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void*>(&k_scan_grad<T, PACKED>),
                                                   hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lds));
        if (err != hipSuccess) return err;
    }
    hipLaunchKernelGGL((k_scan_grad<T, PACKED>), dim3(static_cast<unsigned>(units)), dim3(64), lds, stream, p);
    hipLaunchKernelGGL(k_scan_sum_params, dim3(static_cast<unsigned>(sums)), dim3(256), 0, stream, p);
    hipLaunchKernelGGL((k_scan_sum_bc<T>), dim3(static_cast<unsigned>(bc)), dim3(256), 0, stream, p,
                       scan_tiles(p.E, p.G));
    return hipGetLastError();
}

}  // namespace

hipError_t launch_scan_backward(const ScanParams& p, bool bf16, hipStream_t stream)
{
    if (bf16) return p.seq_idx ? run<uint16_t, true>(p, stream) : run<uint16_t, false>(p, stream);
    return p.seq_idx ? run<float, true>(p, stream) : run<float, false>(p, stream);
}

}  // namespace ssd
