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
// zero, also in front of every tile of 8 tokens, and the gradients of the states
// entering them, from zero too (one pass, k_scan_chunk<kBoth>), a scan over the
// chunks in each direction, then k_scan_grad, which takes its chunk's tiles in
// reverse: the state in front of a tile is the one kept for it and what is left of
// the one entering the chunk; four states at a time, a tile's states
// are computed again from its entering ones and kept, with the decays, in
// registers, and then walked back.  The sums over channels for dB and dC run across
// the lanes: the tile's 64 values of four states, one after the other, are merged in a tree in which every
// level halves the lanes that a value is spread over, two instructions a value
// where a sum of its own would take seven.  Sums over channel tiles, chunks and
// rows are joined in a fixed order by k_scan_sum_params and k_scan_sum_bc.
//
// Bound by vector arithmetic, like the forward: 8 x 2,048 x 1,536 bf16 with a gate 546
// us, of which k_scan_grad 404, where the vector units are busy 72 % of the time (two
// wavefronts a SIMD: a tile's states and decays fill the registers), k_scan_chunk<kBoth>
// 131.  The scalars do not fit their registers either (row pointers, B and C of a tile's
// tokens): of 3,290 vector instructions a tile 240 move them to and from lanes.  For
// packed rows, where every tile asks for sequence edges, the round of four states has
// 1,468 instructions, 299 of those moves, instead of 660: 1 x 16,384 tokens x 1,536 868
// us, k_scan_grad 490 and the scans over chunks 203 (not packed 597).  The states of
// every token written out by the first pass and read again, in place of computing them
// twice, would move 3.2 GB (8 x 2,048 x 1,536), 630 us at a copy's rate.
#include <type_traits>

#include "ssd_internal.h"
#include "ssd_scan.h"

namespace ssd {
namespace {

__device__ __forceinline__ float silu_grad(float z, float s) { return s * fmaf(z, 1.f - s, 1.f); }

constexpr int kPassBatch = 16;

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
    for (int64_t c = p.S - 1; c >= 0; c -= kPassBatch) {
        float own[kPassBatch], d[kPassBatch];
#pragma unroll
        for (int k = 0; k < kPassBatch; ++k) {
            const int64_t at = c - k > 0 ? c - k : 0;
            own[k] = st[at * step];
            d[k] = p.sums[(row * p.S + at) * p.E + e];
        }
#pragma unroll
        for (int k = 0; k < kPassBatch; ++k) {
            const int64_t at = c - k;
            if (at < 0) continue;
            st[at * step] = g;
            const float half = __builtin_amdgcn_exp2f(d[k] * A2 * 0.5f);
            const float through = g * half * half;
            const int64_t t0 = at * p.L, t1 = t0 + p.L < p.T ? t0 + p.L : p.T;
            // (a sequence that ends in the chunk, its last token included, takes nothing from behind it)
            const bool joined = t1 < p.T && (!p.seq_idx || (p.seq_idx[t0] == p.seq_idx[t1 - 1] &&
                                                            p.seq_idx[t1 - 1] == p.seq_idx[t1]));
            g = joined ? own[k] + through : own[k];
        }
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

template <int I, int END, typename F>
__device__ __forceinline__ void each(F&& f)
{
    if constexpr (I < END) {
        f(std::integral_constant<int, I>{});
        each<I + 1, END>(f);
    }
}

constexpr int kQuad = 4;   // states taken at a time

constexpr int kHalf = kBwdTile / 2;

// B and C of half a tile's tokens, four states each.
template <typename T>
struct QuadRows {
    Uniform<T, kQuad> b[kHalf], c[kHalf];

    // from the rows' places on, at most `left` of them (then the last one again)
    __device__ __forceinline__ void load(Rows<const T> B, Rows<const T> C, int left)
    {
#pragma unroll
        for (int i = 0; i < kHalf; ++i) {
            b[i].load(B);
            c[i].load(C);
            B.move(i + 1 < left);
            C.move(i + 1 < left);
        }
    }
    __device__ __forceinline__ void arrive()
    {
#pragma unroll
        for (int i = 0; i < kHalf; ++i) {
            b[i].arrive();
            c[i].arrive();
        }
    }
};

template <bool FIRST, typename R>
__device__ __forceinline__ const R& half(const R& lo, const R& hi)
{
    if constexpr (FIRST)
        return lo;
    else
        return hi;
}

// A tile of k_scan_grad (FULL: all its kBwdTile tokens are real; PARTIAL: a group's
// last channel tile may have lanes without a channel, which add zeros to the sums
// over channels); adds to the channel's sums of dD and ddt_bias.
template <typename T, bool PACKED, bool GATE, bool PARTIAL, bool FULL>
__device__ __forceinline__ void grad_tile(const ScanParams& p, const ScanWork& w, int64_t tile, float* gs, float* as,
                                          float* extra, float bias, float D, float& sumD, float& sumBias)
{
    const bool live = !PARTIAL || w.live;
    const int lane = threadIdx.x, N = static_cast<int>(p.N);
    const int64_t t0 = tile * kBwdTile, out = (w.row * p.T + t0) * p.E + w.e0;
    const int64_t tiles = (p.T + kBwdTile - 1) / kBwdTile;
    const int count = FULL ? kBwdTile : static_cast<int>(w.t1 - t0);
    float d[kBwdTile], xv[kBwdTile], dyg[kBwdTile], du[kBwdTile], sa[kBwdTile], ys[kBwdTile];
    // wanted again at the tile's end only, in shared memory meanwhile: the derivative of
    // dt by dt_in, and dy silu'(z)
    float* const slope = extra + lane;
    float* const zd = slope + kBwdTile * 64;
    unsigned starts = 0, ends = 0;   // bits (packed rows): the token starts / ends a sequence
    {
        Rows<const T> x(p.x, w.row * p.xb + t0 * p.xt + w.e0, p.xt);
        Rows<const T> dt(p.dt, w.row * p.db + t0 * p.dtt + w.e0, p.dtt);
        Rows<const T> z(GATE ? p.z : p.x, GATE ? w.row * p.zb + t0 * p.zt + w.e0 : 0, GATE ? p.zt : 0);
        Rows<const T> dy(p.dy, out, p.E);
        T xr[kBwdTile], dr[kBwdTile], yr[kBwdTile], zr[kBwdTile];
        const unsigned off = lane_offset<T>(w.lane);
#pragma unroll
        for (int u = 0; u < kBwdTile; ++u) {
            xr[u] = x.get(off);
            dr[u] = dt.get(off);
            yr[u] = dy.get(off);
            if (GATE) zr[u] = z.get(off);
            const bool more = FULL || u + 1 < count;   // (at the end: the last token again)
            if (u + 1 == kBwdTile) break;
            x.move(more);
            dt.move(more);
            dy.move(more);
            if (GATE) z.move(more);
        }
#pragma unroll
        for (int u = 0; u < kBwdTile; ++u) {
            xv[u] = widen(xr[u]);
            const float v = widen(dr[u]) + bias, dyv = live ? widen(yr[u]) : 0.f;
            d[u] = v;
            if (p.softplus) {
                const float e = exp_neg<false>(fabsf(v));
                d[u] = softplus_hw(v, e);
                slope[u * 64] = (v >= 0.f ? 1.f : e) * __builtin_amdgcn_rcpf(1.f + e);
            }
            dyg[u] = dyv;
            if (GATE) {
                const float zv = widen(zr[u]), s = sigmoid_hw(zv);
                dyg[u] = dyv * zv * s;
                zd[u * 64] = dyv * silu_grad(zv, s);
            }
            du[u] = sa[u] = ys[u] = 0.f;
            if (PACKED && (FULL || u < count)) {
                if (scan_starts<PACKED>(p, t0 + u)) starts |= 1u << u;
                if (scan_ends<PACKED>(p, t0 + u)) ends |= 1u << u;
            }
        }
    }
    Rows<const T> B0(p.B, w.row * p.bb + t0 * p.bt + w.g * p.N, p.bt), B1 = B0;
    Rows<const T> C0(p.C, w.row * p.cb + t0 * p.ct + w.g * p.N, p.ct), C1 = C0;
    const bool second = FULL || count > kHalf;   // there are tokens in the tile's second half
    B1.p += second ? static_cast<int64_t>(kHalf) * p.bt : 0;
    C1.p += second ? static_cast<int64_t>(kHalf) * p.ct : 0;
    running(B1.p);
    running(C1.p);
    const int left0 = FULL ? kHalf : count, left1 = FULL ? kHalf : second ? count - kHalf : 1;
    Rows<const float> m(p.marks, (w.row * tiles + tile) * p.N * p.E + w.e0, p.E);
    Rows<const float> entering(p.states, (w.row * p.S + w.chunk) * p.N * p.E + w.e0, p.E);
    const float* A_log = p.A_log + w.e * p.N;
    // whether the state entering the chunk reaches the tile (no sequence starts in between)
    bool reached = w.chunk > 0;
    if (PACKED && reached)
        reached = !scan_starts<PACKED>(p, w.t0) &&
                  scalar_load(p.seq_idx + w.t0) == scalar_load(p.seq_idx + (t0 > w.t0 ? t0 - 1 : t0));
    // (it runs on over sequences: where it is not of the tile's own one alone, it is not used)
    const float since = reached ? p.marksums[(w.row * tiles + tile) * p.E + w.e] : 0.f;
    // the value that this lane gets of the 64: token, dB or dC, state
    const int place = static_cast<int>(__brev(static_cast<unsigned>(lane)) >> 26);
    const int tok = kBwdTile - 1 - place / (2 * kQuad);
    float* to = p.pBC + (((w.tile * p.b + w.row) * p.T + t0 + tok) * p.G + w.g) * 2 * p.N +
                (place / kQuad % 2) * p.N + place % kQuad;

    // a round's own values, loaded a round ahead
    float4 al;
    float mn[kQuad], en[kQuad] = {};
    const auto ahead = [&](int q) {
        unsigned off = lane_offset<float>(w.lane);
        al = *reinterpret_cast<const float4*>(A_log + q);
#pragma unroll
        for (int n = 0; n < kQuad; ++n) {
            mn[n] = m.get(off);
            m.move();
        }
        if (reached) {
            off = lane_offset<float>(w.lane);
#pragma unroll
            for (int n = 0; n < kQuad; ++n) {
                en[n] = entering.get(off);
                entering.move();
            }
        }
    };
    ahead(0);
    for (int q = 0; q < N; q += kQuad) {
        float A2[kQuad], h[kQuad], g[kQuad], dA[kQuad];
        float hb[kBwdTile][kQuad], a[kBwdTile][kQuad];   // state before each token, its decay
        QuadRows<T> lo, hi;
        lo.load(B0, C0, left0);
        A2[0] = decay_rate(al.x);
        A2[1] = decay_rate(al.y);
        A2[2] = decay_rate(al.z);
        A2[3] = decay_rate(al.w);
#pragma unroll
        for (int n = 0; n < kQuad; ++n) {
            // (nothing reaches the tile: 0 times 1)
            h[n] = fmaf(__builtin_amdgcn_exp2f(since * A2[n]), en[n], mn[n]);
            g[n] = gs[(q + n) * 64];
            dA[n] = as[(q + n) * 64];
        }
        if (q + kQuad < N) ahead(q + kQuad);
        lo.arrive();
        hi.load(B1, C1, left1);
        __builtin_amdgcn_sched_barrier(0);
        each<0, kBwdTile>([&](auto i) {
            constexpr int u = decltype(i)::value, k = u % kHalf;
            if constexpr (u == kHalf) hi.arrive();
            if (!FULL && u >= count) return;
            if (PACKED && (starts >> u & 1)) {
                const int64_t unit = scan_unit<PACKED>(p, w.row, t0 + u);
#pragma unroll
                for (int n = 0; n < kQuad; ++n) h[n] = p.init ? p.init[(unit * p.E + w.e) * p.N + q + n] : 0.f;
            }
            const Uniform<T, kQuad>&b = half<(u < kHalf)>(lo, hi).b[k], &c = half<(u < kHalf)>(lo, hi).c[k];
            const float in = d[u] * xv[u];
#pragma unroll
            for (int n = 0; n < kQuad; ++n) {
                a[u][n] = __builtin_amdgcn_exp2f(d[u] * A2[n]);
                hb[u][n] = h[n];
                h[n] = fmaf(a[u][n], h[n], in * b[n]);
                if (GATE) ys[u] = fmaf(h[n], c[n], ys[u]);
            }
        });
        // a sequence's last token: g is the final state's gradient; its first one: g is
        // the initial state's
        const auto leave = [&](int u) {
            const int64_t unit = scan_unit<PACKED>(p, w.row, t0 + u);
#pragma unroll
            for (int n = 0; n < kQuad; ++n)
                g[n] = p.dfin && live ? p.dfin[(unit * p.E + w.e) * p.N + q + n] : 0.f;
        };
        const auto arrive = [&](int u) {
            if (!p.dinit || !live) return;
            const int64_t unit = scan_unit<PACKED>(p, w.row, t0 + u);
#pragma unroll
            for (int n = 0; n < kQuad; ++n) p.dinit[(unit * p.E + w.e) * p.N + q + n] = g[n];
        };
        if (!PACKED && t0 + count == p.T) leave(count - 1);
        LaneSums sums;
        lo.load(B0, C0, left0);   // (again, for the way back)
        __builtin_amdgcn_sched_barrier(0);
        each<0, kBwdTile>([&](auto i) {
            constexpr int I = decltype(i)::value, u = kBwdTile - 1 - I;
            constexpr int first = I * 2 * kQuad, k = u % kHalf;
            if constexpr (u == kHalf - 1) lo.arrive();
            // the token's products for dB and dC (one place of the tree each; a token past
            // the end puts zeros)
            float products[2 * kQuad] = {};
            if (FULL || u < count) {
                const Uniform<T, kQuad>&b = half<(u < kHalf)>(lo, hi).b[k], &c = half<(u < kHalf)>(lo, hi).c[k];
                const float in = d[u] * xv[u];
                if (PACKED && (ends >> u & 1)) leave(u);
#pragma unroll
                for (int n = 0; n < kQuad; ++n) {
                    g[n] = fmaf(dyg[u], c[n], g[n]);
                    du[u] = fmaf(g[n], b[n], du[u]);
                    products[n] = g[n] * in;
                    // the state after the token: that before the next one, if no sequence starts there
                    float after;
                    if constexpr (PACKED || !FULL)
                        after = fmaf(a[u][n], hb[u][n], in * b[n]);
                    else
                        after = u + 1 < kBwdTile ? hb[u + 1 < kBwdTile ? u + 1 : u][n] : h[n];
                    products[kQuad + n] = dyg[u] * after;
                    g[n] *= a[u][n];
                    const float e = g[n] * hb[u][n];
                    sa[u] = fmaf(e, A2[n], sa[u]);
                    dA[n] = fmaf(e, d[u], dA[n]);
                }
                if (PACKED && (starts >> u & 1)) arrive(u);
            }
            each<0, 2 * kQuad>([&](auto n) {
                constexpr int k = decltype(n)::value;
                sums.template put<first + k>(live ? products[k] : 0.f, lane);
            });
        });
        if (!PACKED && t0 == 0) arrive(0);
        if (FULL || tok < count) *to = sums.out;
#pragma unroll
        for (int n = 0; n < kQuad; ++n) {
            gs[(q + n) * 64] = g[n];
            as[(q + n) * 64] = dA[n];
        }
        to += kQuad;
        B0.p += kQuad;
        C0.p += kQuad;
        B1.p += kQuad;
        C1.p += kQuad;
    }

    Rows<T> dx(p.dx, out, p.E), ddt(p.ddt, out, p.E), dz(GATE ? p.dz : p.dx, out, p.E);
#pragma unroll
    for (int u = 0; u < kBwdTile; ++u) {
        if (FULL || u < count) {
            float dd = fmaf(xv[u], du[u], sa[u] * 0.69314718f);   // (A2 is A log2(e))
            if (p.softplus) dd *= slope[u * 64];
            sumD = fmaf(dyg[u], xv[u], sumD);
            sumBias += dd;
            if (live) {
                const unsigned off = lane_offset<T>(w.lane);
                dx.put(off, narrow<T>(fmaf(d[u], du[u], D * dyg[u])));
                ddt.put(off, narrow<T>(dd));
                if (GATE) dz.put(off, narrow<T>(zd[u * 64] * fmaf(D, xv[u], ys[u])));
            }
            dx.move();
            ddt.move();
            if (GATE) dz.move();
        }
    }
}

// One wavefront: 64 channels of one chunk, its tiles from the last to the first.
// Shared memory: the states' running gradients g and sums of dA, [2][N][64], and two
// values of each of the tile's tokens, [2][kBwdTile][64].
template <typename T, bool PACKED, bool GATE, bool PARTIAL>
__global__ __launch_bounds__(64, 2) void k_scan_grad(ScanParams p)
{
    extern __shared__ float shared[];
    const int lane = threadIdx.x, N = static_cast<int>(p.N);
    const ScanWork w = scan_work(p, blockIdx.x);
    const bool live = !PARTIAL || w.live;
    float* const gs = shared + lane;
    float* const as = shared + N * 64 + lane;
    float* const extra = shared + 2 * N * 64;
    const float bias = p.dt_bias ? p.dt_bias[w.e] : 0.f, D = p.D ? p.D[w.e] : 0.f;
    float sumD = 0.f, sumBias = 0.f;
    const float* from = p.rstates + (w.row * p.S + w.chunk) * p.N * p.E + w.e;
    for (int n = 0; n < N; ++n) {
        gs[n * 64] = live && p.S > 1 ? from[n * p.E] : 0.f;
        as[n * 64] = 0.f;
    }
    int64_t tile = (w.t1 - 1) / kBwdTile;
    if (w.t1 - tile * kBwdTile < kBwdTile) {
        grad_tile<T, PACKED, GATE, PARTIAL, false>(p, w, tile, gs, as, extra, bias, D, sumD, sumBias);
        --tile;
    }
    for (; tile * kBwdTile >= w.t0; --tile)
        grad_tile<T, PACKED, GATE, PARTIAL, true>(p, w, tile, gs, as, extra, bias, D, sumD, sumBias);
    if (!live) return;
    const int64_t rc = w.row * p.S + w.chunk;
    for (int n = 0; n < N; ++n) p.pA[(rc * p.N + n) * p.E + w.e] = as[n * 64];
    p.pD[rc * 2 * p.E + w.e] = sumD;
    p.pD[(rc * 2 + 1) * p.E + w.e] = sumBias;
}

// dA_log, dD and ddt_bias: sums over rows and chunks, in a fixed order.
__global__ __launch_bounds__(kSumLanes * kSumCols) void k_scan_sum_params(ScanParams p)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kSumCols + threadIdx.x % kSumCols;
    const int64_t ne = p.N * p.E, all = ne + 2 * p.E;
    const bool first = i < ne;   // a column of dA, else one of dD or ddt_bias
    const float v = column_sum(first ? p.pA + i : p.pD + (i - ne), p.b * p.S, first ? ne : 2 * p.E, i < all);
    if (threadIdx.x >= kSumCols || i >= all) return;
    if (first) {
        const int64_t n = i / p.E, e = i - n * p.E;
        p.dA_log[e * p.N + n] = v * (decay_rate(p.A_log[e * p.N + n]) * 0.69314718f);
        return;
    }
    const int64_t j = i - ne;
    float* to = j < p.E ? p.dD : p.ddt_bias;
    if (to) to[j < p.E ? j : j - p.E] = v;
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

template <typename T, bool PACKED, bool GATE, bool PARTIAL>
hipError_t grad(const ScanParams& p, int64_t units, hipStream_t stream)
{
    const size_t lds = 2 * static_cast<size_t>(p.N + kBwdTile) * 64 * sizeof(float);
    if (lds > 65536) {   // (N > 120) beyond the default limit
        const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void*>(&k_scan_grad<T, PACKED, GATE, PARTIAL>),
                                                   hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lds));
        if (err != hipSuccess) return err;
    }
    hipLaunchKernelGGL((k_scan_grad<T, PACKED, GATE, PARTIAL>), dim3(static_cast<unsigned>(units)), dim3(64), lds, stream, p);
    return hipGetLastError();
}

template <typename T, bool PACKED>
hipError_t grads(const ScanParams& p, int64_t units, hipStream_t stream)
{
    const bool partial = p.E / p.G % 64 != 0;
    if (p.z) return partial ? grad<T, PACKED, true, true>(p, units, stream) : grad<T, PACKED, true, false>(p, units, stream);
    return partial ? grad<T, PACKED, false, true>(p, units, stream) : grad<T, PACKED, false, false>(p, units, stream);
}

template <typename T, bool PACKED>
hipError_t run(const ScanParams& p, hipStream_t stream)
{
    const int64_t units = p.b * p.S * p.G * scan_tiles(p.E, p.G);
    const int64_t sums = (p.N * p.E + 2 * p.E + kSumCols - 1) / kSumCols, bc = (p.b * p.T * p.G * 2 * p.N + 255) / 256;
    const int64_t pass = (p.b * p.N * p.E + 255) / 256;
    if (!scan_fits(p) || !fits(sums, kSumLanes * kSumCols) || !fits(bc, 256)) return hipErrorInvalidConfiguration;
    if (hipError_t err = launch_scan_both(p, sizeof(T) == 2, stream); err != hipSuccess) return err;
    if (p.S > 1) {
        if (hipError_t err = launch_scan_pass(p, stream); err != hipSuccess) return err;
        hipLaunchKernelGGL(k_scan_rev_pass, dim3(static_cast<unsigned>(pass)), dim3(256), 0, stream, p);
    }
    if (hipError_t err = grads<T, PACKED>(p, units, stream); err != hipSuccess) return err;
    hipLaunchKernelGGL(k_scan_sum_params, dim3(static_cast<unsigned>(sums)), dim3(kSumLanes * kSumCols), 0, stream, p);
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
