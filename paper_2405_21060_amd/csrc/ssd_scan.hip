// The selective scan of the first kind of block: forward and the single-token
// step.
//
//     h_t = exp(dt_t A) h_{t-1} + dt_t x_t B_t,   y_t = h_t . C_t + D x_t,   y_t *= silu(z_t)
//
// per channel e with N states n of its own decay A_e,n.  Per (token, channel,
// state): a product and exp2 for the decay, a product for the input, a multiply-
// add for the state and one for the output -- bound by vector arithmetic (six
// issue slots; the matrix cores cannot take a product whose factor differs for
// every element), not by HBM.
//
// The recurrence runs over tokens in registers (ssd_scan.h).  Where the channel
// tiles alone do not fill the device, the tokens are cut into chunks of L: their
// states from zero (k_scan_chunk<kStates>), a scan over the chunks
// (k_scan_pass), then the outputs from each chunk's entering state
// (k_scan_chunk<kOutputReady>); the first of the three costs five more slots.
// Sequences of a packed row replace the state at their first token.
//
// Measured (bf16, gate): 4 x 4,096 x 5,120 508 us, the output pass 300 of them, the
// states 240 (traced alone each a little slower); one pass over the tokens needs
// 205 at one slot a cycle and 2.4 GHz, its bytes 132.  1 x 65,536 x 1,536 646 us
// (351, 281 and 57 for the scan over 410 chunks, each alone).  The vector units are busy
// 98 % of the chunk kernels' time.
#include <type_traits>

#include "ssd_internal.h"
#include "ssd_scan.h"

namespace ssd {
namespace {

enum Mode { kOutput, kOutputReady, kStates, kBoth };

// kOutput: y and final states.  kStates: each chunk's state from zero (from the
// initial state in the first one), its sum of dt, and the time steps themselves,
// which kOutputReady then takes as they are (97 instructions a token where kOutput
// has 111).  For the gradients, kBoth: the states, the gradient of the state entering
// each chunk from the chunk's own outputs, sum_t exp(A sum_{s <= t} dt_s) dy~_t C_t
// (walked forwards too, the product of the decays so far kept: one exp2 serves
// both), and in front of every tile of kBwdTile tokens the state, from zero as it
// is, and the sum of dt since the chunk's start.
// Workgroup: a wavefront per 16 states, at most THREADS / 64 of them (the bound
// says how many registers a lane may have; with more than 64 states kBoth does not fit
// them, up to 45 values of a lane are in scratch memory).
//
// A tile is kTok tokens; the next one's are loaded, and its B and C a token ahead,
// before they are needed.  With several wavefronts their shares of y meet in shared
// memory, and wavefront k finishes every token u = k, k + slices, ..
template <typename T, bool PACKED, bool GATE, Mode MODE, int THREADS>
__global__ __launch_bounds__(THREADS) void k_scan_chunk(ScanParams p)
{
    extern __shared__ float shared[];   // outputs with several wavefronts: [2][kTok][slices][64]
    constexpr bool kOne = THREADS == 64, kReady = MODE == kOutputReady, kOut = MODE == kOutput || kReady;
    constexpr bool kBack = MODE == kBoth;
    const int slice = kOne ? 0 : uniform(threadIdx.x >> 6);
    const int slices = kOne ? 1 : static_cast<int>(p.N / kSlice);
    const unsigned col = threadIdx.x & 63;
    const ScanWork w = scan_work(p, blockIdx.x);
    const int n0 = slice * kSlice;
    Rows<const T> x(p.x, w.row * p.xb + w.t0 * p.xt + w.e0, p.xt);
    Rows<const T> dt(p.dt, w.row * p.db + w.t0 * p.dtt + w.e0, p.dtt);
    Rows<const T> z(GATE ? p.z : p.x, GATE ? w.row * p.zb + w.t0 * p.zt + w.e0 : 0, GATE ? p.zt : 0);
    Rows<const T> B(p.B, w.row * p.bb + w.t0 * p.bt + w.g * p.N + n0, p.bt);
    Rows<const T> C(p.C, w.row * p.cb + w.t0 * p.ct + w.g * p.N + n0, p.ct);
    const int64_t out = (w.row * p.T + w.t0) * p.E + w.e0;
    Rows<T> y(p.y, out, p.E);
    Rows<const T> dy(kBack ? p.dy : p.x, kBack ? out : 0, kBack ? p.E : 0);
    Rows<float> steps(p.steps, out, p.E);
    float A2[kSlice], h[kSlice];
    float cum[kSlice], r[kSlice];   // kBoth: decay since the chunk's start, gradient so far
#pragma unroll
    for (int n = 0; n < kSlice; ++n) {
        cum[n] = 1.f;
        r[n] = 0.f;
    }
    load_states(p.A_log, p, 0, w.e, n0, A2);   // (E, N): the layout of one unit
#pragma unroll
    for (int n = 0; n < kSlice; ++n) A2[n] = decay_rate(A2[n]);
    const float bias = p.dt_bias ? p.dt_bias[w.e] : 0.f;
    const float D = kOut && p.D ? p.D[w.e] : 0.f;
    int64_t unit = scan_unit<PACKED>(p, w.row, w.t0);
    float* const st = p.states + ((w.row * p.S + w.chunk) * p.N + n0) * p.E + w.e;
    if (w.chunk == 0) {
        load_states(p.init, p, unit, w.e, n0, h);
    } else if (MODE == kStates || kBack) {
#pragma unroll
        for (int n = 0; n < kSlice; ++n) h[n] = 0.f;
    } else {
#pragma unroll
        for (int n = 0; n < kSlice; ++n) h[n] = st[n * p.E];
    }
    float sum = 0.f;

    const int count = static_cast<int>(w.t1 - w.t0);
    int ahead = 0;   // the token that the pointers of x, dt and z are at
    T xr[kTok], zr[kTok] = {}, yr[kTok];
    std::conditional_t<kReady, float, T> dr[kTok];
    const auto fetch = [&]() __attribute__((always_inline)) {
        const unsigned off = lane_offset<T>(w.lane), off4 = lane_offset<float>(w.lane);
#pragma unroll
        for (int u = 0; u < kTok; ++u) {
            xr[u] = x.get(off);
            if constexpr (kReady)
                dr[u] = steps.get(off4);
            else
                dr[u] = dt.get(off);
            if (GATE) zr[u] = z.get(off);
            if (kBack) yr[u] = dy.get(off);
            const bool more = ++ahead < count;   // (at the end: the last token again)
            x.move(more);
            if constexpr (kReady)
                steps.move(more);
            else
                dt.move(more);
            if (GATE) z.move(more);
            if (kBack) dy.move(more);
        }
    };
    fetch();
    Uniform<T, kSlice> bn, cn;   // the next token's B and C
    bn.load(B);
    if (kOut || kBack) cn.load(C);
    // kBoth: the unit's sequence ends here; its final state's gradient counts too.
    bool open = true;   // no sequence has ended in the chunk yet
    const auto leave = [&]() __attribute__((always_inline)) {
        if (!open) return;
        open = false;
        float f[kSlice];
        load_states(p.dfin, p, unit, w.e, n0, f);
#pragma unroll
        for (int n = 0; n < kSlice; ++n) r[n] = fmaf(cum[n], f[n], r[n]);
    };
    float* part = shared;
    // A tile from token t of the chunk on; FULL: all of its tokens are the chunk's.
    const auto tile = [&](int t, auto full) __attribute__((always_inline)) {
        constexpr bool FULL = decltype(full)::value;
        static_assert(kTok == kBwdTile, "a mark in front of every tile");
        if (kBack && w.live) {
            const int64_t at = w.row * ((p.T + kBwdTile - 1) / kBwdTile) + (w.t0 + t) / kBwdTile;
            float* m = p.marks + (at * p.N + n0) * p.E + w.e;
#pragma unroll
            for (int n = 0; n < kSlice; ++n) m[n * p.E] = h[n];
            if (slice == 0) p.marksums[at * p.E + w.e] = sum;
        }
        float xv[kTok], d[kTok], zv[kTok], dyg[kTok];
#pragma unroll
        for (int u = 0; u < kTok; ++u) {
            xv[u] = widen(xr[u]);
            zv[u] = GATE ? widen(zr[u]) : 0.f;
            if (kBack) dyg[u] = GATE ? widen(yr[u]) * zv[u] * sigmoid_hw(zv[u]) : widen(yr[u]);
        }
#pragma unroll
        for (int u = 0; u < kTok; ++u) d[u] = kReady ? widen(dr[u]) : widen(dr[u]) + bias;
        if (!kReady && p.softplus) {
#pragma unroll
            for (int u = 0; u < kTok; ++u) d[u] = softplus_hw(d[u]);
        }
        fetch();   // the next tile's
        const unsigned off = lane_offset<T>(w.lane), off4 = lane_offset<float>(w.lane);
#pragma unroll
        for (int u = 0; u < kTok; ++u) {
            if (!FULL && t + u >= count) break;
            if (PACKED) {
                if (w.t0 + t + u > 0 && scan_starts<PACKED>(p, w.t0 + t + u)) {
                    // (from the first start behind the chunk's first token on, nothing
                    // reaches back to the state entering it)
                    if (kBack && t + u > 0) leave();
                    unit = scan_unit<PACKED>(p, w.row, w.t0 + t + u);
                    load_states(p.init, p, unit, w.e, n0, h);
                }
            }
            const float in = d[u] * xv[u];
            Uniform<T, kSlice> b = bn, c = cn;
            b.arrive();
            if (kOut || kBack) c.arrive();
            const bool more = t + u + 1 < count;
            B.move(more);
            bn.load(B);
            if (kOut || kBack) {
                C.move(more);
                cn.load(C);
            }
            __builtin_amdgcn_sched_barrier(0);   // the loads stay in front of the token's arithmetic
            if (MODE == kStates || kBack) sum += d[u];
            if (MODE == kStates && slice == 0) {   // (a lane past its group's end: the last one's value again)
                steps.put(off4, d[u]);
                steps.move();
            }
            float ys[2] = {0.f, 0.f};
#pragma unroll
            for (int n = 0; n < kSlice; ++n) {
                const float a = __builtin_amdgcn_exp2f(d[u] * A2[n]);
                h[n] = fmaf(a, h[n], in * b[n]);
                if (kOut) ys[n % 2] = fmaf(h[n], c[n], ys[n % 2]);
                if (kBack && (!PACKED || open)) {
                    cum[n] *= a;
                    r[n] = fmaf(cum[n], dyg[u] * c[n], r[n]);
                }
            }
            if (kOut) {
                if (PACKED && p.fin && w.live && scan_ends<PACKED>(p, w.t0 + t + u))
                    store_states(p.fin, p, unit, w.e, n0, h);
                if (kOne) {
                    float v = fmaf(D, xv[u], ys[0] + ys[1]);
                    if (GATE) v *= zv[u] * sigmoid_hw(zv[u]);
                    y.put(off, narrow<T>(v));   // (so is y)
                    y.move();
                } else {
                    part[(u * slices + slice) * 64 + col] = ys[0] + ys[1];
                }
            }
        }
        if (kOut && !kOne) {
            __syncthreads();
#pragma unroll
            for (int u = 0; u < kTok; ++u) {
                if (!FULL && t + u >= count) break;
                if (u % slices == slice) {
                    float v = 0.f;
                    for (int k = 0; k < slices; ++k) v += part[(u * slices + k) * 64 + col];
                    v = fmaf(D, xv[u], v);
                    if (GATE) v *= zv[u] * sigmoid_hw(zv[u]);
                    y.put(lane_offset<T>(w.lane), narrow<T>(v));
                }
                y.move();
            }
            // (the other half is written next, so one barrier a tile is enough)
            part = part == shared ? shared + kTok * slices * 64 : shared;
        }
    };
    int t = 0;
    for (; t + kTok <= count; t += kTok) tile(t, std::true_type{});
    if (t < count) tile(t, std::false_type{});
    if (kOut && !PACKED && p.fin && w.live && w.t1 == p.T) store_states(p.fin, p, unit, w.e, n0, h);
    if (kBack && scan_ends<PACKED>(p, w.t1 - 1)) leave();
    if ((MODE == kStates || kBack) && w.live && p.S > 1) {
        float* const rs = p.rstates + (st - p.states);
#pragma unroll
        for (int n = 0; n < kSlice; ++n) {
            st[n * p.E] = h[n];
            if (kBack) rs[n * p.E] = r[n];
        }
        if (slice == 0) p.sums[(w.row * p.S + w.chunk) * p.E + w.e] = sum;
    }
}

// The scan over chunks: the states of each chunk (from zero) become the states
// entering it.  A thread per batch row, state and channel.
constexpr int kPassBatch = 16;

__global__ __launch_bounds__(256) void k_scan_pass(ScanParams p)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= p.b * p.N * p.E) return;
    const int64_t e = i % p.E, rn = i / p.E, n = rn % p.N, row = rn / p.N;
    const float A2 = decay_rate(p.A_log[e * p.N + n]);
    float* st = p.states + (row * p.S * p.N + n) * p.E + e;
    const float* sums = p.sums + row * p.S * p.E + e;
    const int64_t step = p.N * p.E;
    float h = st[0];
    for (int64_t c = 1; c < p.S; c += kPassBatch) {
        float s[kPassBatch], d[kPassBatch];
#pragma unroll
        for (int k = 0; k < kPassBatch; ++k) {
            const int64_t at = c + k < p.S - 1 ? c + k : 0;   // (the last chunk's own state is not needed)
            s[k] = st[at * step];
            d[k] = sums[at * p.E];
        }
#pragma unroll
        for (int k = 0; k < kPassBatch; ++k) {
            if (c + k >= p.S) break;
            st[(c + k) * step] = h;
            // the decay in two halves, so that one below 2^-126 still counts
            const float half = __builtin_amdgcn_exp2f(d[k] * A2 * 0.5f);
            h = fmaf(h * half, half, s[k]);
            if (p.seq_idx) {
                const int64_t t0 = (c + k) * p.L, t1 = t0 + p.L < p.T ? t0 + p.L : p.T;
                if (p.seq_idx[t0 - 1] != p.seq_idx[t1 - 1]) h = s[k];   // a sequence starts in the chunk
            }
        }
    }
}

// One token per batch row.  Memory-bound: the state is read and written once.  A
// thread owns 4 consecutive states (16 bytes) of ROWS batch rows, the N / 4 threads
// of a channel are a power-of-two segment of a wavefront.  Several rows a thread
// share A and have their loads in flight together.  256 rows x 5,120 channels bf16
// 41 us with the tensors from HBM (35 at a copy's rate).
template <typename T, int ROWS>
__global__ __launch_bounds__(256) void k_scan_step(ScanParams p, int seg, int log2seg)
{
    const int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) >> log2seg;
    const int n0 = 4 * (threadIdx.x & (seg - 1));
    const int64_t block = i / p.E, e = i - block * p.E, row0 = block * ROWS;
    const bool live = row0 < p.b && n0 < p.N;
    typedef float f4 __attribute__((ext_vector_type(4)));
    float sum[ROWS] = {}, xv[ROWS] = {};
    if (live) {
        const int64_t g = e / (p.E / p.G);
        const T* B = static_cast<const T*>(p.B) + g * p.N + n0;
        const T* C = static_cast<const T*>(p.C) + g * p.N + n0;
        const T* x = static_cast<const T*>(p.x) + e;
        const T* dt = static_cast<const T*>(p.dt) + e;
        f4 st[ROWS];
        Pack<T, 4> b[ROWS], c[ROWS];
        float d[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int64_t row = row0 + r < p.b ? row0 + r : p.b - 1;
            st[r] = *reinterpret_cast<const f4*>(p.fin + (row * p.E + e) * p.N + n0);
            xv[r] = widen(x[row * p.xb]);
            d[r] = widen(dt[row * p.db]);
            b[r] = Pack<T, 4>::load(B + row * p.bb);
            c[r] = Pack<T, 4>::load(C + row * p.cb);
        }
        const auto a = Pack<float, 4>::load(p.A_log + e * p.N + n0);
        const float bias = p.dt_bias ? p.dt_bias[e] : 0.f;
        float A2[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) A2[k] = decay_rate(a[k]);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const float dv = time_step(p, d[r] + bias), in = dv * xv[r];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                st[r][k] = fmaf(__builtin_amdgcn_exp2f(dv * A2[k]), st[r][k], in * b[r][k]);
                sum[r] = fmaf(st[r][k], c[r][k], sum[r]);
            }
            if (row0 + r < p.b)
                __builtin_nontemporal_store(st[r], reinterpret_cast<f4*>(p.fin + ((row0 + r) * p.E + e) * p.N + n0));
        }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        for (int off = seg >> 1; off > 0; off >>= 1) sum[r] += __shfl_xor(sum[r], off, 64);
        if (!live || n0 != 0 || row0 + r >= p.b) continue;
        const int64_t row = row0 + r;
        float v = p.D ? fmaf(p.D[e], xv[r], sum[r]) : sum[r];
        if (p.z) {
            const float zv = widen(static_cast<const T*>(p.z)[row * p.zb + e]);
            v *= zv * sigmoid_hw(zv);
        }
        static_cast<T*>(p.y)[row * p.E + e] = narrow<T>(v);
    }
}

template <typename T, int ROWS>
hipError_t step(const ScanParams& p, hipStream_t stream)
{
    int seg = 4, log2seg = 2;
    while (4 * seg < p.N) {
        seg <<= 1;
        ++log2seg;
    }
    const int64_t grid = ((p.b + ROWS - 1) / ROWS * p.E * seg + 255) / 256;
    if (!fits(grid, 256)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((k_scan_step<T, ROWS>), dim3(static_cast<unsigned>(grid)), dim3(256), 0, stream, p, seg, log2seg);
    return hipGetLastError();
}

template <typename T, bool PACKED, bool GATE, Mode MODE, int THREADS>
hipError_t chunk(const ScanParams& p, hipStream_t stream)
{
    const int64_t units = p.b * p.S * p.G * scan_tiles(p.E, p.G);
    const int slices = static_cast<int>(p.N / kSlice);
    const size_t lds = (MODE == kOutput || MODE == kOutputReady) && slices > 1 ? 2 * kTok * slices * 64 * sizeof(float) : 0;
    hipLaunchKernelGGL((k_scan_chunk<T, PACKED, GATE, MODE, THREADS>), dim3(static_cast<unsigned>(units)), dim3(64 * slices),
                       lds, stream, p);
    return hipGetLastError();
}

template <typename T, bool PACKED, bool GATE, Mode MODE>
hipError_t by_states(const ScanParams& p, hipStream_t stream)
{
    if (p.N <= kSlice) return chunk<T, PACKED, GATE, MODE, 64>(p, stream);
    if (p.N <= 4 * kSlice) return chunk<T, PACKED, GATE, MODE, 256>(p, stream);
    return chunk<T, PACKED, GATE, MODE, 1024>(p, stream);
}

template <typename T, bool PACKED, Mode MODE>
hipError_t by_gate(const ScanParams& p, hipStream_t stream)
{
    if constexpr (MODE != kStates)
        if (p.z) return by_states<T, PACKED, true, MODE>(p, stream);
    return by_states<T, PACKED, false, MODE>(p, stream);
}

template <typename T, Mode MODE>
hipError_t chunks(const ScanParams& p, hipStream_t stream)
{
    return p.seq_idx ? by_gate<T, true, MODE>(p, stream) : by_gate<T, false, MODE>(p, stream);
}

}  // namespace

hipError_t launch_scan_both(const ScanParams& p, bool bf16, hipStream_t stream)
{
    return bf16 ? chunks<uint16_t, kBoth>(p, stream) : chunks<float, kBoth>(p, stream);
}

hipError_t launch_scan_pass(const ScanParams& p, hipStream_t stream)
{
    const int64_t grid = (p.b * p.N * p.E + 255) / 256;
    hipLaunchKernelGGL(k_scan_pass, dim3(static_cast<unsigned>(grid)), dim3(256), 0, stream, p);
    return hipGetLastError();
}

ScanPlan scan_plan(int64_t b, int64_t T, int64_t E, int64_t N, int64_t G, bool backward)
{
    ScanPlan w{};
    const int64_t tiles = G * scan_tiles(E, G), waves = b * tiles * (N / kSlice);
    // Chunks: ten wavefronts a SIMD (10,240; gradients 6,144, three rounds of the two
    // that a SIMD holds of k_scan_grad and two of the three of k_scan_chunk<kBoth>: 8 x
    // 2,048 x 1,536 591 us, 4,096 wavefronts 628, 8,256 648), where there are not one and a half
    // (1,536) without: then the second pass costs more than idle SIMDs do (5,120
    // channels of 1,024 tokens, us by batch rows, whole / in chunks: 12 rows, 960
    // wavefronts, 536 / 451; 16 rows 679 / 571; 20 rows, 1,600, 689 / 771).  No chunk
    // shorter than 16 sqrt(T / 1,024) tokens, the least of a chunk's own time and of
    // the scan over the chunks' (1 x 777 x 5,120 float32: chunks of 16 tokens 61, 32
    // 66, 64 74; 1 x 16,384 x 768: 32 171, 64 147, 128 172), and none below 64 tokens
    // in all.
    int64_t S = waves < 1536 ? (backward ? 6144 : 10240) / waves : 1, shortest = 16;
    while (shortest * shortest * 4 < T) shortest *= 2;
    if (S > T / shortest) S = T / shortest;
    if (S < 1 || T < 64) S = 1;
    const int64_t unit = backward ? kBwdTile : kTok;
    w.L = ((T + S - 1) / S + unit - 1) / unit * unit;
    w.S = (T + w.L - 1) / w.L;
    w.cblocks = scan_tiles(E, G);
    size_t off = 0;
    const auto take = [&](int64_t floats) {
        const size_t at = off;
        off += (static_cast<size_t>(floats) * sizeof(float) + 255) / 256 * 256;
        return at;
    };
    const int64_t st = b * w.S * N * E;
    if (w.S > 1) {
        w.states = take(st);
        w.sums = take(b * w.S * E);
        if (backward)
            w.rstates = take(st);
        else
            w.steps = take(b * T * E);
    }
    if (backward) {
        w.marks = take(b * ((T + kBwdTile - 1) / kBwdTile) * N * E);
        w.marksums = take(b * ((T + kBwdTile - 1) / kBwdTile) * E);
        w.pA = take(st);
        w.pD = take(b * w.S * 2 * E);
        w.pBC = take(w.cblocks * b * T * G * 2 * N);
    }
    w.total = off;
    return w;
}

bool scan_fits(const ScanParams& p)
{
    return fits(p.b * p.S * p.G * scan_tiles(p.E, p.G), 4 * p.N) && fits((p.b * p.N * p.E + 255) / 256, 256);
}

hipError_t launch_scan_forward(const ScanParams& p, bool bf16, hipStream_t stream)
{
    if (!scan_fits(p)) return hipErrorInvalidConfiguration;
    if (p.S > 1) {
        hipError_t err = bf16 ? chunks<uint16_t, kStates>(p, stream) : chunks<float, kStates>(p, stream);
        if (err == hipSuccess) err = launch_scan_pass(p, stream);
        if (err != hipSuccess) return err;
        return bf16 ? chunks<uint16_t, kOutputReady>(p, stream) : chunks<float, kOutputReady>(p, stream);
    }
    return bf16 ? chunks<uint16_t, kOutput>(p, stream) : chunks<float, kOutput>(p, stream);
}

hipError_t launch_scan_step(const ScanParams& p, bool bf16, hipStream_t stream)
{
    // four rows a thread where that leaves the device 4,096 wavefronts (us with one
    // row and with four, 5,120 channels: 256 rows 33.1 and 30.4, 64 rows 10.2 and 9.3,
    // 32 rows, 2,560 wavefronts, 6.4 and 7.0, 4 rows 2.8 and 4.2)
    const bool four = p.b >= 4 && p.b / 4 * p.E * (p.N / 4) >= 4096 * 64;
    if (bf16) return four ? step<uint16_t, 4>(p, stream) : step<uint16_t, 1>(p, stream);
    return four ? step<float, 4>(p, stream) : step<float, 1>(p, stream);
}

}  // namespace ssd
