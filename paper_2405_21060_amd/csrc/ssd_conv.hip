// The block's short causal depthwise convolution with SiLU: forward, gradients
// and the single-token step.
//
//     v_t = bias + sum_{j < W} w_j x_{t-W+1+j},   y_t = v_t sigmoid(v_t)
//     g_t = dy_t s (1 + v_t (1 - s)),  s = sigmoid(v_t)
//     dx_t = sum_k w_{W-1-k} g_{t+k},  dw_j = sum_t g_t x_{t-W+1+j},  db = sum_t g_t
//
// Bound by HBM: x is read and y written once (gradients: x and dy read, dx
// written).  A wavefront takes a strip of consecutive tokens of 64 x V channels
// (V = 2 a lane; 4 and 8 hold more registers and leave fewer wavefronts: forward 4 x
// 4,096 x 5,376 bf16 76 us, 84 and 92, gradients 1 x 32,768 x 6,144 in strips of 128
// tokens 283, 289 and 333) and walks down the tokens with the W - 1 rows
// before the present one in registers, so that a token's row is read once, and
// the W - 1 rows in front of a strip once more.  Sequences of a packed row are the
// wavefront's own control flow: at a sequence's first token the rows in
// registers are replaced by that sequence's state (never multiplied by 0, so
// that nothing of the sequence before is carried over, infinities included).
//
// The gradients walk the same way: dx_t is complete W - 1 tokens later, so W
// running sums move down with the tokens, and a strip goes on for W - 1 tokens
// past its end for those of its last ones.  Each strip's sums of dw and db go to
// a workspace row, added up by k_conv_dw in a fixed order.
#include "ssd_internal.h"
#include "ssd_ops.h"

namespace ssd {
namespace {

constexpr int kWaves = 4;       // wavefronts (strips x channel tiles) per workgroup
constexpr int kBatch = 4;       // tokens whose loads are issued together

// A wavefront's channel tile, token strip and batch row (all uniform), and its
// lane's channels.
struct Work {
    int64_t row, t0, t1;   // tokens [t0, t1)
    int64_t strip;         // over all rows
    int part;
    int64_t c, cp;         // first channel, overall and within its part
    int64_t pw;            // channels of the part
    bool live;             // false: nothing to do
};

template <int V>
__device__ __forceinline__ int64_t tiles_of(const ConvParams& p, int part)
{
    return (p.off[part + 1] - p.off[part] + 64 * V - 1) / (64 * V);
}

template <int V>
__device__ __forceinline__ Work work_of(const ConvParams& p, int64_t R, int64_t strips)
{
    Work w;
    int64_t tiles[3] = {tiles_of<V>(p, 0), 0, 0};
    for (int i = 1; i < p.nparts; ++i) tiles[i] = tiles_of<V>(p, i);
    const int64_t all = tiles[0] + tiles[1] + tiles[2];
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * kWaves + uniform(threadIdx.x >> 6);
    int64_t tile = unit % all;
    w.strip = unit / all;
    w.row = w.strip / strips;
    w.t0 = (w.strip - w.row * strips) * R;
    w.t1 = w.t0 + R < p.T ? w.t0 + R : p.T;
    w.part = 0;
    while (w.part < 2 && tile >= tiles[w.part]) tile -= tiles[w.part++];
    w.pw = p.off[w.part + 1] - p.off[w.part];
    // A part's last vector is moved back so that it ends with the part (two lanes
    // then hold the same channels and write the same values).
    const int64_t at = tile * 64 * V + (threadIdx.x & 63) * V;
    w.live = w.row < p.b && at < w.pw;
    w.cp = at + V <= w.pw ? at : w.pw - V;
    w.c = p.off[w.part] + w.cp;
    return w;
}

// The sequence that a token belongs to.
template <bool PACKED>
__device__ __forceinline__ int64_t unit_of(const ConvParams& p, int64_t row, int64_t t)
{
    if constexpr (!PACKED) return row;
    return held(scalar_load(p.seq_idx + t), p.nseq);
}

template <bool PACKED>
__device__ __forceinline__ bool ends_at(const ConvParams& p, int64_t t)
{
    if (t == p.T - 1) return true;
    if constexpr (!PACKED) return false;
    return scalar_load(p.seq_idx + t) != scalar_load(p.seq_idx + t + 1);
}

template <typename T, int W, int V>
__device__ __forceinline__ void state_row(const ConvParams& p, const void* states, int64_t unit, int r, int64_t c,
                                          float (&v)[V])
{
    if (!states) {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = 0.f;
        return;
    }
    const auto x = Pack<T, V>::load(static_cast<const T*>(states) + (unit * (W - 1) + r) * p.C + c);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = x[e];
}

// win[j] = the row W - 1 - j tokens before t0, j = 0 .. W - 2, from x or from the
// sequence's state; returns how many of them are the sequence's own tokens.
template <typename T, int W, int V, bool PACKED>
__device__ __forceinline__ int rows_before(const ConvParams& p, const T* x, int64_t unit, int64_t t0, int64_t c,
                                           float (&win)[W - 1][V])
{
    int own = 0;
#pragma unroll
    for (int back = 1; back < W; ++back) {
        bool in = own == back - 1 && t0 - back >= 0;
        if constexpr (PACKED)
            if (in) in = scalar_load(p.seq_idx + t0 - back) == scalar_load(p.seq_idx + t0);
        if (in) ++own;
    }
#pragma unroll
    for (int back = 1; back < W; ++back) {
        if (back <= own) {
            const auto v = Pack<T, V>::load(x + (t0 - back) * p.xt + c);
#pragma unroll
            for (int e = 0; e < V; ++e) win[W - 1 - back][e] = v[e];
        } else {
            state_row<T, W, V>(p, p.init, unit, W - 1 - (back - own), c, win[W - 1 - back]);
        }
    }
    return own;
}

template <typename T, int W, int V, bool PACKED>
__global__ __launch_bounds__(64 * kWaves) void k_conv_forward(ConvParams p, int64_t R, int64_t strips)
{
    const Work wk = work_of<V>(p, R, strips);
    if (!wk.live) return;
    const T* x = static_cast<const T*>(p.x) + wk.row * p.xb;
    T* y = static_cast<T*>(p.y[wk.part]) + wk.row * p.T * wk.pw + wk.cp;
    float w[W][V], bias[V], win[W - 1][V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        bias[e] = p.bias ? p.bias[wk.c + e] : 0.f;
#pragma unroll
        for (int j = 0; j < W; ++j) w[j][e] = p.weight[(wk.c + e) * W + j];
    }
    int64_t unit = unit_of<PACKED>(p, wk.row, wk.t0);
    rows_before<T, W, V, PACKED>(p, x, unit, wk.t0, wk.c, win);
    for (int64_t t = wk.t0; t < wk.t1; t += kBatch) {
        Pack<T, V> in[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            if (t + u < wk.t1) in[u] = Pack<T, V>::load(x + (t + u) * p.xt + wk.c);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (t + u >= wk.t1) break;
            if constexpr (PACKED) {
                if (t + u > wk.t0 && scalar_load(p.seq_idx + t + u) != scalar_load(p.seq_idx + t + u - 1)) {
                    unit = unit_of<PACKED>(p, wk.row, t + u);
#pragma unroll
                    for (int j = 0; j < W - 1; ++j) state_row<T, W, V>(p, p.init, unit, j, wk.c, win[j]);
                }
            }
            Pack<T, V> out;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float v = bias[e];
#pragma unroll
                for (int j = 0; j < W - 1; ++j) v = fmaf(w[j][e], win[j][e], v);
                const float now = in[u][e];
                v = fmaf(w[W - 1][e], now, v);
                out.set(e, p.silu ? v * sigmoid_hw(v) : v);
#pragma unroll
                for (int j = 0; j < W - 2; ++j) win[j][e] = win[j + 1][e];
                win[W - 2][e] = now;
            }
            out.store(y + (t + u) * wk.pw);
            if (p.fin && ends_at<PACKED>(p, t + u)) {
                T* f = static_cast<T*>(p.fin) + unit * (W - 1) * p.C + wk.c;
#pragma unroll
                for (int j = 0; j < W - 1; ++j) {
                    Pack<T, V> o;
#pragma unroll
                    for (int e = 0; e < V; ++e) o.set(e, win[j][e]);
                    o.store(f + j * p.C);
                }
            }
        }
    }
}

template <typename T, int W, int V, bool PACKED>
__global__ __launch_bounds__(64 * kWaves) void k_conv_backward(ConvParams p, int64_t R, int64_t strips)
{
    const Work wk = work_of<V>(p, R, strips);
    if (!wk.live) return;
    const T* x = static_cast<const T*>(p.x) + wk.row * p.xb;
    const T* dy = static_cast<const T*>(p.dy[wk.part]) + wk.row * p.T * wk.pw + wk.cp;
    T* dx = static_cast<T*>(p.dx) + wk.row * p.T * p.C + wk.c;
    float w[W][V], bias[V], win[W - 1][V];
    float dw[W][V], db[V];     // this strip's sums
    float sum[W][V];           // sum[k]: the gradient of the row k tokens back, so far
#pragma unroll
    for (int e = 0; e < V; ++e) {
        bias[e] = p.bias ? p.bias[wk.c + e] : 0.f;
        db[e] = 0.f;
#pragma unroll
        for (int j = 0; j < W; ++j) {
            w[j][e] = p.weight[(wk.c + e) * W + j];
            dw[j][e] = sum[j][e] = 0.f;
        }
    }
    int64_t unit = unit_of<PACKED>(p, wk.row, wk.t0);
    // the sequence's first token, or one at least W - 1 tokens before the strip
    int64_t start = wk.t0 - rows_before<T, W, V, PACKED>(p, x, unit, wk.t0, wk.c, win);

    // The finished gradient of the row at token `tok`: a token of this strip, or a
    // row of the state of a sequence that starts in this strip.
    const auto emit = [&](int64_t tok, const float (&v)[V]) {
        T* to = nullptr;
        if (tok >= start) {
            if (tok >= wk.t0 && tok < wk.t1) to = dx + tok * p.C;
        } else if (start >= wk.t0 && p.dinit) {
            to = static_cast<T*>(p.dinit) + (unit * (W - 1) + (tok - start + W - 1)) * p.C + wk.c;
        }
        if (!to) return;
        Pack<T, V> o;
#pragma unroll
        for (int e = 0; e < V; ++e) o.set(e, v[e]);
        o.store(to);
    };

    const int64_t stop = wk.t1 + W - 1 < p.T ? wk.t1 + W - 1 : p.T;
    bool done = false;
    for (int64_t t = wk.t0; t < stop && !done; t += kBatch) {
        Pack<T, V> in[kBatch], din[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            if (t + u < stop) {
                in[u] = Pack<T, V>::load(x + (t + u) * p.xt + wk.c);
                din[u] = Pack<T, V>::load(dy + (t + u) * wk.pw);
            }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int64_t now = t + u;
            if (now >= stop || done) break;
            const bool mine = now < wk.t1;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float v = bias[e];
#pragma unroll
                for (int j = 0; j < W - 1; ++j) v = fmaf(w[j][e], win[j][e], v);
                const float xv = in[u][e];
                v = fmaf(w[W - 1][e], xv, v);
                float g = din[u][e];
                if (p.silu) {
                    const float s = sigmoid_hw(v);
                    g *= s * fmaf(v, 1.f - s, 1.f);
                }
                if (mine) {
                    db[e] += g;
#pragma unroll
                    for (int j = 0; j < W - 1; ++j) dw[j][e] = fmaf(g, win[j][e], dw[j][e]);
                    dw[W - 1][e] = fmaf(g, xv, dw[W - 1][e]);
                }
#pragma unroll
                for (int k = 0; k < W; ++k) sum[k][e] = fmaf(w[W - 1 - k][e], g, sum[k][e]);
#pragma unroll
                for (int j = 0; j < W - 2; ++j) win[j][e] = win[j + 1][e];
                win[W - 2][e] = xv;
            }
            if (ends_at<PACKED>(p, now)) {
                // the sequence ends here: what is still open is finished, with the
                // final state's gradient (its rows are the last W - 1 ones)
#pragma unroll
                for (int k = W - 1; k >= 0; --k) {
                    float v[V];
#pragma unroll
                    for (int e = 0; e < V; ++e) v[e] = sum[k][e];
                    if (k < W - 1 && p.dfin) {
                        float d[V];
                        state_row<T, W, V>(p, p.dfin, unit, W - 2 - k, wk.c, d);
#pragma unroll
                        for (int e = 0; e < V; ++e) v[e] += d[e];
                    }
                    emit(now - k, v);
                }
                done = now + 1 >= wk.t1;
                if (PACKED && !done) {
                    start = now + 1;
                    unit = unit_of<PACKED>(p, wk.row, start);
#pragma unroll
                    for (int j = 0; j < W - 1; ++j) state_row<T, W, V>(p, p.init, unit, j, wk.c, win[j]);
#pragma unroll
                    for (int k = 0; k < W; ++k)
#pragma unroll
                        for (int e = 0; e < V; ++e) sum[k][e] = 0.f;
                }
            } else {
                emit(now - (W - 1), sum[W - 1]);
#pragma unroll
                for (int e = 0; e < V; ++e) {
#pragma unroll
                    for (int k = W - 1; k > 0; --k) sum[k][e] = sum[k - 1][e];
                    sum[0][e] = 0.f;
                }
            }
        }
    }
    float* part = p.partial + wk.strip * (W + 1) * p.C + wk.c;
#pragma unroll
    for (int e = 0; e < V; ++e) {
#pragma unroll
        for (int j = 0; j < W; ++j) part[j * p.C + e] = dw[j][e];
        part[W * p.C + e] = db[e];
    }
}

// dweight and dbias: the strips' partial sums, in a fixed order.
__global__ __launch_bounds__(kSumLanes * kSumCols) void k_conv_dw(ConvParams p, int64_t strips)
{
    const int64_t cols = (p.W + 1) * p.C, i = static_cast<int64_t>(blockIdx.x) * kSumCols + threadIdx.x % kSumCols;
    const float v = column_sum(p.partial + i, strips, cols, i < cols);
    if (threadIdx.x >= kSumCols || i >= cols) return;
    const int64_t j = i / p.C, c = i - j * p.C;
    if (j < p.W)
        p.dweight[c * p.W + j] = v;
    else if (p.dbias)
        p.dbias[c] = v;
}

// One token per batch row: V channels a thread, the state's rows read, used and
// moved up by one in place.
template <typename T, int W, int V>
__global__ __launch_bounds__(256) void k_conv_step(ConvParams p)
{
    const int64_t per = p.C / V, i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= p.b * per) return;
    const int64_t row = i / per, c = (i - row * per) * V;
    const auto in = Pack<T, V>::load(static_cast<const T*>(p.x) + row * p.xb + c);
    T* st = static_cast<T*>(p.fin) + row * (W - 1) * p.C + c;
    Pack<T, V> old[W - 1], out;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) old[j] = Pack<T, V>::load(st + j * p.C);
#pragma unroll
    for (int e = 0; e < V; ++e) {
        float v = p.bias ? p.bias[c + e] : 0.f;
#pragma unroll
        for (int j = 0; j < W - 1; ++j) v = fmaf(p.weight[(c + e) * W + j], old[j][e], v);
        v = fmaf(p.weight[(c + e) * W + W - 1], in[e], v);
        out.set(e, p.silu ? v * sigmoid_hw(v) : v);
    }
#pragma unroll
    for (int j = 0; j + 1 < W - 1; ++j) old[j + 1].store(st + j * p.C);
    in.store(st + (W - 2) * p.C);
    out.store(static_cast<T*>(p.y[0]) + row * p.C + c);
}

int64_t channel_tiles(const ConvParams& p, int V)
{
    int64_t n = 0;
    for (int i = 0; i < p.nparts; ++i) n += (p.off[i + 1] - p.off[i] + 64 * V - 1) / (64 * V);
    return n;
}

// Vectors of two channels, where every part has that many.
bool vectors(const ConvParams& p)
{
    for (int i = 0; i < p.nparts; ++i)
        if (p.off[i + 1] - p.off[i] < 2) return false;
    return true;
}

// Tokens per strip: longer strips read fewer rows twice, shorter ones give more
// wavefronts; the longest that leaves 4,096 (four a SIMD), else the shortest.  The
// longest is 32 tokens (64: 80 us for the forward above) and 256 for the gradients
// (275 us; 128: 283, 64: 297), whose strips have a row of partial sums each.
int64_t strip_tokens(int64_t b, int64_t T, int64_t tiles, int64_t longest, int64_t shortest)
{
    int64_t R = longest;
    while (R > shortest && b * tiles * ((T + R - 1) / R) < 4096) R /= 2;
    return R;
}

template <typename T, int W, int V, bool PACKED>
hipError_t run(const ConvParams& p, int64_t R, bool backward, hipStream_t stream)
{
    const int64_t strips = (p.T + R - 1) / R;
    const int64_t units = channel_tiles(p, V) * strips * p.b;
    const int64_t grid = (units + kWaves - 1) / kWaves;
    if (!fits(grid, 64 * kWaves) || !fits((W + 1) * p.C, kSumLanes)) return hipErrorInvalidConfiguration;
    if (backward)
        hipLaunchKernelGGL((k_conv_backward<T, W, V, PACKED>), dim3(static_cast<unsigned>(grid)), dim3(64 * kWaves), 0,
                           stream, p, R, strips);
    else
        hipLaunchKernelGGL((k_conv_forward<T, W, V, PACKED>), dim3(static_cast<unsigned>(grid)), dim3(64 * kWaves), 0,
                           stream, p, R, strips);
    return hipGetLastError();
}

template <typename T, int W>
hipError_t by_vector(const ConvParams& p, int64_t R, bool backward, hipStream_t stream)
{
    if (vectors(p)) return p.seq_idx ? run<T, W, 2, true>(p, R, backward, stream) : run<T, W, 2, false>(p, R, backward, stream);
    return p.seq_idx ? run<T, W, 1, true>(p, R, backward, stream) : run<T, W, 1, false>(p, R, backward, stream);
}

template <typename T>
hipError_t by_width(const ConvParams& p, int64_t R, bool backward, hipStream_t stream)
{
    switch (p.W) {
    case 2: return by_vector<T, 2>(p, R, backward, stream);
    case 3: return by_vector<T, 3>(p, R, backward, stream);
    default: return by_vector<T, 4>(p, R, backward, stream);
    }
}

template <typename T, int W>
hipError_t step(const ConvParams& p, hipStream_t stream)
{
    const int64_t n = p.C % 4 == 0 ? p.b * (p.C / 4) : p.b * p.C;
    const int64_t grid = (n + 255) / 256;
    if (!fits(grid, 256)) return hipErrorInvalidConfiguration;
    if (p.C % 4 == 0)
        hipLaunchKernelGGL((k_conv_step<T, W, 4>), dim3(static_cast<unsigned>(grid)), dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL((k_conv_step<T, W, 1>), dim3(static_cast<unsigned>(grid)), dim3(256), 0, stream, p);
    return hipGetLastError();
}

template <typename T>
hipError_t step_by_width(const ConvParams& p, hipStream_t stream)
{
    return p.W == 2 ? step<T, 2>(p, stream) : p.W == 3 ? step<T, 3>(p, stream) : step<T, 4>(p, stream);
}

}  // namespace

// (by the channels alone, not by the parts: the workspace depends on it)
int64_t conv_bwd_strip(int64_t b, int64_t T, int64_t C) { return strip_tokens(b, T, (C + 127) / 128, 256, 16); }

hipError_t launch_conv_forward(const ConvParams& p, bool bf16, hipStream_t stream)
{
    const int64_t R = strip_tokens(p.b, p.T, channel_tiles(p, vectors(p) ? 2 : 1), 32, 4);
    return bf16 ? by_width<uint16_t>(p, R, false, stream) : by_width<float>(p, R, false, stream);
}

hipError_t launch_conv_backward(const ConvParams& p, bool bf16, hipStream_t stream)
{
    const int64_t R = conv_bwd_strip(p.b, p.T, p.C), strips = p.b * ((p.T + R - 1) / R);
    const hipError_t err = bf16 ? by_width<uint16_t>(p, R, true, stream) : by_width<float>(p, R, true, stream);
    if (err != hipSuccess) return err;
    const int64_t cols = (p.W + 1) * p.C;
    hipLaunchKernelGGL(k_conv_dw, dim3(static_cast<unsigned>((cols + kSumCols - 1) / kSumCols)),
                       dim3(kSumLanes * kSumCols), 0, stream, p, strips);
    return hipGetLastError();
}

hipError_t launch_conv_step(const ConvParams& p, bool bf16, hipStream_t stream)
{
    return bf16 ? step_by_width<uint16_t>(p, stream) : step_by_width<float>(p, stream);
}

}  // namespace ssd
