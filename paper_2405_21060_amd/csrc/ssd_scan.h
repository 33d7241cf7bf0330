// Device pieces that the selective scan's forward (ssd_scan.hip) and gradients
// (ssd_scan_bwd.hip) share.
//
// A lane holds a channel and a wavefront 64 of them, so that B_t and C_t, which
// all channels of a group share, are uniform: they come through the scalar cache
// into scalar registers, and every product with them takes one operand from there
// (no shared memory, no sum across lanes for y).  A lane holds 16 states of its
// channel in registers; more states take more wavefronts.
#pragma once

#include "ssd_ops.h"

namespace ssd {

constexpr int kSlice = 16;     // states a lane holds
constexpr int kTok = 8;        // tokens whose loads are issued together
constexpr int kBwdTile = 8;    // tokens per tile of the gradients

// A wavefront's place: channel tile (64 channels of one group), chunk, batch row.
struct ScanWork {
    int64_t row, chunk, t0, t1;
    int64_t g, e0;     // group, first channel
    unsigned lane;     // the lane's channel from there (a lane past its group's end: the last one)
    int64_t e;         // the same, from 0
    int64_t tile;      // channel tile within the group
    bool live;
};

__host__ __device__ __forceinline__ int64_t scan_tiles(int64_t E, int64_t G) { return (E / G + 63) / 64; }

__device__ __forceinline__ ScanWork scan_work(const ScanParams& p, int64_t unit)
{
    ScanWork w;
    const int64_t per = scan_tiles(p.E, p.G), all = per * p.G, eg = p.E / p.G;
    const int64_t at = unit / all, tile = unit - at * all;
    w.row = at / p.S;
    w.chunk = at - w.row * p.S;
    w.t0 = w.chunk * p.L;
    w.t1 = w.t0 + p.L < p.T ? w.t0 + p.L : p.T;
    w.g = tile / per;
    w.tile = tile - w.g * per;
    w.e0 = w.g * eg + w.tile * 64;
    const int64_t left = eg - w.tile * 64;
    const unsigned lane = threadIdx.x & 63;
    w.live = lane < left;
    w.lane = w.live ? lane : static_cast<unsigned>(left - 1);
    w.e = w.e0 + w.lane;
    return w;
}

template <bool PACKED>
__device__ __forceinline__ int64_t scan_unit(const ScanParams& p, int64_t row, int64_t t)
{
    if constexpr (!PACKED) return row;
    return held(scalar_load(p.seq_idx + t), p.nseq);
}

// Whether token t > 0 starts a sequence / token t ends one.
template <bool PACKED>
__device__ __forceinline__ bool scan_starts(const ScanParams& p, int64_t t)
{
    if (t == 0) return true;
    if constexpr (!PACKED) return false;
    return scalar_load(p.seq_idx + t) != scalar_load(p.seq_idx + t - 1);
}

template <bool PACKED>
__device__ __forceinline__ bool scan_ends(const ScanParams& p, int64_t t)
{
    if (t == p.T - 1) return true;
    if constexpr (!PACKED) return false;
    return scalar_load(p.seq_idx + t) != scalar_load(p.seq_idx + t + 1);
}

// Keeps a running scalar as it is: the compiler would otherwise make it anew for
// every token, by 64-bit products of the token and the stride.
template <typename P>
__device__ __forceinline__ void running(P& p) { asm volatile("" : "+s"(p)); }

// A lane's offset in a row of T, made where it is used: a load or store then adds
// the 32-bit offset to the scalar pointer itself (widened ahead of a loop, it takes a
// 64-bit addition for every access).
template <typename T>
__device__ __forceinline__ unsigned lane_offset(unsigned lane)
{
    unsigned off = lane * sizeof(T);
    asm volatile("" : "+v"(off));
    return off;
}

// A tensor's row of a token, walked from token to token: a uniform pointer and the
// lane's offset.
template <typename T>
struct Rows {
    typedef __attribute__((address_space(1))) T* pointer;
    pointer p;
    int step;   // elements to the next token's row

    __device__ __forceinline__ Rows(const void* base, int64_t first, int64_t stride)
        : p((pointer)(reinterpret_cast<uintptr_t>(base) + first * sizeof(T))), step(static_cast<int>(stride)) {}
    // `off`: the lane's offset in bytes (lane_offset)
    __device__ __forceinline__ pointer at(unsigned off) const
    {
        typedef __attribute__((address_space(1))) char* bytes;
        return (pointer)((bytes)p + off);
    }
    __device__ __forceinline__ T get(unsigned off) const { return *at(off); }
    __device__ __forceinline__ void put(unsigned off, T v) const { *at(off) = v; }
    __device__ __forceinline__ void move(bool on = true)
    {
        p += on ? step : 0;
        running(p);
    }
};

// K uniform values (4-byte aligned) of a row, through the scalar cache: the words
// as they were read, and what they hold.
template <typename T, int K>
struct Uniform {
    static constexpr int D = K * sizeof(T) / 4;
    typedef uint32_t words __attribute__((ext_vector_type(D)));
    typedef uint32_t words_in_memory __attribute__((ext_vector_type(D), aligned(4)));
    words w;

    __device__ __forceinline__ void load(const Rows<const T>& r)
    {
        w = *reinterpret_cast<const __attribute__((address_space(4))) words_in_memory*>((uintptr_t)r.p);
    }
    // Waits for the words here, so that loads issued after are not waited for.
    __device__ __forceinline__ void arrive() { asm volatile("" : "+s"(w)); }
    __device__ __forceinline__ float operator[](int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        return __uint_as_float(i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    }
};

// A lane's 16 states of a unit, in the caller's layout (units, E, N).
__device__ __forceinline__ void load_states(const float* s, const ScanParams& p, int64_t unit, int64_t e, int n0,
                                            float (&h)[kSlice])
{
    if (!s) {
#pragma unroll
        for (int n = 0; n < kSlice; ++n) h[n] = 0.f;
        return;
    }
    const float4* at = reinterpret_cast<const float4*>(s + (unit * p.E + e) * p.N + n0);
#pragma unroll
    for (int k = 0; k < kSlice / 4; ++k) {
        const float4 v = at[k];
        h[4 * k] = v.x;
        h[4 * k + 1] = v.y;
        h[4 * k + 2] = v.z;
        h[4 * k + 3] = v.w;
    }
}

__device__ __forceinline__ void store_states(float* s, const ScanParams& p, int64_t unit, int64_t e, int n0,
                                             const float (&h)[kSlice])
{
    float4* at = reinterpret_cast<float4*>(s + (unit * p.E + e) * p.N + n0);
#pragma unroll
    for (int k = 0; k < kSlice / 4; ++k) at[k] = make_float4(h[4 * k], h[4 * k + 1], h[4 * k + 2], h[4 * k + 3]);
}

// A in log2 units: exp(dt A) = exp2(dt A2).  A_log is held to [-104, 88], so that A is
// finite and a time step of 0 keeps the state, as it does where A = -exp(A_log) is
// beyond float32; a step above 1e-36 forgets it.  (minimum and maximum, not a median: a NaN
// stays one.)
__device__ __forceinline__ float decay_rate(float a_log)
{
    const float a = __builtin_elementwise_minimum(__builtin_elementwise_maximum(a_log, -104.f), 88.f);
    return exp_of(a) * -kLog2e;
}

__device__ __forceinline__ float time_step(const ScanParams& p, float v) { return p.softplus ? softplus_hw(v) : v; }

hipError_t launch_scan_both(const ScanParams& p, bool bf16, hipStream_t stream);
hipError_t launch_scan_pass(const ScanParams& p, hipStream_t stream);
bool scan_fits(const ScanParams& p);   // the grids of the chunk and pass kernels

}  // namespace ssd
