// C ABI of the operators around the layer: the short convolution, the selective
// scan, the residual addition with norm.  Validation, workspace planning, launch;
// no HIP call is made before the arguments have been validated.
#include "ssd.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "ssd_internal.h"
#include "ssd_ops.h"

namespace {

// Elements of a tensor: the layer's limit (16 x 2^31).
constexpr double kMostElems = 16.0 * 0x7fffffffLL;

bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

bool known(int32_t dtype) { return dtype == SSD_DTYPE_F32 || dtype == SSD_DTYPE_BF16; }

size_t size_of(int32_t dtype) { return dtype == SSD_DTYPE_BF16 ? 2 : 4; }

// (a launcher that finds a grid too large says so before it launches anything)
int status(hipError_t err)
{
    return err == hipSuccess ? SSD_OK : err == hipErrorInvalidConfiguration ? SSD_ERR_TOO_LARGE : SSD_ERR_LAUNCH;
}

// Packed rows: one row, as many sequences as fit.
int check_packed(bool packed, int64_t batch, int64_t seqlen, int64_t nseq)
{
    if (!packed) return SSD_OK;
    if (batch != 1) return SSD_ERR_SEQIDX_BATCH;
    return nseq < 1 || nseq > seqlen ? SSD_ERR_BAD_SHAPE : SSD_OK;
}

// Strides: not negative, the furthest element within the tensor limit.
bool reaches(int64_t batch, int64_t bs, int64_t seqlen, int64_t ts, int64_t last)
{
    return static_cast<double>(batch - 1) * bs + static_cast<double>(seqlen - 1) * ts + last <= 4 * kMostElems;
}

// ---- convolution ---------------------------------------------------------------

int validate_conv(const ssd_conv_problem* prob, bool packed, bool step, ssd::ConvParams* p)
{
    if (!prob) return SSD_ERR_NULL_ARG;
    if (!known(prob->dtype)) return SSD_ERR_BAD_DTYPE;
    const int64_t T = step ? 1 : prob->seqlen;
    if (prob->batch < 1 || T < 1 || prob->channels < 1 || prob->width < 1) return SSD_ERR_BAD_SHAPE;
    if (prob->width < 2 || prob->width > 4) return SSD_ERR_UNSUPPORTED_DIMS;
    *p = ssd::ConvParams{};
    p->b = prob->batch;
    p->T = T;
    p->C = prob->channels;
    p->W = static_cast<int>(prob->width);
    p->silu = prob->silu != 0;
    // (strides over a single row or token play no part)
    p->xb = p->b > 1 ? prob->x_batch_stride : 0;
    p->xt = T > 1 ? prob->x_token_stride : 0;
    if (!step) {
        if (prob->nparts < 1 || prob->nparts > 3) return SSD_ERR_BAD_SHAPE;
        p->nparts = static_cast<int>(prob->nparts);
        int64_t at = 0;
        for (int i = 0; i < p->nparts; ++i) {
            if (prob->parts[i] < 1 || prob->parts[i] > p->C - at) return SSD_ERR_BAD_SHAPE;
            p->off[i] = at;
            at += prob->parts[i];
        }
        if (at != p->C) return SSD_ERR_BAD_SHAPE;
        for (int i = p->nparts; i < 4; ++i) p->off[i] = at;
        if (const int rc = check_packed(packed, p->b, T, prob->nseq); rc != SSD_OK) return rc;
    }
    if (p->xb < 0 || p->xt < 0) return SSD_ERR_BAD_SHAPE;
    p->nseq = packed ? prob->nseq : p->b;
    if (static_cast<double>(p->b) * T * p->C > kMostElems || static_cast<double>(p->nseq) * 4 * p->C > kMostElems ||
        !reaches(p->b, p->xb, T, p->xt, p->C))
        return SSD_ERR_TOO_LARGE;
    return SSD_OK;
}

size_t conv_workspace(const ssd::ConvParams& p)
{
    const int64_t R = ssd::conv_bwd_strip(p.b, p.T, p.C);
    return static_cast<size_t>(p.b * ((p.T + R - 1) / R)) * (p.W + 1) * p.C * sizeof(float);
}

// ---- selective scan ------------------------------------------------------------

int validate_scan(const ssd_scan_problem* prob, bool packed, bool step, bool z, ssd::ScanParams* p)
{
    if (!prob) return SSD_ERR_NULL_ARG;
    if (!known(prob->dtype)) return SSD_ERR_BAD_DTYPE;
    const int64_t T = step ? 1 : prob->seqlen;
    if (prob->batch < 1 || T < 1 || prob->channels < 1 || prob->dstate < 1 || prob->ngroups < 1 ||
        prob->channels % prob->ngroups != 0)
        return SSD_ERR_BAD_SHAPE;
    if (prob->dstate % 16 != 0 || prob->dstate > 256) return SSD_ERR_UNSUPPORTED_DIMS;
    *p = ssd::ScanParams{};
    p->b = prob->batch;
    p->T = T;
    p->E = prob->channels;
    p->N = prob->dstate;
    p->G = prob->ngroups;
    p->softplus = prob->dt_softplus != 0;
    if (p->b > 1) {   // (strides over a single row or token play no part)
        p->xb = prob->x_batch_stride;
        p->db = prob->dt_batch_stride;
        p->zb = z ? prob->z_batch_stride : 0;
        p->bb = prob->b_batch_stride;
        p->cb = prob->c_batch_stride;
    }
    if (T > 1) {
        p->xt = prob->x_token_stride;
        p->dtt = prob->dt_token_stride;
        p->zt = z ? prob->z_token_stride : 0;
        p->bt = prob->b_token_stride;
        p->ct = prob->c_token_stride;
    }
    if (!step) {
        if (const int rc = check_packed(packed, p->b, T, prob->nseq); rc != SSD_OK) return rc;
    }
    for (int64_t s : {p->xb, p->xt, p->db, p->dtt, p->zb, p->zt, p->bb, p->bt, p->cb, p->ct})
        if (s < 0) return SSD_ERR_BAD_SHAPE;
    p->nseq = packed ? prob->nseq : p->b;
    const double act = static_cast<double>(p->b) * T * p->E, bc = static_cast<double>(p->b) * T * p->G * p->N;
    if (act > kMostElems || bc > kMostElems || static_cast<double>(p->nseq) * p->E * p->N > kMostElems ||
        !reaches(p->b, p->xb, T, p->xt, p->E) || !reaches(p->b, p->db, T, p->dtt, p->E) ||
        !reaches(p->b, p->zb, T, p->zt, p->E) || !reaches(p->b, p->bb, T, p->bt, p->G * p->N) ||
        !reaches(p->b, p->cb, T, p->ct, p->G * p->N))
        return SSD_ERR_TOO_LARGE;
    // the kernels step from token to token in 32 bits
    for (int64_t s : {p->E, p->xt, p->dtt, p->zt, p->bt, p->ct})
        if (s > INT32_MAX) return SSD_ERR_TOO_LARGE;
    return SSD_OK;
}

// B and C go through the scalar cache, which reads whole words.
bool whole_words(const ssd::ScanParams& p, int32_t dtype, const void* B, const void* C)
{
    if (!aligned(B, 4) || !aligned(C, 4)) return false;
    return dtype == SSD_DTYPE_F32 || (p.bb % 2 == 0 && p.bt % 2 == 0 && p.cb % 2 == 0 && p.ct % 2 == 0);
}

ssd::ScanPlan plan(const ssd::ScanParams& p, bool backward)
{
    return ssd::scan_plan(p.b, p.T, p.E, p.N, p.G, backward);
}

void place(const ssd::ScanPlan& w, void* workspace, ssd::ScanParams* p)
{
    char* base = static_cast<char*>(workspace);
    const auto at = [&](size_t off) { return reinterpret_cast<float*>(base + off); };
    p->S = w.S;
    p->L = w.L;
    p->states = at(w.states);
    p->sums = at(w.sums);
    p->steps = at(w.steps);
    p->rstates = at(w.rstates);
    p->marks = at(w.marks);
    p->marksums = at(w.marksums);
    p->pA = at(w.pA);
    p->pD = at(w.pD);
    p->pBC = at(w.pBC);
}

int scan_bytes(const ssd_scan_problem* prob, bool backward, size_t* bytes)
{
    if (!bytes) return SSD_ERR_NULL_ARG;
    ssd::ScanParams p;
    const int rc = validate_scan(prob, false, false, false, &p);
    if (rc == SSD_OK) *bytes = plan(p, backward).total;
    return rc;
}

// ---- residual addition and norm --------------------------------------------------

int validate_norm(const ssd_norm_problem* prob, ssd::NormParams* p)
{
    if (!prob) return SSD_ERR_NULL_ARG;
    if (!known(prob->dtype) || !known(prob->residual_dtype) ||
        (prob->dtype == SSD_DTYPE_F32 && prob->residual_dtype != SSD_DTYPE_F32))
        return SSD_ERR_BAD_DTYPE;
    if (prob->rows < 1 || prob->channels < 1) return SSD_ERR_BAD_SHAPE;
    if (prob->channels > 32768) return SSD_ERR_UNSUPPORTED_DIMS;
    if (!(prob->eps >= 0.f) || !std::isfinite(prob->eps)) return SSD_ERR_BAD_OPTION;
    if (static_cast<double>(prob->rows) * prob->channels > kMostElems) return SSD_ERR_TOO_LARGE;
    *p = ssd::NormParams{};
    p->rows = prob->rows;
    p->C = prob->channels;
    p->eps = prob->eps;
    return SSD_OK;
}

}  // namespace

extern "C" int ssd_conv_forward(const ssd_conv_problem* prob, const void* x, const float* weight, const float* bias,
                                const void* initial_states, const int32_t* seq_idx, void* const* y, void* final_states,
                                void* stream)
{
    ssd::ConvParams p;
    if (const int rc = validate_conv(prob, seq_idx != nullptr, false, &p); rc != SSD_OK) return rc;
    if (!x || !weight || !y) return SSD_ERR_NULL_ARG;
    for (int i = 0; i < p.nparts; ++i)
        if (!(p.y[i] = y[i])) return SSD_ERR_NULL_ARG;
    p.x = x;
    p.weight = weight;
    p.bias = bias;
    p.init = initial_states;
    p.seq_idx = seq_idx;
    p.fin = final_states;
    return status(ssd::launch_conv_forward(p, prob->dtype == SSD_DTYPE_BF16, static_cast<hipStream_t>(stream)));
}

extern "C" int ssd_conv_backward_workspace_bytes(const ssd_conv_problem* prob, size_t* bytes)
{
    if (!bytes) return SSD_ERR_NULL_ARG;
    ssd::ConvParams p;
    const int rc = validate_conv(prob, false, false, &p);
    if (rc == SSD_OK) *bytes = conv_workspace(p);
    return rc;
}

extern "C" int ssd_conv_backward(const ssd_conv_problem* prob, const void* x, const float* weight, const float* bias,
                                 const void* initial_states, const int32_t* seq_idx, const void* const* dy,
                                 const void* dfinal_states, void* dx, float* dweight, float* dbias,
                                 void* dinitial_states, void* workspace, size_t workspace_bytes, void* stream)
{
    ssd::ConvParams p;
    if (const int rc = validate_conv(prob, seq_idx != nullptr, false, &p); rc != SSD_OK) return rc;
    if (!x || !weight || !dy || !dx || !dweight) return SSD_ERR_NULL_ARG;
    for (int i = 0; i < p.nparts; ++i)
        if (!(p.dy[i] = dy[i])) return SSD_ERR_NULL_ARG;
    if (!workspace || workspace_bytes < conv_workspace(p)) return SSD_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return SSD_ERR_UNSUPPORTED_DIMS;
    p.x = x;
    p.weight = weight;
    p.bias = bias;
    p.init = initial_states;
    p.seq_idx = seq_idx;
    p.dfin = dfinal_states;
    p.dx = dx;
    p.dweight = dweight;
    p.dbias = dbias;
    p.dinit = dinitial_states;
    p.partial = static_cast<float*>(workspace);
    return status(ssd::launch_conv_backward(p, prob->dtype == SSD_DTYPE_BF16, static_cast<hipStream_t>(stream)));
}

extern "C" int ssd_conv_step(const ssd_conv_problem* prob, const void* x, const float* weight, const float* bias,
                             void* state, void* y, void* stream)
{
    ssd::ConvParams p;
    if (const int rc = validate_conv(prob, false, true, &p); rc != SSD_OK) return rc;
    if (!x || !weight || !state || !y) return SSD_ERR_NULL_ARG;
    p.x = x;
    p.weight = weight;
    p.bias = bias;
    p.fin = state;
    p.y[0] = y;
    return status(ssd::launch_conv_step(p, prob->dtype == SSD_DTYPE_BF16, static_cast<hipStream_t>(stream)));
}

extern "C" int ssd_scan_workspace_bytes(const ssd_scan_problem* prob, size_t* bytes)
{
    return scan_bytes(prob, false, bytes);
}

extern "C" int ssd_scan_forward(const ssd_scan_problem* prob, const void* x, const void* dt, const float* A_log,
                                const void* B, const void* C, const float* D, const void* z, const float* dt_bias,
                                const float* initial_states, const int32_t* seq_idx, void* y, float* final_states,
                                void* workspace, size_t workspace_bytes, void* stream)
{
    ssd::ScanParams p;
    if (const int rc = validate_scan(prob, seq_idx != nullptr, false, z != nullptr, &p); rc != SSD_OK) return rc;
    if (!x || !dt || !A_log || !B || !C || !y) return SSD_ERR_NULL_ARG;
    if (!whole_words(p, prob->dtype, B, C) || !aligned(A_log, 16) || !aligned(initial_states, 16) ||
        !aligned(final_states, 16))
        return SSD_ERR_UNSUPPORTED_DIMS;
    const ssd::ScanPlan w = plan(p, false);
    if (workspace_bytes < w.total || (w.total && !workspace)) return SSD_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return SSD_ERR_UNSUPPORTED_DIMS;
    place(w, workspace, &p);
    p.x = x;
    p.dt = dt;
    p.A_log = A_log;
    p.B = B;
    p.C = C;
    p.D = D;
    p.z = z;
    p.dt_bias = dt_bias;
    p.init = initial_states;
    p.seq_idx = seq_idx;
    p.y = y;
    p.fin = final_states;
    return status(ssd::launch_scan_forward(p, prob->dtype == SSD_DTYPE_BF16, static_cast<hipStream_t>(stream)));
}

extern "C" int ssd_scan_backward_workspace_bytes(const ssd_scan_problem* prob, size_t* bytes)
{
    return scan_bytes(prob, true, bytes);
}

extern "C" int ssd_scan_backward(const ssd_scan_problem* prob, const void* x, const void* dt, const float* A_log,
                                 const void* B, const void* C, const float* D, const void* z, const float* dt_bias,
                                 const float* initial_states, const int32_t* seq_idx, const void* dy,
                                 const float* dfinal_states, void* dx, void* ddt, float* dA_log, void* dB, void* dC,
                                 float* dD, void* dz, float* ddt_bias, float* dinitial_states, void* workspace,
                                 size_t workspace_bytes, void* stream)
{
    ssd::ScanParams p;
    if (const int rc = validate_scan(prob, seq_idx != nullptr, false, z != nullptr, &p); rc != SSD_OK) return rc;
    if (!x || !dt || !A_log || !B || !C || !dy || !dx || !ddt || !dA_log || !dB || !dC || (z && !dz))
        return SSD_ERR_NULL_ARG;
    if (!whole_words(p, prob->dtype, B, C) || !aligned(A_log, 16) || !aligned(initial_states, 16) ||
        !aligned(dfinal_states, 16) || !aligned(dinitial_states, 16))
        return SSD_ERR_UNSUPPORTED_DIMS;
    const ssd::ScanPlan w = plan(p, true);
    if (!workspace || workspace_bytes < w.total) return SSD_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return SSD_ERR_UNSUPPORTED_DIMS;
    place(w, workspace, &p);
    p.x = x;
    p.dt = dt;
    p.A_log = A_log;
    p.B = B;
    p.C = C;
    p.D = D;
    p.z = z;
    p.dt_bias = dt_bias;
    p.init = initial_states;
    p.seq_idx = seq_idx;
    p.dy = dy;
    p.dfin = dfinal_states;
    p.dx = dx;
    p.ddt = ddt;
    p.dA_log = dA_log;
    p.dB = dB;
    p.dC = dC;
    p.dD = D ? dD : nullptr;
    p.dz = z ? dz : nullptr;
    p.ddt_bias = dt_bias ? ddt_bias : nullptr;
    p.dinit = dinitial_states;
    return status(ssd::launch_scan_backward(p, prob->dtype == SSD_DTYPE_BF16, static_cast<hipStream_t>(stream)));
}

extern "C" int ssd_scan_step(const ssd_scan_problem* prob, const void* x, const void* dt, const float* A_log,
                             const void* B, const void* C, const float* D, const void* z, const float* dt_bias,
                             float* state, void* y, void* stream)
{
    ssd::ScanParams p;
    if (const int rc = validate_scan(prob, false, true, z != nullptr, &p); rc != SSD_OK) return rc;
    if (!x || !dt || !A_log || !B || !C || !state || !y) return SSD_ERR_NULL_ARG;
    if (!aligned(state, 16)) return SSD_ERR_UNSUPPORTED_DIMS;
    p.x = x;
    p.dt = dt;
    p.A_log = A_log;
    p.B = B;
    p.C = C;
    p.D = D;
    p.z = z;
    p.dt_bias = dt_bias;
    p.fin = state;
    p.y = y;
    return status(ssd::launch_scan_step(p, prob->dtype == SSD_DTYPE_BF16, static_cast<hipStream_t>(stream)));
}

extern "C" int ssd_add_norm(const ssd_norm_problem* prob, const void* x, const void* residual, const float* weight,
                            void* y, float* scale, void* residual_out, void* stream)
{
    ssd::NormParams p;
    if (const int rc = validate_norm(prob, &p); rc != SSD_OK) return rc;
    const bool q8 = prob->out_dtype == SSD_DTYPE_I8 || prob->out_dtype == SSD_DTYPE_E4M3;
    if (!q8 && prob->out_dtype != prob->dtype) return SSD_ERR_BAD_DTYPE;
    if (!x || !y || (q8 && !scale)) return SSD_ERR_NULL_ARG;
    p.x = x;
    p.res = residual;
    p.weight = weight;
    p.y = y;
    p.scale = scale;
    p.res_out = residual_out;
    const ssd::NormOut out = !q8 ? ssd::kNormSame : prob->out_dtype == SSD_DTYPE_I8 ? ssd::kNormI8 : ssd::kNormE4M3;
    return status(ssd::launch_add_norm(p, prob->dtype == SSD_DTYPE_BF16, prob->residual_dtype == SSD_DTYPE_BF16, out,
                                       static_cast<hipStream_t>(stream)));
}

extern "C" int ssd_add_norm_backward_workspace_bytes(const ssd_norm_problem* prob, size_t* bytes)
{
    if (!bytes) return SSD_ERR_NULL_ARG;
    ssd::NormParams p;
    const int rc = validate_norm(prob, &p);
    if (rc == SSD_OK) *bytes = static_cast<size_t>(ssd::norm_bwd_partials(p.rows, p.C)) * p.C * sizeof(float);
    return rc;
}

extern "C" int ssd_add_norm_backward(const ssd_norm_problem* prob, const void* dy, const void* residual,
                                     const float* weight, const void* dresidual_out, void* dx, void* dresidual,
                                     float* dweight, void* workspace, size_t workspace_bytes, void* stream)
{
    ssd::NormParams p;
    if (const int rc = validate_norm(prob, &p); rc != SSD_OK) return rc;
    if (!dy || !residual || (!dx && !dresidual)) return SSD_ERR_NULL_ARG;
    const size_t need = static_cast<size_t>(ssd::norm_bwd_partials(p.rows, p.C)) * p.C * sizeof(float);
    if (dweight && (!workspace || workspace_bytes < need)) return SSD_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return SSD_ERR_UNSUPPORTED_DIMS;
    p.x = dy;
    p.res = residual;
    p.weight = weight;
    p.dres = dresidual_out;
    p.y = dx;
    p.res_out = dresidual;
    p.dweight = dweight;
    p.partial = dweight ? static_cast<float*>(workspace) : nullptr;
    return status(ssd::launch_add_norm_backward(p, prob->dtype == SSD_DTYPE_BF16,
                                                prob->residual_dtype == SSD_DTYPE_BF16,
                                                static_cast<hipStream_t>(stream)));
}
