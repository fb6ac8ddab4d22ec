// C ABI of the forecasting operators: argument validation, workspace carving, launches.
#include <string.h>

#include "themis_forecast_internal.h"

namespace themis {
namespace {

constexpr size_t kAlign = 256;
inline size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }

int done(cudaError_t e) { return e == cudaSuccess ? THEMIS_OK : record_cuda_error(e); }

inline size_t size_of(int32_t dtype) { return dtype == THEMIS_DTYPE_F32 ? 4 : 2; }

// --- selective scan ---------------------------------------------------------------------------

int validate_ssm(const themis_ssm_problem_t *pr, bool step = false)
{
    if (!pr) return THEMIS_E_INVALID_ARG;
    if (pr->batch < 0 || pr->length < 0 || pr->channels < 1 || pr->state < 1 || pr->groups < 1) return THEMIS_E_INVALID_ARG;
    if (pr->channels % pr->groups != 0) return THEMIS_E_INVALID_ARG;
    if (pr->dtype < THEMIS_DTYPE_F32 || pr->dtype > THEMIS_DTYPE_F16 || pr->flags != 0) return THEMIS_E_INVALID_ARG;
    const int64_t strides[] = {pr->x_row, pr->x_time, pr->dt_row, pr->dt_time, pr->z_row, pr->z_time,
                               pr->b_row, pr->b_time, pr->b_group, pr->c_row, pr->c_time, pr->c_group};
    for (int64_t s : strides)
        if (s < 0) return THEMIS_E_INVALID_ARG;
    if (pr->state > THEMIS_SSM_MAX_STATE) return THEMIS_E_UNSUPPORTED_SIZE;
    if (pr->conv_width < THEMIS_SSM_MIN_CONV || pr->conv_width > THEMIS_SSM_MAX_CONV) return THEMIS_E_UNSUPPORTED_SIZE;
    if (!step && pr->length > (1 << 30)) return THEMIS_E_UNSUPPORTED_SIZE;    // times are 32-bit, up to the end of the last part
    if (pr->channels > 65535) return THEMIS_E_UNSUPPORTED_SIZE;      // tiles of channels are a grid's second axis
    return THEMIS_OK;
}

bool inputs_ok(const themis_ssm_inputs_t *in)
{
    return in && in->x && in->dt && in->b && in->c && in->a && in->conv_weight;
}

// Fills the split plan and the workspace pointers (base may be NULL: sizes only).
size_t carve_ssm(const themis_ssm_problem_t *pr, bool backward, char *base, SsmParams *p)
{
    if (backward) ssm_backward_plan(pr, p);
    else ssm_forward_plan(pr, p);
    size_t off = 0;
    auto take = [&](size_t floats) {
        float *at = base ? reinterpret_cast<float *>(base + off) : nullptr;
        off = align_up(off + floats * sizeof(float));
        return at;
    };
    const size_t B = pr->batch, D = pr->channels, N = pr->state, W = pr->conv_width;
    if (p->splits > 1) {
        p->split_state = take(B * p->splits * D * N);
        p->split_step = take(B * p->splits * D);
    }
    if (backward) {
        p->part_par = take(B * p->splits * D * (N + 8));
        p->part_bc = take((size_t)p->tiles_per_group * B * pr->length * pr->groups * 2 * N);
        if (p->splits > 1) {
            p->conv_head = take(B * p->splits * (W - 1) * D);
            p->conv_tail = take(B * p->splits * (W - 1) * D);
        }
    }
    return off;
}

int check_workspace(size_t need, const void *ws, size_t bytes)
{
    if (need == 0) return THEMIS_OK;
    if (!ws || ((uintptr_t)ws & (kAlign - 1))) return THEMIS_E_INVALID_ARG;
    return bytes < need ? THEMIS_E_WORKSPACE_TOO_SMALL : THEMIS_OK;
}

// one thread per element in blocks of 256 along a grid's first axis
bool grid_fits(double elements) { return elements / 256 < 2147483647.0; }

cudaError_t copy_or_clear(void *to, const void *from, size_t bytes, cudaStream_t st)
{
    if (!to || bytes == 0) return cudaSuccess;
    return from ? cudaMemcpyAsync(to, from, bytes, cudaMemcpyDeviceToDevice, st) : cudaMemsetAsync(to, 0, bytes, st);
}

// --- linear -----------------------------------------------------------------------------------

int validate_linear(const themis_linear_problem_t *pr)
{
    if (!pr) return THEMIS_E_INVALID_ARG;
    if (pr->rows < 0 || pr->out_features < 1 || pr->in_features < 1) return THEMIS_E_INVALID_ARG;
    if ((pr->dtype != THEMIS_DTYPE_BF16 && pr->dtype != THEMIS_DTYPE_F16) || pr->flags != 0) return THEMIS_E_INVALID_ARG;
    if (pr->activation < THEMIS_ACT_NONE || pr->activation > THEMIS_ACT_GELU) return THEMIS_E_INVALID_ARG;
    if (pr->x_row < pr->in_features || pr->weight_row < pr->in_features || pr->residual_row < pr->out_features ||
        pr->dy_row < pr->out_features)
        return THEMIS_E_INVALID_ARG;
    // row counts of the tensor maps and of the tiles are 32-bit; leaves room to round up
    if (pr->rows > (1 << 30) || pr->out_features > (1 << 24) || pr->in_features > (1 << 24)) return THEMIS_E_UNSUPPORTED_SIZE;
    return THEMIS_OK;
}

inline bool unaligned(const void *a, const void *b, const void *c)
{
    return (((uintptr_t)a | (uintptr_t)b | (uintptr_t)c) & 15u) != 0;
}

}  // namespace
}  // namespace themis

using namespace themis;

extern "C" {

int themis_ssm_checkpoints(const themis_ssm_problem_t *problem, int32_t *out_count)
{
    int rc = validate_ssm(problem);
    if (rc != THEMIS_OK) return rc;
    if (!out_count) return THEMIS_E_INVALID_ARG;
    *out_count = (problem->length + THEMIS_SSM_CHUNK - 1) / THEMIS_SSM_CHUNK;
    return THEMIS_OK;
}

int themis_ssm_workspace_bytes(const themis_ssm_problem_t *problem, int backward, size_t *out_bytes)
{
    int rc = validate_ssm(problem);
    if (rc != THEMIS_OK) return rc;
    if (!out_bytes) return THEMIS_E_INVALID_ARG;
    SsmParams p;
    memset(&p, 0, sizeof(p));
    *out_bytes = problem->batch > 0 && problem->length > 0 ? carve_ssm(problem, backward != 0, nullptr, &p) : 0;
    return THEMIS_OK;
}

int themis_ssm_forward(const themis_ssm_problem_t *problem, const themis_ssm_inputs_t *in,
                       const themis_ssm_outputs_t *out, void *d_workspace, size_t workspace_bytes, void *cuda_stream)
{
    int rc = validate_ssm(problem);
    if (rc != THEMIS_OK) return rc;
    if (!in || !out) return THEMIS_E_INVALID_ARG;
    // parts of a row run at the same time: a state must not change while another part reads it
    if (out->ssm_state && out->ssm_state == in->ssm_state) return THEMIS_E_INVALID_ARG;
    if (out->conv_state && out->conv_state == in->conv_state) return THEMIS_E_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const size_t rows = problem->batch, D = problem->channels;
    if (problem->batch == 0 || problem->length == 0) {
        cudaError_t e = copy_or_clear(out->ssm_state, in->ssm_state, rows * D * problem->state * sizeof(float), st);
        if (e == cudaSuccess)
            e = copy_or_clear(out->conv_state, in->conv_state, rows * D * (problem->conv_width - 1) * size_of(problem->dtype), st);
        return done(e);
    }
    if (!inputs_ok(in) || !out->y) return THEMIS_E_INVALID_ARG;
    SsmParams p;
    memset(&p, 0, sizeof(p));
    p.pr = *problem;
    p.in = *in;
    p.out = *out;
    rc = check_workspace(carve_ssm(problem, false, static_cast<char *>(d_workspace), &p), d_workspace, workspace_bytes);
    if (rc != THEMIS_OK) return rc;
    return done(launch_ssm_forward(p, st));
}

int themis_ssm_backward(const themis_ssm_problem_t *problem, const themis_ssm_inputs_t *in, const float *checkpoints,
                        const void *dy, const themis_ssm_grads_t *grads, void *d_workspace, size_t workspace_bytes,
                        void *cuda_stream)
{
    int rc = validate_ssm(problem);
    if (rc != THEMIS_OK) return rc;
    if (!in || !grads) return THEMIS_E_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (problem->batch == 0 || problem->length == 0) {
        const size_t D = problem->channels;
        cudaError_t e = copy_or_clear(grads->a, nullptr, D * problem->state * sizeof(float), st);
        if (e == cudaSuccess) e = copy_or_clear(grads->conv_weight, nullptr, D * problem->conv_width * sizeof(float), st);
        if (e == cudaSuccess) e = copy_or_clear(grads->conv_bias, nullptr, D * sizeof(float), st);
        if (e == cudaSuccess) e = copy_or_clear(grads->skip, nullptr, D * sizeof(float), st);
        if (e == cudaSuccess) e = copy_or_clear(grads->dt_bias, nullptr, D * sizeof(float), st);
        return done(e);
    }
    if (!inputs_ok(in) || !checkpoints || !dy || (grads->z && !in->z)) return THEMIS_E_INVALID_ARG;
    if (!grid_fits((double)problem->batch * problem->length * problem->groups * 2 * problem->state)) return THEMIS_E_UNSUPPORTED_SIZE;
    SsmParams p;
    memset(&p, 0, sizeof(p));
    p.pr = *problem;
    p.in = *in;
    p.grads = *grads;
    p.checkpoints = checkpoints;
    p.dy = dy;
    rc = check_workspace(carve_ssm(problem, true, static_cast<char *>(d_workspace), &p), d_workspace, workspace_bytes);
    if (rc != THEMIS_OK) return rc;
    return done(launch_ssm_backward(p, st));
}

int themis_ssm_step(const themis_ssm_problem_t *problem, const themis_ssm_inputs_t *in,
                    const themis_ssm_outputs_t *out, void *cuda_stream)
{
    int rc = validate_ssm(problem, true);
    if (rc != THEMIS_OK) return rc;
    if (!in || !out) return THEMIS_E_INVALID_ARG;
    if (problem->batch == 0) return THEMIS_OK;
    if (!inputs_ok(in) || !in->conv_state || !in->ssm_state || !out->y || !out->conv_state || !out->ssm_state)
        return THEMIS_E_INVALID_ARG;
    if (!grid_fits((double)problem->batch * problem->channels * 16)) return THEMIS_E_UNSUPPORTED_SIZE;
    SsmParams p;
    memset(&p, 0, sizeof(p));
    p.pr = *problem;
    p.in = *in;
    p.out = *out;
    return done(launch_ssm_step(p, static_cast<cudaStream_t>(cuda_stream)));
}

int themis_linear_workspace_bytes(const themis_linear_problem_t *problem, int backward, int is_unaligned, size_t *out_bytes)
{
    int rc = validate_linear(problem);
    if (rc != THEMIS_OK) return rc;
    if (!out_bytes) return THEMIS_E_INVALID_ARG;
    *out_bytes = problem->rows == 0 ? 0
               : backward ? linear_backward_workspace(*problem, is_unaligned != 0)
                          : linear_forward_workspace(*problem, is_unaligned != 0);
    return THEMIS_OK;
}

int themis_linear_forward(const themis_linear_problem_t *problem, const void *d_x, const void *d_weight, const float *d_bias,
                          const void *d_residual, void *d_y, void *d_pre, int32_t *d_status, void *d_workspace,
                          size_t workspace_bytes, void *cuda_stream)
{
    int rc = validate_linear(problem);
    if (rc != THEMIS_OK) return rc;
    if (problem->rows == 0) return THEMIS_OK;
    if (!d_x || !d_weight || !d_y) return THEMIS_E_INVALID_ARG;
    rc = check_workspace(linear_forward_workspace(*problem, unaligned(d_x, d_weight, nullptr)), d_workspace, workspace_bytes);
    if (rc != THEMIS_OK) return rc;
    LinearParams p;
    memset(&p, 0, sizeof(p));
    p.pr = *problem;
    p.x = d_x; p.weight = d_weight; p.bias = d_bias; p.residual = d_residual;
    p.y = d_y; p.pre_out = d_pre; p.status = d_status;
    p.ws = static_cast<char *>(d_workspace);
    return done(launch_linear_forward(p, static_cast<cudaStream_t>(cuda_stream)));
}

int themis_linear_backward(const themis_linear_problem_t *problem, const void *d_dy, const void *d_x, const void *d_weight,
                           const void *d_pre, void *d_dx, void *d_dweight, float *d_dbias, int32_t *d_status,
                           void *d_workspace, size_t workspace_bytes, void *cuda_stream)
{
    int rc = validate_linear(problem);
    if (rc != THEMIS_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (problem->rows == 0) {
        cudaError_t e = copy_or_clear(d_dweight, nullptr, (size_t)problem->out_features * problem->in_features * 2, st);
        if (e == cudaSuccess) e = copy_or_clear(d_dbias, nullptr, (size_t)problem->out_features * sizeof(float), st);
        return done(e);
    }
    if (!d_dy || (d_dx && !d_weight) || (d_dweight && !d_x)) return THEMIS_E_INVALID_ARG;
    if (problem->activation != THEMIS_ACT_NONE && !d_pre) return THEMIS_E_INVALID_ARG;
    rc = check_workspace(linear_backward_workspace(*problem, unaligned(d_dy, d_x, d_weight)), d_workspace, workspace_bytes);
    if (rc != THEMIS_OK) return rc;
    LinearParams p;
    memset(&p, 0, sizeof(p));
    p.pr = *problem;
    p.dy = d_dy; p.x = d_x; p.weight = d_weight; p.pre_in = d_pre;
    p.dx = d_dx; p.dweight = d_dweight; p.dbias = d_dbias; p.status = d_status;
    p.ws = static_cast<char *>(d_workspace);
    return done(launch_linear_backward(p, st));
}

}  // extern "C"
