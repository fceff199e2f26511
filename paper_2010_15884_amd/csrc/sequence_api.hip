// C-ABI layer of the operators on channels-last sequences: argument validation and status reporting.  Every check runs before the
// first HIP call, so the error paths work on a host without a GPU.
#include "sysconv.h"

#include "launch.h"
#include "sequence.h"

#include <initializer_list>

namespace {

using sysconv::hip_status;

typedef unsigned __int128 Wide;

constexpr int kMostRows = 1 << 30;                 // int arithmetic on positions rounds up to whole tiles
constexpr int kMostChannels = 1 << 24;
constexpr long long kMostStride = 1LL << 40;

bool known_dtype(int t) { return t == SYS_F32 || t == SYS_F16 || t == SYS_BF16; }
size_t bytes_of(int dtype) { return dtype == SYS_F32 ? 4 : 2; }

// Address ranges of a call: what is written must meet nothing else.
struct Ranges {
    static constexpr int kMost = 24;
    uintptr_t from[kMost], to[kMost];
    bool written[kMost];
    int count = 0;
    bool misaligned = false;

    void add(const void* p, Wide elements, size_t element, bool out)
    {
        if (!p) return;
        if ((uintptr_t)p % element) misaligned = true;
        if (!elements) return;
        from[count] = (uintptr_t)p;
        const Wide end = (Wide)(uintptr_t)p + elements * element;
        to[count] = end > (Wide)UINTPTR_MAX ? UINTPTR_MAX : (uintptr_t)end;
        written[count++] = out;
    }
    void in(const void* p, Wide elements, size_t element) { add(p, elements, element, false); }
    void out(const void* p, Wide elements, size_t element) { add(p, elements, element, true); }
    // One that is given though none is needed is held apart as well: whether a misplaced one is refused does not depend on the sizes.
    void workspace(const void* p, size_t bytes) { add(p, bytes ? bytes / sizeof(float) : 1, sizeof(float), true); }

    bool overlap() const
    {
        for (int i = 0; i < count; ++i)
            for (int j = i + 1; j < count; ++j)
                if ((written[i] || written[j]) && from[i] < to[j] && from[j] < to[i]) return true;
        return false;
    }
};

// Elements from the first to the last of a [batch, rows, columns] tensor with these strides.
Wide extent(long long batch, long long rows, long long columns, long long batch_stride, long long row_stride)
{
    if (batch < 1 || rows < 1 || columns < 1) return 0;
    return (Wide)(batch - 1) * (Wide)batch_stride + (Wide)(rows - 1) * (Wide)row_stride + (Wide)columns;
}

bool bad_stride(long long s) { return s < 0 || s > kMostStride; }

// Rows of an output that overlap.
bool rows_meet(long long batch, long long rows, long long columns, long long batch_stride, long long row_stride)
{
    if (rows > 1 && row_stride < columns) return true;
    return batch > 1 && rows > 0 && (Wide)batch_stride < extent(1, rows, columns, 0, row_stride);
}

// ---------------------------------------------------------------- causal convolution

int check(const sys_causal_conv1d_t& p, bool step, bool writes_y)
{
    if (p.batch < 0 || p.length < 0 || p.channels < 1 || (step && p.slots < 0)) return SYS_ERR_SIZE;
    if (bad_stride(p.x_batch) || bad_stride(p.x_row) || bad_stride(p.y_batch) || bad_stride(p.y_row)) return SYS_ERR_SIZE;
    if (writes_y && (step ? rows_meet(1, p.batch, p.channels, 0, p.y_batch) : rows_meet(p.batch, p.length, p.channels, p.y_batch, p.y_row))) return SYS_ERR_SIZE;
    if (!known_dtype(p.dtype) || (p.param_dtype != p.dtype && p.param_dtype != SYS_F32)) return SYS_ERR_UNSUPPORTED;
    if (p.activation != SYS_ACT_NONE && p.activation != SYS_ACT_SILU) return SYS_ERR_UNSUPPORTED;
    if (p.width < 2 || p.width > SYS_MAX_CAUSAL_WIDTH) return SYS_ERR_UNSUPPORTED;
    if (p.length > kMostRows || p.channels > kMostChannels) return SYS_ERR_UNSUPPORTED;
    return SYS_OK;
}

// ---------------------------------------------------------------- selective scan

int check(const sys_selective_scan_t& p, bool step, bool writes_y)
{
    if (p.batch < 0 || p.length < 0 || p.channels < 1 || p.states < 1 || p.groups < 1 || (step && p.slots < 0)) return SYS_ERR_SIZE;
    if (p.channels % p.groups) return SYS_ERR_SIZE;
    const long long strides[] = {p.u_batch, p.u_row, p.delta_batch, p.delta_row, p.z_batch, p.z_row, p.b_batch, p.b_row, p.c_batch, p.c_row, p.y_batch, p.y_row};
    for (long long s : strides)
        if (bad_stride(s)) return SYS_ERR_SIZE;
    if (writes_y && (step ? rows_meet(1, p.batch, p.channels, 0, p.y_batch) : rows_meet(p.batch, p.length, p.channels, p.y_batch, p.y_row))) return SYS_ERR_SIZE;
    if (!known_dtype(p.dtype) || (p.softplus != 0 && p.softplus != 1) || p.states > SYS_MAX_STATES) return SYS_ERR_UNSUPPORTED;
    if (p.length > kMostRows || p.channels > kMostChannels) return SYS_ERR_UNSUPPORTED;
    if (!step && p.length > 1)
        for (long long s : {p.u_row, p.delta_row, p.z_row, p.b_row, p.c_row, p.y_row})
            if (s > SYS_MAX_SCAN_ROW) return SYS_ERR_UNSUPPORTED;
    return SYS_OK;
}

// ---------------------------------------------------------------- group norm

int check(const sys_group_norm_t& p, bool writes_y)
{
    if (p.batch < 0 || p.rows < 1 || p.channels < 1 || p.groups < 1 || p.channels % p.groups || !(p.eps >= 0.0f)) return SYS_ERR_SIZE;
    if (bad_stride(p.x_batch) || bad_stride(p.x_row) || bad_stride(p.y_batch) || bad_stride(p.y_row)) return SYS_ERR_SIZE;
    if (writes_y && rows_meet(p.batch, p.rows, p.channels, p.y_batch, p.y_row)) return SYS_ERR_SIZE;
    if (!known_dtype(p.dtype) || (p.param_dtype != p.dtype && p.param_dtype != SYS_F32)) return SYS_ERR_UNSUPPORTED;
    if (p.activation < SYS_ACT_NONE || p.activation > SYS_ACT_RELU || p.reserved) return SYS_ERR_UNSUPPORTED;
    if (p.rows > kMostStride || p.channels > kMostChannels) return SYS_ERR_UNSUPPORTED;
    return SYS_OK;
}

// The addresses of a call, after its sizes: SYS_OK if it may run.
int check(const Ranges& r)
{
    if (r.misaligned) return SYS_ERR_UNSUPPORTED;
    return r.overlap() ? SYS_ERR_ALIAS : SYS_OK;
}

}  // namespace

extern "C" {

int sys_causal_conv1d(const sys_causal_conv1d_t* p, const void* d_x, const void* d_w, const void* d_bias, const void* d_state, const int* d_lengths,
                      void* d_y, void* d_state_out, hipStream_t stream)
{
    if (!p) return SYS_ERR_NULL;
    int st = check(*p, false, true);
    if (st != SYS_OK) return st;
    const bool some = p->batch > 0 && p->length > 0;
    if (!d_w || (some && (!d_x || !d_y))) return SYS_ERR_NULL;
    const size_t e = bytes_of(p->dtype), pe = bytes_of(p->param_dtype);
    const Wide state = (Wide)p->batch * (p->width - 1) * p->channels;
    Ranges r;
    r.in(d_x, extent(p->batch, p->length, p->channels, p->x_batch, p->x_row), e);
    r.in(d_w, (Wide)p->channels * p->width, pe);
    r.in(d_bias, p->channels, pe);
    r.in(d_state, state, e);
    r.in(d_lengths, p->batch, sizeof(int));
    r.out(d_y, extent(p->batch, p->length, p->channels, p->y_batch, p->y_row), e);
    r.out(d_state_out, state, e);
    if ((st = check(r)) != SYS_OK || !p->batch) return st;
    sysconv::CausalConvArgs a = {};
    a.x = d_x, a.w = d_w, a.bias = d_bias, a.state = d_state, a.lengths = d_lengths, a.y = d_y, a.state_out = d_state_out;
    return hip_status(sysconv::launch_causal_conv(*p, a, stream));
}

int sys_causal_conv1d_backward(const sys_causal_conv1d_t* p, const void* d_dy, const void* d_x, const void* d_w, const void* d_bias, const void* d_state,
                               const int* d_lengths, const void* d_dstate_out, void* d_dx, void* d_dw, void* d_dbias, void* d_dstate, void* d_workspace,
                               hipStream_t stream)
{
    if (!p) return SYS_ERR_NULL;
    int st = check(*p, false, false);
    if (st != SYS_OK) return st;
    const bool some = p->batch > 0 && p->length > 0;
    const size_t need = sys_causal_conv1d_backward_workspace(p);
    if (!d_w || !d_dw || (some && (!d_dy || !d_x || !d_dx)) || (need && !d_workspace) || (d_dbias && !d_bias) || (d_dstate && !d_state)) return SYS_ERR_NULL;
    const size_t e = bytes_of(p->dtype), pe = bytes_of(p->param_dtype);
    const Wide state = (Wide)p->batch * (p->width - 1) * p->channels;
    Ranges r;
    r.in(d_dy, extent(p->batch, p->length, p->channels, p->y_batch, p->y_row), e);
    r.in(d_x, extent(p->batch, p->length, p->channels, p->x_batch, p->x_row), e);
    r.in(d_w, (Wide)p->channels * p->width, pe);
    r.in(d_bias, p->channels, pe);
    r.in(d_state, state, e);
    r.in(d_lengths, p->batch, sizeof(int));
    r.in(d_dstate_out, state, e);
    r.out(d_dx, (Wide)p->batch * p->length * p->channels, e);
    r.out(d_dw, (Wide)p->channels * p->width, pe);
    r.out(d_dbias, p->channels, pe);
    r.out(d_dstate, state, e);
    r.workspace(d_workspace, need);
    if ((st = check(r)) != SYS_OK) return st;
    sysconv::CausalConvArgs a = {};
    a.dy = d_dy, a.x = d_x, a.w = d_w, a.bias = d_bias, a.state = d_state, a.lengths = d_lengths, a.dstate_out = d_dstate_out;
    a.dx = d_dx, a.dw = d_dw, a.dbias = d_dbias, a.dstate = d_dstate, a.workspace = (float*)d_workspace;
    return hip_status(sysconv::launch_causal_conv_grad(*p, a, stream));
}

size_t sys_causal_conv1d_backward_workspace(const sys_causal_conv1d_t* p)
{
    return p && check(*p, false, false) == SYS_OK ? sysconv::causal_conv_grad_workspace(*p) : 0;
}

int sys_causal_conv1d_update(const sys_causal_conv1d_t* p, const void* d_x, const void* d_w, const void* d_bias, const void* d_state, const int* d_slots,
                             void* d_y, void* d_state_out, hipStream_t stream)
{
    if (!p) return SYS_ERR_NULL;
    int st = check(*p, true, true);
    if (st != SYS_OK) return st;
    if (!d_slots && p->slots < p->batch) return SYS_ERR_SIZE;
    if (!d_w || (p->batch && (!d_x || !d_y)) || (p->slots && (!d_state || !d_state_out))) return SYS_ERR_NULL;
    const size_t e = bytes_of(p->dtype), pe = bytes_of(p->param_dtype);
    const Wide state = (Wide)p->slots * (p->width - 1) * p->channels;
    Ranges r;
    r.in(d_x, extent(1, p->batch, p->channels, 0, p->x_batch), e);
    r.in(d_w, (Wide)p->channels * p->width, pe);
    r.in(d_bias, p->channels, pe);
    if (d_state != d_state_out) r.in(d_state, state, e);
    r.in(d_slots, p->batch, sizeof(int));
    r.out(d_y, extent(1, p->batch, p->channels, 0, p->y_batch), e);
    r.out(d_state_out, state, e);
    if ((st = check(r)) != SYS_OK || !p->batch) return st;
    sysconv::CausalConvArgs a = {};
    a.x = d_x, a.w = d_w, a.bias = d_bias, a.state = d_state, a.slots = d_slots, a.y = d_y, a.state_out = d_state_out;
    return hip_status(sysconv::launch_causal_conv_step(*p, a, stream));
}

int sys_selective_scan(const sys_selective_scan_t* p, const void* d_u, const void* d_delta, const float* d_A, const void* d_B, const void* d_C,
                       const float* d_D, const void* d_z, const float* d_delta_bias, const float* d_state, const int* d_lengths, void* d_y,
                       float* d_state_out, void* d_workspace, hipStream_t stream)
{
    if (!p) return SYS_ERR_NULL;
    int st = check(*p, false, true);
    if (st != SYS_OK) return st;
    const bool some = p->batch > 0 && p->length > 0;
    const size_t need = sys_selective_scan_workspace(p);
    if (!d_A || (some && (!d_u || !d_delta || !d_B || !d_C || !d_y)) || (need && !d_workspace)) return SYS_ERR_NULL;
    const size_t e = bytes_of(p->dtype);
    const Wide state = (Wide)p->batch * p->channels * p->states;
    const long long row = (long long)p->groups * p->states;
    Ranges r;
    r.in(d_u, extent(p->batch, p->length, p->channels, p->u_batch, p->u_row), e);
    r.in(d_delta, extent(p->batch, p->length, p->channels, p->delta_batch, p->delta_row), e);
    r.in(d_z, extent(p->batch, p->length, p->channels, p->z_batch, p->z_row), e);
    r.in(d_B, extent(p->batch, p->length, row, p->b_batch, p->b_row), e);
    r.in(d_C, extent(p->batch, p->length, row, p->c_batch, p->c_row), e);
    r.in(d_A, (Wide)p->channels * p->states, sizeof(float));
    r.in(d_D, p->channels, sizeof(float));
    r.in(d_delta_bias, p->channels, sizeof(float));
    r.in(d_state, state, sizeof(float));
    r.in(d_lengths, p->batch, sizeof(int));
    r.out(d_y, extent(p->batch, p->length, p->channels, p->y_batch, p->y_row), e);
    r.out(d_state_out, state, sizeof(float));
    r.workspace(d_workspace, need);
    if ((st = check(r)) != SYS_OK || !p->batch) return st;
    sysconv::ScanArgs a = {};
    a.u = d_u, a.delta = d_delta, a.a = d_A, a.b = d_B, a.c = d_C, a.d = d_D, a.z = d_z, a.delta_bias = d_delta_bias, a.state = d_state;
    a.lengths = d_lengths, a.y = d_y, a.state_out = d_state_out, a.workspace = (float*)d_workspace;
    return hip_status(sysconv::launch_scan(*p, a, stream));
}

size_t sys_selective_scan_workspace(const sys_selective_scan_t* p)
{
    return p && check(*p, false, false) == SYS_OK ? sysconv::scan_workspace(*p) : 0;
}

int sys_selective_scan_backward(const sys_selective_scan_t* p, const void* d_dy, const void* d_u, const void* d_delta, const float* d_A, const void* d_B,
                                const void* d_C, const float* d_D, const void* d_z, const float* d_delta_bias, const float* d_state, const int* d_lengths,
                                const float* d_dstate_out, void* d_du, void* d_ddelta, float* d_dA, void* d_dB, void* d_dC, float* d_dD, void* d_dz,
                                float* d_ddelta_bias, float* d_dstate, void* d_workspace, hipStream_t stream)
{
    if (!p) return SYS_ERR_NULL;
    int st = check(*p, false, false);
    if (st != SYS_OK) return st;
    const bool some = p->batch > 0 && p->length > 0;
    const size_t need = sys_selective_scan_backward_workspace(p);
    if (!d_A || !d_dA || (some && (!d_dy || !d_u || !d_delta || !d_B || !d_C || !d_du || !d_ddelta || !d_dB || !d_dC)) || (need && !d_workspace)) return SYS_ERR_NULL;
    if ((d_dD && !d_D) || (d_ddelta_bias && !d_delta_bias) || (d_dstate && !d_state) || (some && !d_z != !d_dz)) return SYS_ERR_NULL;
    const size_t e = bytes_of(p->dtype);
    const Wide state = (Wide)p->batch * p->channels * p->states, values = (Wide)p->batch * p->length * p->channels;
    const long long row = (long long)p->groups * p->states;
    Ranges r;
    r.in(d_dy, extent(p->batch, p->length, p->channels, p->y_batch, p->y_row), e);
    r.in(d_u, extent(p->batch, p->length, p->channels, p->u_batch, p->u_row), e);
    r.in(d_delta, extent(p->batch, p->length, p->channels, p->delta_batch, p->delta_row), e);
    r.in(d_z, extent(p->batch, p->length, p->channels, p->z_batch, p->z_row), e);
    r.in(d_B, extent(p->batch, p->length, row, p->b_batch, p->b_row), e);
    r.in(d_C, extent(p->batch, p->length, row, p->c_batch, p->c_row), e);
    r.in(d_A, (Wide)p->channels * p->states, sizeof(float));
    r.in(d_D, p->channels, sizeof(float));
    r.in(d_delta_bias, p->channels, sizeof(float));
    r.in(d_state, state, sizeof(float));
    r.in(d_lengths, p->batch, sizeof(int));
    r.in(d_dstate_out, state, sizeof(float));
    r.out(d_du, values, e);
    r.out(d_ddelta, values, e);
    r.out(d_dA, (Wide)p->channels * p->states, sizeof(float));
    r.out(d_dB, (Wide)p->batch * p->length * row, e);
    r.out(d_dC, (Wide)p->batch * p->length * row, e);
    r.out(d_dD, p->channels, sizeof(float));
    r.out(d_dz, values, e);
    r.out(d_ddelta_bias, p->channels, sizeof(float));
    r.out(d_dstate, state, sizeof(float));
    r.workspace(d_workspace, need);
    if ((st = check(r)) != SYS_OK) return st;
    sysconv::ScanArgs a = {};
    a.dy = d_dy, a.u = d_u, a.delta = d_delta, a.a = d_A, a.b = d_B, a.c = d_C, a.d = d_D, a.z = d_z, a.delta_bias = d_delta_bias, a.state = d_state;
    a.lengths = d_lengths, a.dstate_out = d_dstate_out, a.du = d_du, a.ddelta = d_ddelta, a.da = d_dA, a.db = d_dB, a.dc = d_dC, a.dd = d_dD;
    a.dz = d_dz, a.ddelta_bias = d_ddelta_bias, a.dstate = d_dstate, a.workspace = (float*)d_workspace;
    return hip_status(sysconv::launch_scan_grad(*p, a, stream));
}

size_t sys_selective_scan_backward_workspace(const sys_selective_scan_t* p)
{
    return p && check(*p, false, false) == SYS_OK ? sysconv::scan_grad_workspace(*p) : 0;
}

int sys_selective_scan_update(const sys_selective_scan_t* p, const void* d_u, const void* d_delta, const float* d_A, const void* d_B, const void* d_C,
                              const float* d_D, const void* d_z, const float* d_delta_bias, const float* d_state, const int* d_slots, void* d_y,
                              float* d_state_out, hipStream_t stream)
{
    if (!p) return SYS_ERR_NULL;
    int st = check(*p, true, true);
    if (st != SYS_OK) return st;
    if (!d_slots && p->slots < p->batch) return SYS_ERR_SIZE;
    if (!d_A || (p->batch && (!d_u || !d_delta || !d_B || !d_C || !d_y)) || (p->slots && (!d_state || !d_state_out))) return SYS_ERR_NULL;
    const size_t e = bytes_of(p->dtype);
    const Wide state = (Wide)p->slots * p->channels * p->states;
    const long long row = (long long)p->groups * p->states;
    Ranges r;
    r.in(d_u, extent(1, p->batch, p->channels, 0, p->u_batch), e);
    r.in(d_delta, extent(1, p->batch, p->channels, 0, p->delta_batch), e);
    r.in(d_z, extent(1, p->batch, p->channels, 0, p->z_batch), e);
    r.in(d_B, extent(1, p->batch, row, 0, p->b_batch), e);
    r.in(d_C, extent(1, p->batch, row, 0, p->c_batch), e);
    r.in(d_A, (Wide)p->channels * p->states, sizeof(float));
    r.in(d_D, p->channels, sizeof(float));
    r.in(d_delta_bias, p->channels, sizeof(float));
    if (d_state != d_state_out) r.in(d_state, state, sizeof(float));
    r.in(d_slots, p->batch, sizeof(int));
    r.out(d_y, extent(1, p->batch, p->channels, 0, p->y_batch), e);
    r.out(d_state_out, state, sizeof(float));
    if ((st = check(r)) != SYS_OK || !p->batch) return st;
    sysconv::ScanArgs a = {};
    a.u = d_u, a.delta = d_delta, a.a = d_A, a.b = d_B, a.c = d_C, a.d = d_D, a.z = d_z, a.delta_bias = d_delta_bias, a.state = d_state;
    a.slots = d_slots, a.y = d_y, a.state_out = d_state_out;
    return hip_status(sysconv::launch_scan_step(*p, a, stream));
}

int sys_group_norm(const sys_group_norm_t* p, const void* d_x, const void* d_w, const void* d_b, void* d_y, float* d_mean, float* d_rstd,
                   void* d_workspace, hipStream_t stream)
{
    if (!p) return SYS_ERR_NULL;
    int st = check(*p, true);
    if (st != SYS_OK) return st;
    const size_t need = sys_group_norm_workspace(p);
    if ((p->batch && (!d_x || !d_y)) || (need && !d_workspace)) return SYS_ERR_NULL;
    const size_t e = bytes_of(p->dtype), pe = bytes_of(p->param_dtype);
    const Wide groups = (Wide)p->batch * p->groups;
    Ranges r;
    r.in(d_x, extent(p->batch, p->rows, p->channels, p->x_batch, p->x_row), e);
    r.in(d_w, p->channels, pe);
    r.in(d_b, p->channels, pe);
    r.out(d_y, extent(p->batch, p->rows, p->channels, p->y_batch, p->y_row), e);
    r.out(d_mean, groups, sizeof(float));
    r.out(d_rstd, groups, sizeof(float));
    r.workspace(d_workspace, need);
    if ((st = check(r)) != SYS_OK || !p->batch) return st;
    sysconv::NormArgs a = {};
    a.x = d_x, a.w = d_w, a.b = d_b, a.y = d_y, a.mean = d_mean, a.rstd = d_rstd, a.workspace = (float*)d_workspace;
    return hip_status(sysconv::launch_group_norm(*p, a, stream));
}

size_t sys_group_norm_workspace(const sys_group_norm_t* p)
{
    return p && check(*p, false) == SYS_OK ? sysconv::group_norm_workspace(*p) : 0;
}

int sys_group_norm_backward(const sys_group_norm_t* p, const void* d_dy, const void* d_x, const void* d_w, const void* d_b, const float* d_mean,
                            const float* d_rstd, void* d_dx, void* d_dw, void* d_db, void* d_workspace, hipStream_t stream)
{
    if (!p) return SYS_ERR_NULL;
    int st = check(*p, false);
    if (st != SYS_OK) return st;
    const size_t need = sys_group_norm_backward_workspace(p);
    if ((p->batch && (!d_dy || !d_x || !d_mean || !d_rstd || !d_dx)) || (need && !d_workspace) || (d_dw && !d_w) || (d_db && !d_b)) return SYS_ERR_NULL;
    const size_t e = bytes_of(p->dtype), pe = bytes_of(p->param_dtype);
    const Wide groups = (Wide)p->batch * p->groups;
    Ranges r;
    r.in(d_dy, extent(p->batch, p->rows, p->channels, p->y_batch, p->y_row), e);
    r.in(d_x, extent(p->batch, p->rows, p->channels, p->x_batch, p->x_row), e);
    r.in(d_w, p->channels, pe);
    r.in(d_b, p->channels, pe);
    r.in(d_mean, groups, sizeof(float));
    r.in(d_rstd, groups, sizeof(float));
    r.out(d_dx, (Wide)p->batch * (Wide)p->rows * p->channels, e);
    r.out(d_dw, p->channels, pe);
    r.out(d_db, p->channels, pe);
    r.workspace(d_workspace, need);
    if ((st = check(r)) != SYS_OK) return st;
    sysconv::NormArgs a = {};
    a.dy = d_dy, a.x = d_x, a.w = d_w, a.b = d_b, a.mean_in = d_mean, a.rstd_in = d_rstd, a.dx = d_dx, a.dw = d_dw, a.db = d_db;
    a.workspace = (float*)d_workspace;
    return hip_status(sysconv::launch_group_norm_grad(*p, a, stream));
}

size_t sys_group_norm_backward_workspace(const sys_group_norm_t* p)
{
    return p && check(*p, false) == SYS_OK ? sysconv::group_norm_grad_workspace(*p) : 0;
}

}  // extern "C"
