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

// ---------------------------------------------------------------- norm of queries and keys

int check(const sys_head_norm_t& p, bool writes_y)
{
    if (p.batch < 0 || p.length < 0 || p.q_heads < 1 || p.k_heads < 0 || p.dim < 1 || p.positions < 0 || !(p.eps >= 0.0f)) return SYS_ERR_SIZE;
    if (p.rotary < 0 || p.rotary > p.dim || p.rotary % 2) return SYS_ERR_SIZE;
    for (long long s : {p.q_batch, p.q_row, p.k_batch, p.k_row, p.yq_batch, p.yq_row, p.yk_batch, p.yk_row})
        if (bad_stride(s)) return SYS_ERR_SIZE;
    if (p.dim > SYS_MAX_HEAD_DIM || p.q_heads > kMostChannels / p.dim || p.k_heads > kMostChannels / p.dim) return SYS_ERR_UNSUPPORTED;
    if (writes_y && rows_meet(p.batch, p.length, (long long)p.q_heads * p.dim, p.yq_batch, p.yq_row)) return SYS_ERR_SIZE;
    if (writes_y && p.k_heads && rows_meet(p.batch, p.length, (long long)p.k_heads * p.dim, p.yk_batch, p.yk_row)) return SYS_ERR_SIZE;
    if (!known_dtype(p.dtype) || (p.param_dtype != p.dtype && p.param_dtype != SYS_F32)) return SYS_ERR_UNSUPPORTED;
    if ((p.norm != SYS_NORM_RMS && p.norm != SYS_NORM_L2) || (p.interleaved != 0 && p.interleaved != 1)) return SYS_ERR_UNSUPPORTED;
    return p.length > kMostRows ? SYS_ERR_UNSUPPORTED : SYS_OK;
}

// The tables of a call that turns something.
int check_tables(const sys_head_norm_t& p, bool some, const void* cosine, const void* sine, const void* positions)
{
    if (!p.rotary || !some) return SYS_OK;
    if (!positions && p.length > p.positions) return SYS_ERR_SIZE;
    return p.positions && (!cosine || !sine) ? SYS_ERR_NULL : SYS_OK;
}

// ---------------------------------------------------------------- gated delta rule

int check(const sys_gated_delta_t& p, bool step, bool writes_y)
{
    if (p.batch < 0 || p.length < 0 || p.key_heads < 1 || p.value_heads < 1 || p.key_dim < 1 || p.value_dim < 1 || (step && p.slots < 0)) return SYS_ERR_SIZE;
    if (p.value_heads % p.key_heads) return SYS_ERR_SIZE;
    for (long long s : {p.q_batch, p.q_row, p.k_batch, p.k_row, p.v_batch, p.v_row, p.delta_batch, p.delta_row, p.beta_batch, p.beta_row, p.y_batch, p.y_row})
        if (bad_stride(s)) return SYS_ERR_SIZE;
    if (p.key_dim > SYS_MAX_KEY_DIM || p.value_dim > SYS_MAX_VALUE_DIM) return SYS_ERR_UNSUPPORTED;
    if (p.value_heads > kMostChannels / p.value_dim || p.key_heads > kMostChannels / p.key_dim) return SYS_ERR_UNSUPPORTED;
    const long long columns = (long long)p.value_heads * p.value_dim;
    if (writes_y && (step ? rows_meet(1, p.batch, columns, 0, p.y_batch) : rows_meet(p.batch, p.length, columns, p.y_batch, p.y_row))) return SYS_ERR_SIZE;
    if (!known_dtype(p.dtype) || (p.softplus != 0 && p.softplus != 1) || (p.sigmoid != 0 && p.sigmoid != 1) || p.reserved) return SYS_ERR_UNSUPPORTED;
    if (p.length > kMostRows) return SYS_ERR_UNSUPPORTED;
    if (!step && p.length > 1)
        for (long long s : {p.q_row, p.k_row, p.v_row, p.delta_row, p.beta_row, p.y_row})
            if (s > SYS_MAX_DELTA_ROW) return SYS_ERR_UNSUPPORTED;
    return SYS_OK;
}

// What every form of the rule reads; rows: positions of a sequence (1 for single tokens, whose row strides mean nothing).
void delta_inputs(Ranges& r, const sys_gated_delta_t& p, long long rows, const void* q, const void* k, const void* v, const void* delta, const float* a,
                  const void* beta, const float* delta_bias)
{
    const size_t e = bytes_of(p.dtype);
    const long long keys = (long long)p.key_heads * p.key_dim, values = (long long)p.value_heads * p.value_dim;
    r.in(q, extent(p.batch, rows, keys, p.q_batch, p.q_row), e);
    r.in(k, extent(p.batch, rows, keys, p.k_batch, p.k_row), e);
    r.in(v, extent(p.batch, rows, values, p.v_batch, p.v_row), e);
    r.in(delta, extent(p.batch, rows, p.value_heads, p.delta_batch, p.delta_row), e);
    r.in(beta, extent(p.batch, rows, p.value_heads, p.beta_batch, p.beta_row), e);
    r.in(a, p.value_heads, sizeof(float));
    r.in(delta_bias, p.value_heads, sizeof(float));
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

int sys_head_norm(const sys_head_norm_t* p, const void* d_q, const void* d_k, const void* d_wq, const void* d_wk, const float* d_cos, const float* d_sin,
                  const int* d_positions, const int* d_lengths, void* d_yq, void* d_yk, hipStream_t stream)
{
    if (!p) return SYS_ERR_NULL;
    int st = check(*p, true);
    if (st != SYS_OK) return st;
    const bool some = p->batch > 0 && p->length > 0;
    if (some && (!d_q || !d_yq || (p->k_heads && (!d_k || !d_yk)))) return SYS_ERR_NULL;
    if ((st = check_tables(*p, some, d_cos, d_sin, d_positions)) != SYS_OK) return st;
    const size_t e = bytes_of(p->dtype), pe = bytes_of(p->param_dtype);
    const long long q_columns = (long long)p->q_heads * p->dim, k_columns = (long long)p->k_heads * p->dim;
    const Wide table = (Wide)p->positions * (p->rotary / 2);
    Ranges r;
    r.in(d_q, extent(p->batch, p->length, q_columns, p->q_batch, p->q_row), e);
    r.in(d_k, extent(p->batch, p->length, k_columns, p->k_batch, p->k_row), e);
    r.in(d_wq, p->dim, pe);
    r.in(d_wk, p->dim, pe);
    r.in(d_cos, table, sizeof(float));
    r.in(d_sin, table, sizeof(float));
    r.in(d_positions, (Wide)p->batch * p->length, sizeof(int));
    r.in(d_lengths, p->batch, sizeof(int));
    r.out(d_yq, extent(p->batch, p->length, q_columns, p->yq_batch, p->yq_row), e);
    r.out(d_yk, extent(p->batch, p->length, k_columns, p->yk_batch, p->yk_row), e);
    if ((st = check(r)) != SYS_OK || !some) return st;
    sysconv::HeadNormArgs a = {};
    a.q = d_q, a.k = d_k, a.wq = d_wq, a.wk = d_wk, a.cosine = d_cos, a.sine = d_sin, a.positions = d_positions, a.lengths = d_lengths, a.yq = d_yq, a.yk = d_yk;
    return hip_status(sysconv::launch_head_norm(*p, a, stream));
}

int sys_head_norm_backward(const sys_head_norm_t* p, const void* d_dyq, const void* d_dyk, const void* d_q, const void* d_k, const void* d_wq,
                           const void* d_wk, const float* d_cos, const float* d_sin, const int* d_positions, const int* d_lengths, void* d_dq, void* d_dk,
                           void* d_dwq, void* d_dwk, void* d_workspace, hipStream_t stream)
{
    if (!p) return SYS_ERR_NULL;
    int st = check(*p, false);
    if (st != SYS_OK) return st;
    const bool some = p->batch > 0 && p->length > 0;
    const size_t need = sys_head_norm_backward_workspace(p);
    if (some && (!d_dyq || !d_q || !d_dq || (p->k_heads && (!d_dyk || !d_k || !d_dk)))) return SYS_ERR_NULL;
    if ((need && !d_workspace && (d_dwq || d_dwk)) || (d_dwq && !d_wq) || (d_dwk && (!d_wk || !p->k_heads))) return SYS_ERR_NULL;
    if ((st = check_tables(*p, some, d_cos, d_sin, d_positions)) != SYS_OK) return st;
    const size_t e = bytes_of(p->dtype), pe = bytes_of(p->param_dtype);
    const long long q_columns = (long long)p->q_heads * p->dim, k_columns = (long long)p->k_heads * p->dim;
    const Wide table = (Wide)p->positions * (p->rotary / 2);
    Ranges r;
    r.in(d_dyq, extent(p->batch, p->length, q_columns, p->yq_batch, p->yq_row), e);
    r.in(d_dyk, extent(p->batch, p->length, k_columns, p->yk_batch, p->yk_row), e);
    r.in(d_q, extent(p->batch, p->length, q_columns, p->q_batch, p->q_row), e);
    r.in(d_k, extent(p->batch, p->length, k_columns, p->k_batch, p->k_row), e);
    r.in(d_wq, p->dim, pe);
    r.in(d_wk, p->dim, pe);
    r.in(d_cos, table, sizeof(float));
    r.in(d_sin, table, sizeof(float));
    r.in(d_positions, (Wide)p->batch * p->length, sizeof(int));
    r.in(d_lengths, p->batch, sizeof(int));
    r.out(d_dq, (Wide)p->batch * p->length * q_columns, e);
    r.out(d_dk, (Wide)p->batch * p->length * k_columns, e);
    r.out(d_dwq, p->dim, pe);
    r.out(d_dwk, p->dim, pe);
    r.workspace(d_workspace, need);
    if ((st = check(r)) != SYS_OK || (!some && !d_dwq && !d_dwk)) return st;
    sysconv::HeadNormArgs a = {};
    a.q = d_q, a.k = d_k, a.wq = d_wq, a.wk = d_wk, a.dyq = d_dyq, a.dyk = d_dyk, a.cosine = d_cos, a.sine = d_sin, a.positions = d_positions;
    a.lengths = d_lengths, a.yq = d_dq, a.yk = d_dk, a.dwq = d_dwq, a.dwk = d_dwk, a.workspace = (float*)d_workspace;
    return hip_status(sysconv::launch_head_norm_grad(*p, a, stream));
}

size_t sys_head_norm_backward_workspace(const sys_head_norm_t* p)
{
    return p && check(*p, false) == SYS_OK ? sysconv::head_norm_grad_workspace(*p) : 0;
}

int sys_gated_delta_rule(const sys_gated_delta_t* p, const void* d_q, const void* d_k, const void* d_v, const void* d_delta, const float* d_A,
                         const void* d_beta, const float* d_delta_bias, const float* d_state, const int* d_lengths, void* d_y, float* d_state_out,
                         void* d_workspace, hipStream_t stream)
{
    if (!p) return SYS_ERR_NULL;
    int st = check(*p, false, true);
    if (st != SYS_OK) return st;
    const bool some = p->batch > 0 && p->length > 0;
    const size_t need = sys_gated_delta_rule_workspace(p);
    if (!d_A || (some && (!d_q || !d_k || !d_v || !d_delta || !d_beta || !d_y)) || (need && !d_workspace)) return SYS_ERR_NULL;
    const Wide state = (Wide)p->batch * p->value_heads * p->key_dim * p->value_dim;
    Ranges r;
    delta_inputs(r, *p, p->length, d_q, d_k, d_v, d_delta, d_A, d_beta, d_delta_bias);
    r.in(d_state, state, sizeof(float));
    r.in(d_lengths, p->batch, sizeof(int));
    r.out(d_y, extent(p->batch, p->length, (long long)p->value_heads * p->value_dim, p->y_batch, p->y_row), bytes_of(p->dtype));
    r.out(d_state_out, state, sizeof(float));
    r.workspace(d_workspace, need);
    if ((st = check(r)) != SYS_OK || !p->batch) return st;
    sysconv::DeltaArgs a = {};
    a.q = d_q, a.k = d_k, a.v = d_v, a.delta = d_delta, a.beta = d_beta, a.a = d_A, a.delta_bias = d_delta_bias, a.state = d_state, a.lengths = d_lengths;
    a.y = d_y, a.state_out = d_state_out, a.workspace = d_workspace;
    return hip_status(sysconv::launch_delta(*p, a, stream));
}

int sys_gated_delta_rule_backward(const sys_gated_delta_t* p, const void* d_dy, const void* d_q, const void* d_k, const void* d_v, const void* d_delta,
                                  const float* d_A, const void* d_beta, const float* d_delta_bias, const float* d_state, const int* d_lengths,
                                  const float* d_dstate_out, void* d_dq, void* d_dk, void* d_dv, void* d_ddelta, float* d_dA, void* d_dbeta,
                                  float* d_ddelta_bias, float* d_dstate, void* d_workspace, hipStream_t stream)
{
    if (!p) return SYS_ERR_NULL;
    int st = check(*p, false, false);
    if (st != SYS_OK) return st;
    const bool some = p->batch > 0 && p->length > 0;
    const size_t need = sys_gated_delta_rule_backward_workspace(p);
    if (!d_A || !d_dA || (some && (!d_dy || !d_q || !d_k || !d_v || !d_delta || !d_beta || !d_dq || !d_dk || !d_dv || !d_ddelta || !d_dbeta))) return SYS_ERR_NULL;
    if ((need && !d_workspace) || (d_ddelta_bias && !d_delta_bias) || (d_dstate && !d_state)) return SYS_ERR_NULL;
    const size_t e = bytes_of(p->dtype);
    const Wide state = (Wide)p->batch * p->value_heads * p->key_dim * p->value_dim, rows = (Wide)p->batch * p->length;
    const long long keys = (long long)p->key_heads * p->key_dim, values = (long long)p->value_heads * p->value_dim;
    Ranges r;
    delta_inputs(r, *p, p->length, d_q, d_k, d_v, d_delta, d_A, d_beta, d_delta_bias);
    r.in(d_dy, extent(p->batch, p->length, values, p->y_batch, p->y_row), e);
    r.in(d_state, state, sizeof(float));
    r.in(d_lengths, p->batch, sizeof(int));
    r.in(d_dstate_out, state, sizeof(float));
    r.out(d_dq, rows * keys, e);
    r.out(d_dk, rows * keys, e);
    r.out(d_dv, rows * values, e);
    r.out(d_ddelta, rows * p->value_heads, e);
    r.out(d_dA, p->value_heads, sizeof(float));
    r.out(d_dbeta, rows * p->value_heads, e);
    r.out(d_ddelta_bias, p->value_heads, sizeof(float));
    r.out(d_dstate, state, sizeof(float));
    r.workspace(d_workspace, need);
    if ((st = check(r)) != SYS_OK) return st;
    sysconv::DeltaArgs a = {};
    a.q = d_q, a.k = d_k, a.v = d_v, a.delta = d_delta, a.beta = d_beta, a.a = d_A, a.delta_bias = d_delta_bias, a.state = d_state, a.lengths = d_lengths;
    a.dy = d_dy, a.dstate_out = d_dstate_out, a.dq = d_dq, a.dk = d_dk, a.dv = d_dv, a.ddelta = d_ddelta, a.da = d_dA, a.dbeta = d_dbeta;
    a.ddelta_bias = d_ddelta_bias, a.dstate = d_dstate, a.workspace = d_workspace;
    return hip_status(sysconv::launch_delta_grad(*p, a, stream));
}

size_t sys_gated_delta_rule_backward_workspace(const sys_gated_delta_t* p)
{
    return p && check(*p, false, false) == SYS_OK ? sysconv::delta_grad_workspace(*p) : 0;
}

size_t sys_gated_delta_rule_workspace(const sys_gated_delta_t* p)
{
    return p && check(*p, false, false) == SYS_OK ? sysconv::delta_workspace(*p) : 0;
}

int sys_gated_delta_rule_update(const sys_gated_delta_t* p, const void* d_q, const void* d_k, const void* d_v, const void* d_delta, const float* d_A,
                                const void* d_beta, const float* d_delta_bias, const float* d_state, const int* d_slots, void* d_y, float* d_state_out,
                                hipStream_t stream)
{
    if (!p) return SYS_ERR_NULL;
    int st = check(*p, true, true);
    if (st != SYS_OK) return st;
    if (!d_slots && p->slots < p->batch) return SYS_ERR_SIZE;
    if (!d_A || (p->batch && (!d_q || !d_k || !d_v || !d_delta || !d_beta || !d_y)) || (p->slots && (!d_state || !d_state_out))) return SYS_ERR_NULL;
    const Wide state = (Wide)p->slots * p->value_heads * p->key_dim * p->value_dim;
    Ranges r;
    delta_inputs(r, *p, 1, d_q, d_k, d_v, d_delta, d_A, d_beta, d_delta_bias);
    if (d_state != d_state_out) r.in(d_state, state, sizeof(float));
    r.in(d_slots, p->batch, sizeof(int));
    r.out(d_y, extent(1, p->batch, (long long)p->value_heads * p->value_dim, 0, p->y_batch), bytes_of(p->dtype));
    r.out(d_state_out, state, sizeof(float));
    if ((st = check(r)) != SYS_OK || !p->batch) return st;
    sysconv::DeltaArgs a = {};
    a.q = d_q, a.k = d_k, a.v = d_v, a.delta = d_delta, a.beta = d_beta, a.a = d_A, a.delta_bias = d_delta_bias, a.state = d_state, a.slots = d_slots;
    a.y = d_y, a.state_out = d_state_out;
    return hip_status(sysconv::launch_delta_step(*p, a, stream));
}

}  // extern "C"
