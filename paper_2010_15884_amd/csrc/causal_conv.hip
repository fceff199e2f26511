// Short causal convolution of every channel, channels last: forward, gradients, and single tokens.
//
//   pre[t][c] = bias[c] + sum_j w[c][j] x[t-(K-1)+j][c],   y = act(pre)
//   dpre = dy act'(pre);  dx[t] = sum_j w[j] dpre[t+K-1-j];  dw[j] = sum_t dpre[t] x[t-(K-1)+j];  dbias = sum_t dpre[t]
//
// All three are bound by memory: K <= 8 multiply-adds an element beside 4 to 12 bytes.  A lane owns 16 bytes of neighbouring channels
// and walks down the rows, so every load and store of a wavefront is a contiguous piece of a row and the taps stay in registers.
#include "launch.h"
#include "sequence.h"

namespace sysconv {
namespace {

constexpr int kThreads = 256;

// The taps of V channels.  w is [channels][K].
template <int K, int V>
__device__ __forceinline__ void load_taps(const sys_causal_conv1d_t& p, const void* w, int c0, float (&tap)[K][V])
{
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < K; ++j) tap[j][i] = load_param(w, (size_t)(c0 + i) * K + j, p.param_dtype);
}

template <int V>
__device__ __forceinline__ void load_bias(const sys_causal_conv1d_t& p, const void* bias, int c0, float (&b)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) b[i] = bias ? load_param(bias, (size_t)c0 + i, p.param_dtype) : 0.0f;
}

// The lanes of a row hold V channels each; the last one begins earlier where the channels are no multiple of V, and both lanes
// that then hold a channel compute and store the same values.
template <int V>
__device__ __forceinline__ int first_channel(int lane, int channels)
{
    const int c = lane * V;
    return c + V <= channels ? c : channels - V;
}

// Row e of state ++ x (e = t + K-1), zeros where there is none.
template <typename T, int K, int V>
__device__ __forceinline__ void load_row(const T* x, const T* state, long long x_row, int channels, int e, int len, int c0, float (&out)[V])
{
    const int t = e - (K - 1);
    if (t >= 0 && t < len) Channels<T, V>::load(x + t * x_row + c0, out);
    else if (t < 0 && e >= 0 && state) Channels<T, V>::load(state + (size_t)e * channels + c0, out);
    else {
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = 0.0f;
    }
}

constexpr int kRows = 8;           // rows a lane in the forward kernel

template <typename T, int K, int V>
__global__ __launch_bounds__(kThreads) void causal_conv_kernel(sys_causal_conv1d_t p, CausalConvArgs a, int blocks_a_sequence, int lanes_a_row)
{
    const int b = blockIdx.x / blocks_a_sequence;
    const int at = (blockIdx.x - b * blocks_a_sequence) * kThreads + threadIdx.x;
    const int chunk = at / lanes_a_row, t0 = chunk * kRows;
    // the rows past the last one are there for the state behind the sequence
    if (t0 >= p.length && !(t0 == 0 && p.length == 0)) return;
    const int c0 = first_channel<V>(at - chunk * lanes_a_row, p.channels);
    const int len = sequence_length(a.lengths, b, p.length);
    const T* x = (const T*)a.x + b * p.x_batch;
    const T* state = a.state ? (const T*)a.state + (size_t)b * (K - 1) * p.channels : nullptr;
    T* y = (T*)a.y + b * p.y_batch + c0;

    float rows[K - 1 + kRows][V];
    if (t0 >= K - 1 && t0 + kRows <= len) {
#pragma unroll
        for (int r = 0; r < K - 1 + kRows; ++r) Channels<T, V>::load(x + (t0 - (K - 1) + r) * p.x_row + c0, rows[r]);
    } else {
#pragma unroll
        for (int r = 0; r < K - 1 + kRows; ++r) load_row<T, K, V>(x, state, p.x_row, p.channels, t0 + r, len, c0, rows[r]);
    }
    float tap[K][V], bias[V];
    load_taps<K, V>(p, a.w, c0, tap);
    load_bias<V>(p, a.bias, c0, bias);
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        if (t0 + r >= p.length) break;
        float out[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float pre = bias[i];
#pragma unroll
            for (int j = 0; j < K; ++j) pre = __builtin_fmaf(tap[j][i], rows[r + j][i], pre);
            out[i] = t0 + r < len ? (p.activation == SYS_ACT_SILU ? silu(pre) : pre) : 0.0f;
        }
        Channels<T, V>::store(y + (t0 + r) * p.y_row, out);
    }
    // the chunk that holds the last position (the first one of an empty sequence) leaves the state
    const int last = len > 0 ? (len - 1) / kRows : 0;
    if (a.state_out && chunk == last) {
        T* s = (T*)a.state_out + (size_t)b * (K - 1) * p.channels + c0;
        for (int j = 0; j < K - 1; ++j) {
            float row[V];
            load_row<T, K, V>(x, state, p.x_row, p.channels, len + j, len, c0, row);
            Channels<T, V>::store(s + (size_t)j * p.channels, row);
        }
    }
}

// ---------------------------------------------------------------- gradients

constexpr int kRun = 64;           // rows a lane in the backward kernel
constexpr int kRunWaves = 4;       // runs a workgroup: a wavefront each, whose sums for the taps are added in LDS

// In rows e of state ++ x, e = 0 .. len+K-2: dext[e] = sum_j w[j] dpre[e-j] (dpre is 0 outside 0 .. len-1), plus the gradient of
// the state behind the sequence in its last K-1 rows; the first K-1 rows are the gradient of the state before it.  Going down
// the rows, dpre[e] needs rows e .. e+K-1 of state ++ x, and dext[e] the last K values of dpre, so one window of each moves
// along.  A run begins K-1 rows early to fill the window of dpre.
template <typename T, int K, int V>
__global__ __launch_bounds__(kRunWaves * 64) void causal_conv_grad_kernel(sys_causal_conv1d_t p, CausalConvArgs a, int runs, int groups_a_sequence, int lane_blocks)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int lanes_a_row = (p.channels + V - 1) / V;
    const int lane_block = blockIdx.x % lane_blocks;
    const int rest = blockIdx.x / lane_blocks;
    const int b = rest / groups_a_sequence, group = rest - b * groups_a_sequence;
    const int run = group * kRunWaves + wave;
    const int channel_lane = lane_block * 64 + lane;
    const bool there = channel_lane < lanes_a_row && run < runs;
    const int c0 = first_channel<V>(channel_lane < lanes_a_row ? channel_lane : 0, p.channels);
    const int len = sequence_length(a.lengths, b, p.length);
    const T* x = (const T*)a.x + b * p.x_batch;
    const T* dy = (const T*)a.dy + b * p.y_batch + c0;
    const T* state = a.state ? (const T*)a.state + (size_t)b * (K - 1) * p.channels : nullptr;
    const T* dstate_out = a.dstate_out ? (const T*)a.dstate_out + (size_t)b * (K - 1) * p.channels + c0 : nullptr;
    T* dstate = a.dstate ? (T*)a.dstate + (size_t)b * (K - 1) * p.channels + c0 : nullptr;
    T* dx = (T*)a.dx + (size_t)b * p.length * p.channels + c0;

    float sums[K + 1][V];              // of the taps and the bias
#pragma unroll
    for (int j = 0; j <= K; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) sums[j][i] = 0.0f;

    if (there) {
        float tap[K][V], bias[V];
        load_taps<K, V>(p, a.w, c0, tap);
        load_bias<V>(p, a.bias, c0, bias);
        const int begin = run * kRun, total = p.length + K - 1;
        const int end = begin + kRun < total ? begin + kRun : total;
        float rows[K][V], dpre[K][V];  // rows e .. e+K-1; dpre[e-(K-1)] .. dpre[e]
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) dpre[j][i] = rows[j][i] = 0.0f;
#pragma unroll
        for (int j = 1; j < K; ++j) load_row<T, K, V>(x, state, p.x_row, p.channels, begin - (K - 1) + j - 1, len, c0, rows[j]);
        for (int e = begin - (K - 1); e < end; ++e) {
            float g[V];
#pragma unroll
            for (int j = 0; j + 1 < K; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) { rows[j][i] = rows[j + 1][i]; dpre[j][i] = dpre[j + 1][i]; }
            load_row<T, K, V>(x, state, p.x_row, p.channels, e + K - 1, len, c0, rows[K - 1]);
            const bool on = e >= 0 && e < len;
            if (on) Channels<T, V>::load(dy + e * p.y_row, g);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float pre = bias[i];
#pragma unroll
                for (int j = 0; j < K; ++j) pre = __builtin_fmaf(tap[j][i], rows[j][i], pre);
                dpre[K - 1][i] = on ? (p.activation == SYS_ACT_SILU ? g[i] * silu_grad(pre) : g[i]) : 0.0f;
            }
            if (e < begin) continue;
            float out[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                out[i] = 0.0f;
#pragma unroll
                for (int j = 0; j < K; ++j) out[i] = __builtin_fmaf(tap[j][i], dpre[K - 1 - j][i], out[i]);
            }
            if (on) {                  // (0 * a row that holds a NaN would be one)
#pragma unroll
                for (int i = 0; i < V; ++i) {
#pragma unroll
                    for (int j = 0; j < K; ++j) sums[j][i] = __builtin_fmaf(dpre[K - 1][i], rows[j][i], sums[j][i]);
                    sums[K][i] += dpre[K - 1][i];
                }
            }
            if (dstate_out && e >= len && e < len + K - 1) {
                float more[V];
                Channels<T, V>::load(dstate_out + (size_t)(e - len) * p.channels, more);
#pragma unroll
                for (int i = 0; i < V; ++i) out[i] += more[i];
            }
            if (e < K - 1) {
                if (dstate) Channels<T, V>::store(dstate + (size_t)e * p.channels, out);
            } else {
                Channels<T, V>::store(dx + (size_t)(e - (K - 1)) * p.channels, out);
            }
        }
    }

    // the workgroup's sums, [K+1][channels] a workgroup
    __shared__ float shared[kRunWaves][64 * V];
    float* to = a.workspace + (size_t)(b * groups_a_sequence + group) * (K + 1) * p.channels;
#pragma unroll
    for (int j = 0; j <= K; ++j) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) shared[wave][i * 64 + lane] = sums[j][i];
        __syncthreads();
        if (wave == 0 && channel_lane < lanes_a_row) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float s = shared[0][i * 64 + lane];
#pragma unroll
                for (int w = 1; w < kRunWaves; ++w) s += shared[w][i * 64 + lane];
                to[(size_t)j * p.channels + c0 + i] = s;
            }
        }
    }
}

// Sums of the parts, in one order: 16 columns x 16 parts a workgroup, then the 16.
__global__ __launch_bounds__(kThreads) void causal_conv_taps_kernel(sys_causal_conv1d_t p, CausalConvArgs a, int parts)
{
    const int column = blockIdx.x * 16 + (threadIdx.x & 15), share = threadIdx.x >> 4;
    const int columns = (p.width + 1) * p.channels;
    float s = 0.0f;
    if (column < columns)
        for (int i = share; i < parts; i += 16) s += a.workspace[(size_t)i * columns + column];
    __shared__ float shared[16][16];
    shared[share][threadIdx.x & 15] = s;
    __syncthreads();
    if (share || column >= columns) return;
    for (int i = 1; i < 16; ++i) s += shared[i][threadIdx.x];
    const int j = column / p.channels, c = column - j * p.channels;
    if (j < p.width) store_param(a.dw, (size_t)c * p.width + j, p.param_dtype, s);
    else if (a.dbias) store_param(a.dbias, c, p.param_dtype, s);
}

// ---------------------------------------------------------------- single tokens

// A lane reads the K-1 rows of its channels and writes them a row further, so a cache may be updated in place.
template <typename T, int K, int V>
__global__ __launch_bounds__(kThreads) void causal_conv_step_kernel(sys_causal_conv1d_t p, CausalConvArgs a, int lanes_a_row)
{
    const long long at = (long long)blockIdx.x * kThreads + threadIdx.x;
    const int r = (int)(at / lanes_a_row);
    if (r >= p.batch) return;
    const int c0 = (int)(at - (long long)r * lanes_a_row) * V;
    const int slot = a.slots ? a.slots[r] : r;
    T* y = (T*)a.y + r * p.y_batch + c0;
    float out[V];
    if (slot < 0 || slot >= p.slots) {
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = 0.0f;
        Channels<T, V>::store(y, out);
        return;
    }
    const size_t base = (size_t)slot * (K - 1) * p.channels + c0;
    float rows[K][V], tap[K][V], bias[V];
#pragma unroll
    for (int j = 0; j + 1 < K; ++j) Channels<T, V>::load((const T*)a.state + base + (size_t)j * p.channels, rows[j]);
    Channels<T, V>::load((const T*)a.x + r * p.x_batch + c0, rows[K - 1]);
    load_taps<K, V>(p, a.w, c0, tap);
    load_bias<V>(p, a.bias, c0, bias);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        float pre = bias[i];
#pragma unroll
        for (int j = 0; j < K; ++j) pre = __builtin_fmaf(tap[j][i], rows[j][i], pre);
        out[i] = p.activation == SYS_ACT_SILU ? silu(pre) : pre;
    }
    Channels<T, V>::store(y, out);
#pragma unroll
    for (int j = 0; j + 1 < K; ++j) Channels<T, V>::store((T*)a.state_out + base + (size_t)j * p.channels, rows[j + 1]);
}

// ---------------------------------------------------------------- launches

int runs_of(const sys_causal_conv1d_t& p) { return (p.length + p.width - 1 + kRun - 1) / kRun; }
int run_groups_of(const sys_causal_conv1d_t& p) { return (runs_of(p) + kRunWaves - 1) / kRunWaves; }

template <typename T, int K, int V>
hipError_t launch_forward(const sys_causal_conv1d_t& p, const CausalConvArgs& a, hipStream_t s)
{
    const int lanes = (p.channels + V - 1) / V;
    const long long chunks = p.length ? (p.length + kRows - 1) / kRows : 1;
    const long long blocks = (chunks * lanes + kThreads - 1) / kThreads;
    if (chunks * lanes > 0x7fffffffLL - kThreads || blocks * p.batch > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((causal_conv_kernel<T, K, V>), dim3((unsigned)(blocks * p.batch)), dim3(kThreads), 0, s, p, a, (int)blocks, lanes);
    return hipGetLastError();
}

template <typename T, int K, int V>
hipError_t launch_backward(const sys_causal_conv1d_t& p, const CausalConvArgs& a, hipStream_t s)
{
    const int lanes = (p.channels + V - 1) / V, lane_blocks = (lanes + 63) / 64, groups = run_groups_of(p);
    const long long blocks = (long long)lane_blocks * groups * p.batch;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    if (blocks) {
        hipLaunchKernelGGL((causal_conv_grad_kernel<T, K, V>), dim3((unsigned)blocks), dim3(kRunWaves * 64), 0, s, p, a, runs_of(p), groups, lane_blocks);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const long long columns = (long long)(p.width + 1) * p.channels;
    hipLaunchKernelGGL(causal_conv_taps_kernel, dim3((unsigned)((columns + 15) / 16)), dim3(kThreads), 0, s, p, a, groups * p.batch);
    return hipGetLastError();
}

template <typename T, int K, int V>
hipError_t launch_step(const sys_causal_conv1d_t& p, const CausalConvArgs& a, hipStream_t s)
{
    const int lanes = p.channels / V;
    const long long blocks = ((long long)lanes * p.batch + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((causal_conv_step_kernel<T, K, V>), dim3((unsigned)blocks), dim3(kThreads), 0, s, p, a, lanes);
    return hipGetLastError();
}

enum Form { kForward, kBackward, kStep };

template <typename T, int K>
hipError_t launch_width(Form form, const sys_causal_conv1d_t& p, const CausalConvArgs& a, hipStream_t s)
{
    constexpr int V = kLaneChannels<T>;
    switch (form) {
    case kForward: return p.channels >= V ? launch_forward<T, K, V>(p, a, s) : launch_forward<T, K, 1>(p, a, s);
    case kBackward: return p.channels >= V ? launch_backward<T, K, V>(p, a, s) : launch_backward<T, K, 1>(p, a, s);
    // lanes that share channels would read states that others have moved on
    default: return p.channels % V == 0 ? launch_step<T, K, V>(p, a, s) : launch_step<T, K, 1>(p, a, s);
    }
}

template <typename T>
hipError_t launch_type(Form form, const sys_causal_conv1d_t& p, const CausalConvArgs& a, hipStream_t s)
{
    switch (p.width) {
    case 2: return launch_width<T, 2>(form, p, a, s);
    case 3: return launch_width<T, 3>(form, p, a, s);
    case 4: return launch_width<T, 4>(form, p, a, s);
    case 5: return launch_width<T, 5>(form, p, a, s);
    case 6: return launch_width<T, 6>(form, p, a, s);
    case 7: return launch_width<T, 7>(form, p, a, s);
    case 8: return launch_width<T, 8>(form, p, a, s);
    default: return hipErrorInvalidValue;
    }
}

hipError_t launch(Form form, const sys_causal_conv1d_t& p, const CausalConvArgs& a, hipStream_t s)
{
    switch (p.dtype) {
    case SYS_F32: return launch_type<float>(form, p, a, s);
    case SYS_F16: return launch_type<f16_t>(form, p, a, s);
    default: return launch_type<bf16_t>(form, p, a, s);
    }
}

}  // namespace

hipError_t launch_causal_conv(const sys_causal_conv1d_t& p, const CausalConvArgs& a, hipStream_t s) { return launch(kForward, p, a, s); }
hipError_t launch_causal_conv_grad(const sys_causal_conv1d_t& p, const CausalConvArgs& a, hipStream_t s) { return launch(kBackward, p, a, s); }
hipError_t launch_causal_conv_step(const sys_causal_conv1d_t& p, const CausalConvArgs& a, hipStream_t s) { return launch(kStep, p, a, s); }

size_t causal_conv_grad_workspace(const sys_causal_conv1d_t& p)
{
    return (size_t)run_groups_of(p) * p.batch * (p.width + 1) * p.channels * sizeof(float);
}

}  // namespace sysconv
