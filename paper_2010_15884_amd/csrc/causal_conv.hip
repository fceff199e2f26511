// Short causal convolution of every channel, channels last: forward, gradients, and single tokens.
//
//   pre[t][c] = bias[c] + sum_j w[c][j] x[t-(K-1)+j][c],   y = act(pre)
//   dpre = dy act'(pre);  dx[t] = sum_j w[j] dpre[t+K-1-j];  dw[j] = sum_t dpre[t] x[t-(K-1)+j];  dbias = sum_t dpre[t]
//
// All three are bound by memory: K <= 8 multiply-adds an element beside 4 to 12 bytes.  A lane owns 16 bytes of neighbouring channels
// and walks down the rows, so every load and store of a wavefront is a contiguous piece of a row and the taps stay in registers.
//
// Measured, bf16, 4 taps, SiLU: 2 x 4096 positions x 4096 channels 24.7 us, 5.4 TB/s of the bytes of x and y (a copy of as many: 22 us);
// gradients of 4 x 2048 x 4096 50.5 us, 4.0 TB/s of x, dy and dx (by the profiler about 48 the kernel, 5 the sums of the taps' parts);
// 8 tokens of 2048 channels some 3.5 us, a launch.
#include <type_traits>

#include "launch.h"
#include "sequence.h"

namespace sysconv {
namespace {

constexpr int kThreads = 256;

// The taps of V channels: V * K values in a row of w, [channels][K].
template <typename T, int K, int V>
__device__ __forceinline__ void load_taps(const sys_causal_conv1d_t& p, const void* w, int c0, float (&tap)[K][V])
{
    float flat[V * K];
    load_params<T, V * K>(w, (size_t)c0 * K, p.param_dtype, flat);
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < K; ++j) tap[j][i] = flat[i * K + j];
}

template <typename T, int V>
__device__ __forceinline__ void load_bias(const sys_causal_conv1d_t& p, const void* bias, int c0, float (&b)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) b[i] = 0.0f;
    if (bias) load_params<T, V>(bias, (size_t)c0, p.param_dtype, b);
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
__device__ __forceinline__ typename Channels<T, V>::Raw raw_row(const T* x, const T* state, long long x_row, int channels, int e, int len, int c0)
{
    const int t = e - (K - 1);
    if (t >= 0 && t < len) return Channels<T, V>::raw(x + t * x_row + c0);
    if (t < 0 && e >= 0 && state) return Channels<T, V>::raw(state + (size_t)e * channels + c0);
    return typename Channels<T, V>::Raw{};
}

template <typename T, int K, int V>
__device__ __forceinline__ void load_row(const T* x, const T* state, long long x_row, int channels, int e, int len, int c0, float (&out)[V])
{
    Channels<T, V>::values(raw_row<T, K, V>(x, state, x_row, channels, e, len, c0), out);
}

template <typename T, int K, int V, int ROWS>
__global__ __launch_bounds__(kThreads) void causal_conv_kernel(sys_causal_conv1d_t p, CausalConvArgs a, int blocks_a_sequence, int lanes_a_row)
{
    const unsigned block = xcd_place(blockIdx.x, gridDim.x);
    const int b = block / blocks_a_sequence;
    const int at = (block - b * blocks_a_sequence) * kThreads + threadIdx.x;
    const int chunk = at / lanes_a_row, t0 = chunk * ROWS;
    // the rows past the last one are there for the state behind the sequence
    if (t0 >= p.length && !(t0 == 0 && p.length == 0)) return;
    const int c0 = first_channel<V>(at - chunk * lanes_a_row, p.channels);
    const int len = sequence_length(a.lengths, b, p.length);
    const T* x = (const T*)a.x + b * p.x_batch;
    const T* state = a.state ? (const T*)a.state + (size_t)b * (K - 1) * p.channels : nullptr;
    T* y = (T*)a.y + b * p.y_batch + c0;

    typename Channels<T, V>::Raw raw[K - 1 + ROWS];
    if (t0 >= K - 1 && t0 + ROWS <= len) {
        const T* from = x + (t0 - (K - 1)) * p.x_row + c0;
#pragma unroll
        for (int r = 0; r < K - 1 + ROWS; ++r) raw[r] = Channels<T, V>::raw(from + r * p.x_row);
    } else {
#pragma unroll
        for (int r = 0; r < K - 1 + ROWS; ++r) raw[r] = raw_row<T, K, V>(x, state, p.x_row, p.channels, t0 + r, len, c0);
    }
    float tap[K][V], bias[V], rows[K][V];
    load_taps<T, K, V>(p, a.w, c0, tap);
    load_bias<T, V>(p, a.bias, c0, bias);
#pragma unroll
    for (int j = 0; j + 1 < K; ++j) Channels<T, V>::values(raw[j], rows[j + 1]);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        if (t0 + r >= p.length) break;
#pragma unroll
        for (int j = 0; j + 1 < K; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) rows[j][i] = rows[j + 1][i];
        Channels<T, V>::values(raw[r + K - 1], rows[K - 1]);
        float out[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float pre = bias[i];
#pragma unroll
            for (int j = 0; j < K; ++j) pre = __builtin_fmaf(tap[j][i], rows[j][i], pre);
            out[i] = pre;
        }
        if (p.activation == SYS_ACT_SILU) {
#pragma unroll
            for (int i = 0; i < V; ++i) out[i] = silu(out[i]);
        }
        if (t0 + r >= len) {
#pragma unroll
            for (int i = 0; i < V; ++i) out[i] = 0.0f;
        }
        Channels<T, V>::store_nt(y + (t0 + r) * p.y_row, out);
    }
    // the chunk that holds the last position (the first one of an empty sequence) leaves the state
    const int last = len > 0 ? (len - 1) / ROWS : 0;
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

constexpr int kRun = 32;           // rows a lane in the backward kernel (4 x 2048 x 4096 in bf16, 16 / 32 / 64: 51.8 / 47.3 / 49.6 us)
constexpr int kRunWaves = 4;       // runs a workgroup: a wavefront each, whose sums for the taps are added in LDS
constexpr int kAhead = 2;          // rows whose loads are in flight while as many are worked on (4: 55 us, its registers leave three wavefronts a SIMD;
                                   // 4 and a branch for the activation of every row: 48.6)

// What a lane of the backward kernel carries down the rows.  In rows e of state ++ x, e = 0 .. len+K-2: dext[e] = sum_j w[j] dpre[e-j]
// (dpre is 0 outside 0 .. len-1), plus the gradient of the state behind the sequence in its last K-1 rows; the first K-1 rows are the
// gradient of the state before it.  Going down the rows, dpre[e] needs rows e .. e+K-1 of state ++ x, and dext[e] the last K values of
// dpre, so one window of each moves along.  A run begins K-1 rows early to fill the window of dpre.
template <typename T, int K, int V>
struct GradWindow {
    float tap[K][V], bias[V];
    float rows[K][V], dpre[K][V];      // rows e .. e+K-1; dpre[e-(K-1)] .. dpre[e]
    float sums[K + 1][V];              // of the taps and the bias

    // the windows move on by a row: next is row e+K-1 of state ++ x
    __device__ __forceinline__ void move(typename Channels<T, V>::Raw next)
    {
#pragma unroll
        for (int j = 0; j + 1 < K; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) rows[j][i] = rows[j + 1][i], dpre[j][i] = dpre[j + 1][i];
        Channels<T, V>::values(next, rows[K - 1]);
    }
    template <bool SILU>
    __device__ __forceinline__ void differentiate(typename Channels<T, V>::Raw dy)
    {
        Channels<T, V>::values(dy, dpre[K - 1]);
        if (!SILU) return;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float pre = bias[i];
#pragma unroll
            for (int j = 0; j < K; ++j) pre = __builtin_fmaf(tap[j][i], rows[j][i], pre);
            dpre[K - 1][i] *= silu_grad(pre);
        }
    }
    __device__ __forceinline__ void nothing()
    {
#pragma unroll
        for (int i = 0; i < V; ++i) dpre[K - 1][i] = 0.0f;
    }
    __device__ __forceinline__ void add()
    {
#pragma unroll
        for (int i = 0; i < V; ++i) {
#pragma unroll
            for (int j = 0; j < K; ++j) sums[j][i] = __builtin_fmaf(dpre[K - 1][i], rows[j][i], sums[j][i]);
            sums[K][i] += dpre[K - 1][i];
        }
    }
    __device__ __forceinline__ void output(float (&out)[V]) const
    {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            out[i] = 0.0f;
#pragma unroll
            for (int j = 0; j < K; ++j) out[i] = __builtin_fmaf(tap[j][i], dpre[K - 1 - j][i], out[i]);
        }
    }
};

// Rows begin .. end-1 of dext.  WHOLE: every row of x and dy that they need exists, and none is a state's; else each is asked for (the
// same for all lanes of a wavefront).  Either way kAhead rows are in flight while as many are worked on.
template <typename T, int K, int V, bool WHOLE, bool SILU>
__device__ __forceinline__ void grad_run(const sys_causal_conv1d_t& p, const CausalConvArgs& a, GradWindow<T, K, V>& w, const T* x, const T* dy, const T* state,
                                         int b, int c0, int len, int begin, int end)
{
    typedef Channels<T, V> C;
    const T* dstate_out = a.dstate_out ? (const T*)a.dstate_out + (size_t)b * (K - 1) * p.channels + c0 : nullptr;
    T* dstate = a.dstate ? (T*)a.dstate + (size_t)b * (K - 1) * p.channels + c0 : nullptr;
    T* dx = (T*)a.dx + (size_t)b * p.length * p.channels + c0;
    const T* whole_x = x + (begin - (K - 1)) * p.x_row + c0;           // row `begin` of state ++ x
    const T* whole_dy = dy + begin * p.y_row;
    auto load_x = [&](int e) { return WHOLE ? C::raw(whole_x + (e - begin) * p.x_row) : raw_row<T, K, V>(x, state, p.x_row, p.channels, e, len, c0); };
    auto load_dy = [&](int e) { return WHOLE || (e >= 0 && e < len) ? C::raw(WHOLE ? whole_dy + (e - begin) * p.y_row : dy + e * p.y_row) : typename C::Raw{}; };
    const int zero_from = len ? len + K - 1 : 0;                       // rows that no dpre reaches (0 times an infinite tap would be a NaN)
    typename C::Raw first[K - 1], more[K - 1], more_dy[K - 1], ahead[kAhead], ahead_dy[kAhead];
#pragma unroll
    for (int j = 0; j < K - 1; ++j) {
        first[j] = load_x(begin - (K - 1) + j);
        more[j] = load_x(begin + j);
        more_dy[j] = load_dy(begin - (K - 1) + j);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) ahead[k] = load_x(begin + K - 1 + k), ahead_dy[k] = load_dy(begin + k);
#pragma unroll
    for (int j = 0; j < K - 1; ++j) C::values(first[j], w.rows[j + 1]);
#pragma unroll
    for (int j = 0; j < K - 1; ++j) {
        w.move(more[j]);
        const int e = begin - (K - 1) + j;
        if (WHOLE || (e >= 0 && e < len)) w.template differentiate<SILU>(more_dy[j]);
        else w.nothing();              // (the derivative times a dy of 0 may be a NaN)
    }
    for (int e0 = begin; e0 < end; e0 += kAhead) {
        typename C::Raw now[kAhead], now_dy[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) now[k] = ahead[k], now_dy[k] = ahead_dy[k];
        const int next = !WHOLE || e0 + kAhead < end ? e0 + kAhead : e0;            // (the last round loads its own rows once more)
#pragma unroll
        for (int k = 0; k < kAhead; ++k) ahead[k] = load_x(next + K - 1 + k), ahead_dy[k] = load_dy(next + k);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int e = e0 + k;
            w.move(now[k]);
            float out[V];
            if (WHOLE || (e >= 0 && e < len)) {
                w.template differentiate<SILU>(now_dy[k]);
                w.add();               // (0 * a row that holds a NaN would be one)
            } else {
                w.nothing();
            }
            w.output(out);
            if (WHOLE) {
                C::store_nt(dx + (size_t)(e - (K - 1)) * p.channels, out);
                continue;
            }
            if (e >= end) break;
            if (e >= zero_from) {
#pragma unroll
                for (int i = 0; i < V; ++i) out[i] = 0.0f;
            }
            if (dstate_out && e >= len && e < len + K - 1) {
                float tail[V];
                C::load(dstate_out + (size_t)(e - len) * p.channels, tail);
#pragma unroll
                for (int i = 0; i < V; ++i) out[i] += tail[i];
            }
            if (e >= K - 1) C::store_nt(dx + (size_t)(e - (K - 1)) * p.channels, out);
            else if (dstate) C::store(dstate + (size_t)e * p.channels, out);
        }
    }
}

template <typename T, int K, int V>
__global__ __launch_bounds__(kRunWaves * 64) void causal_conv_grad_kernel(sys_causal_conv1d_t p, CausalConvArgs a, int runs, int groups_a_sequence, int lane_blocks)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lanes_a_row = (p.channels + V - 1) / V;
    const unsigned block = xcd_place(blockIdx.x, gridDim.x);
    const int lane_block = block % lane_blocks;
    const int rest = block / lane_blocks;
    const int b = rest / groups_a_sequence, group = rest - b * groups_a_sequence;
    const int run = group * kRunWaves + wave;
    const int channel_lane = lane_block * 64 + lane;
    const bool there = channel_lane < lanes_a_row && run < runs;
    const int c0 = first_channel<V>(channel_lane < lanes_a_row ? channel_lane : 0, p.channels);
    const int len = sequence_length(a.lengths, b, p.length);
    const T* x = (const T*)a.x + b * p.x_batch;
    const T* dy = (const T*)a.dy + b * p.y_batch + c0;
    const T* state = a.state ? (const T*)a.state + (size_t)b * (K - 1) * p.channels : nullptr;

    GradWindow<T, K, V> w;
#pragma unroll
    for (int j = 0; j <= K; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) w.sums[j][i] = 0.0f;
    if (there) {
        load_taps<T, K, V>(p, a.w, c0, w.tap);
        load_bias<T, V>(p, a.bias, c0, w.bias);
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) w.dpre[j][i] = w.rows[j][i] = 0.0f;
        // the last run goes on through the K-1 rows behind the sequence
        const int begin = run * kRun;
        auto go = [&](auto silu_there) {
            constexpr bool kSilu = decltype(silu_there)::value;
            if (begin >= 2 * (K - 1) && begin + kRun <= len && run != runs - 1) grad_run<T, K, V, true, kSilu>(p, a, w, x, dy, state, b, c0, len, begin, begin + kRun);
            else grad_run<T, K, V, false, kSilu>(p, a, w, x, dy, state, b, c0, len, begin, run == runs - 1 ? p.length + K - 1 : begin + kRun);
        };
        if (p.activation == SYS_ACT_SILU) go(std::true_type());
        else go(std::false_type());
    }

    // the workgroup's sums, [K+1][channels] a workgroup
    __shared__ float shared[kRunWaves][64 * V];
    float* to = a.workspace + (size_t)(b * groups_a_sequence + group) * (K + 1) * p.channels;
#pragma unroll
    for (int j = 0; j <= K; ++j) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) shared[wave][i * 64 + lane] = w.sums[j][i];
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
    load_taps<T, K, V>(p, a.w, c0, tap);
    load_bias<T, V>(p, a.bias, c0, bias);
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

// Channels a lane of the forward kernel.
int lane_channels(const sys_causal_conv1d_t& p)
{
    const int v = p.dtype == SYS_F32 ? kLaneChannels<float> : kLaneChannels<f16_t>;
    return p.channels >= v ? v : 1;
}

int runs_of(const sys_causal_conv1d_t& p) { return p.length ? (p.length + kRun - 1) / kRun : 1; }
int run_groups_of(const sys_causal_conv1d_t& p) { return (runs_of(p) + kRunWaves - 1) / kRunWaves; }

template <typename T, int K, int V, int ROWS>
hipError_t launch_rows(const sys_causal_conv1d_t& p, const CausalConvArgs& a, hipStream_t s)
{
    const int lanes = (p.channels + V - 1) / V;
    const long long chunks = p.length ? (p.length + ROWS - 1) / ROWS : 1;
    const long long blocks = (chunks * lanes + kThreads - 1) / kThreads;
    if (chunks * lanes > 0x7fffffffLL - kThreads || blocks * p.batch > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((causal_conv_kernel<T, K, V, ROWS>), dim3((unsigned)(blocks * p.batch)), dim3(kThreads), 0, s, p, a, (int)blocks, lanes);
    return hipGetLastError();
}

template <typename T, int K, int V>
hipError_t launch_forward(const sys_causal_conv1d_t& p, const CausalConvArgs& a, hipStream_t s)
{
    return causal_conv_rows_a_lane(p) == 16 ? launch_rows<T, K, V, 16>(p, a, s) : launch_rows<T, K, V, 4>(p, a, s);
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
    case kForward: return lane_channels(p) == V ? launch_forward<T, K, V>(p, a, s) : launch_forward<T, K, 1>(p, a, s);
    // half as wide: the windows, taps and sums of 16 bytes take 230 registers (4 taps; level in time) or more than there are (8)
    case kBackward: return p.channels >= V / 2 ? launch_backward<T, K, V / 2>(p, a, s) : launch_backward<T, K, 1>(p, a, s);
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

// 16 rows read the K-1 rows above a chunk the least often, where they leave three wavefronts a SIMD, 4 leave the most (K = 4 in bf16, 4 / 8 / 16 rows:
// 1 x 2048 x 1024 3.8 / 4.8 / 6.8 us, 4 x 1024 x 2048 8.0 / 8.8 / 9.1, 8 x 2048 x 1024 14.2 / 14.1 / 14.6, 4 x 4096 x 2048 26.6 / 25.3 / 24.3).
int causal_conv_rows_a_lane(const sys_causal_conv1d_t& p)
{
    const int v = lane_channels(p);
    const double waves = (double)p.batch * p.length * ((p.channels + v - 1) / v) / (16 * 64);
    return waves >= 3 * 1024 ? 16 : 4;
}

hipError_t launch_causal_conv(const sys_causal_conv1d_t& p, const CausalConvArgs& a, hipStream_t s) { return launch(kForward, p, a, s); }
hipError_t launch_causal_conv_grad(const sys_causal_conv1d_t& p, const CausalConvArgs& a, hipStream_t s) { return launch(kBackward, p, a, s); }
hipError_t launch_causal_conv_step(const sys_causal_conv1d_t& p, const CausalConvArgs& a, hipStream_t s) { return launch(kStep, p, a, s); }

size_t causal_conv_grad_workspace(const sys_causal_conv1d_t& p)
{
    return (size_t)run_groups_of(p) * p.batch * (p.width + 1) * p.channels * sizeof(float);
}

}  // namespace sysconv
