// Group norm with an activation, channels last: y = act((x - mean) rstd w + b), statistics over the rows of a batch entry and the
// channels of a group.  Bound by memory: some ten operations a value beside its bytes.
//
// A lane holds V neighbouring channels of one group (16 bytes, or what divides a group's channels) and walks down the rows.
// Values and squares are never summed as they come, so a mean far from zero costs no digits of the variance: the group's first
// value is taken off every other one, eight differences at a time give their own mean and sum of squared distances, and
// (count, mean, distances) are merged pairwise, n = n1 + n2, mean = mean1 + d n2/n, M2 = M2_1 + M2_2 + d^2 n1 n2/n with
// d = mean2 - mean1 (the first value may be far from all others).
#include "launch.h"
#include "sequence.h"

namespace sysconv {
namespace {

constexpr int kThreads = 256;

struct NormShape {
    int columns;                   // lanes a row: channels / V
    int columns_a_group;
    int chunks;                    // of the rows, a workgroup each
    long long chunk_rows;
};

struct Moments {
    float n, mean, m2;
};

__device__ __forceinline__ Moments merged(Moments a, Moments b)
{
    const float n = a.n + b.n;
    const float share = n > 0.0f ? b.n * fast_rcp(n) : 0.0f, d = b.mean - a.mean;
    return {n, b.n > 0.0f ? __builtin_fmaf(d, share, a.mean) : a.mean, b.n > 0.0f ? a.m2 + b.m2 + d * d * a.n * share : a.m2};
}

__device__ __forceinline__ Moments over_wave(Moments m)
{
    for (int k = 1; k < 64; k <<= 1) m = merged(m, Moments{__shfl_xor(m.n, k), __shfl_xor(m.mean, k), __shfl_xor(m.m2, k)});
    return m;
}

__device__ __forceinline__ float activated(float v, int activation)
{
    if (activation == SYS_ACT_SILU) return silu(v);
    return activation == SYS_ACT_RELU ? (v > 0.0f ? v : v != v ? v : 0.0f) : v;
}

__device__ __forceinline__ float activated_grad(float v, int activation)
{
    if (activation == SYS_ACT_SILU) return silu_grad(v);
    return activation == SYS_ACT_RELU ? (v > 0.0f ? 1.0f : 0.0f) : 1.0f;
}

// Where a lane of a workgroup works: 256 lanes side by side in a row, or several rows of fewer.
struct Lanes {
    int wide, tall, column, row;
    bool there;
    __device__ __forceinline__ Lanes(int columns)
    {
        wide = columns < kThreads ? columns : kThreads;
        tall = kThreads / wide;
        row = (int)threadIdx.x / wide;
        column = (int)threadIdx.x - row * wide;
        there = row < tall;
    }
};

// ---------------------------------------------------------------- forward

// What is taken off a group's values: the first one of the batch entry.
template <typename T>
__device__ __forceinline__ float group_first(const sys_group_norm_t& p, const T* x, int group)
{
    return (float)x[(long long)group * (p.channels / p.groups)];
}

// Moments of every column of a chunk of rows: [batch][chunk][column] Moments.
template <typename T, int V>
__global__ __launch_bounds__(kThreads) void norm_moments_kernel(sys_group_norm_t p, NormArgs a, NormShape shape)
{
    constexpr int kBatchRows = 8 / V;
    const int b = blockIdx.x / shape.chunks, chunk = blockIdx.x - b * shape.chunks;
    const Lanes at(shape.columns);
    const long long begin = chunk * shape.chunk_rows, end = begin + shape.chunk_rows < p.rows ? begin + shape.chunk_rows : p.rows;
    const T* x = (const T*)a.x + b * p.x_batch;
    Moments* to = (Moments*)a.workspace + ((size_t)b * shape.chunks + chunk) * shape.columns;
    __shared__ Moments shared[kThreads];
    for (int c0 = 0; c0 < shape.columns; c0 += at.wide) {
        const int column = c0 + at.column;
        Moments m = {0.0f, 0.0f, 0.0f};
        if (at.there && column < shape.columns) {
            const float first = group_first<T>(p, x, column / shape.columns_a_group);
            for (long long r = begin + at.row; r < end; r += (long long)at.tall * kBatchRows) {
                float v[kBatchRows][V], sum = 0.0f, count = 0.0f, square = 0.0f;
#pragma unroll
                for (int k = 0; k < kBatchRows; ++k) {
                    const bool on = r + (long long)k * at.tall < end;
                    Channels<T, V>::load(x + (on ? r + (long long)k * at.tall : r) * p.x_row + (long long)column * V, v[k]);
                    count += on ? (float)V : 0.0f;
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        v[k][i] -= first;
                        sum += on ? v[k][i] : 0.0f;
                    }
                }
                const float mean = sum * fast_rcp(count);
#pragma unroll
                for (int k = 0; k < kBatchRows; ++k) {
                    const bool on = r + (long long)k * at.tall < end;
#pragma unroll
                    for (int i = 0; i < V; ++i) square += on ? (v[k][i] - mean) * (v[k][i] - mean) : 0.0f;
                }
                m = merged(m, Moments{count, mean, square});
            }
        }
        __syncthreads();
        shared[threadIdx.x] = m;
        __syncthreads();
        if (at.row == 0 && column < shape.columns) {
            for (int k = 1; k < at.tall; ++k) m = merged(m, shared[k * at.wide + at.column]);
            to[column] = m;
        }
    }
}

// mean and rstd of every group, a wavefront each: [batch][group] pairs behind the moments, and the caller's arrays.
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_statistics_kernel(sys_group_norm_t p, NormArgs a, NormShape shape)
{
    const long long at = ((long long)blockIdx.x * kThreads + threadIdx.x) >> 6;
    if (at >= (long long)p.batch * p.groups) return;
    const int b = (int)(at / p.groups), group = (int)(at - (long long)b * p.groups), lane = threadIdx.x & 63;
    const Moments* from = (const Moments*)a.workspace + (size_t)b * shape.chunks * shape.columns + (size_t)group * shape.columns_a_group;
    Moments m = {0.0f, 0.0f, 0.0f};
    const long long all = (long long)shape.chunks * shape.columns_a_group;
    for (long long k = lane; k < all; k += 64) {
        const long long chunk = k / shape.columns_a_group;
        m = merged(m, from[chunk * shape.columns + (k - chunk * shape.columns_a_group)]);
    }
    m = over_wave(m);
    if (lane) return;
    const float rstd = 1.0f / __builtin_sqrtf(m.m2 / m.n + p.eps);
    float* to = (float*)((Moments*)a.workspace + (size_t)p.batch * shape.chunks * shape.columns) + 2 * at;
    const float mean = m.mean + group_first<T>(p, (const T*)a.x + b * p.x_batch, group);
    to[0] = mean;
    to[1] = rstd;
    if (a.mean) a.mean[at] = mean;
    if (a.rstd) a.rstd[at] = rstd;
}

template <typename T, int V>
__global__ __launch_bounds__(kThreads) void norm_apply_kernel(sys_group_norm_t p, NormArgs a, NormShape shape)
{
    const int b = blockIdx.x / shape.chunks, chunk = blockIdx.x - b * shape.chunks;
    const Lanes at(shape.columns);
    if (!at.there) return;
    const long long begin = chunk * shape.chunk_rows, end = begin + shape.chunk_rows < p.rows ? begin + shape.chunk_rows : p.rows;
    const T* x = (const T*)a.x + b * p.x_batch;
    T* y = (T*)a.y + b * p.y_batch;
    const float* statistics = (const float*)((const Moments*)a.workspace + (size_t)p.batch * shape.chunks * shape.columns) + 2 * (size_t)b * p.groups;
    for (int column = at.column; column < shape.columns; column += at.wide) {
        const int group = column / shape.columns_a_group;
        const float mean = statistics[2 * group], rstd = statistics[2 * group + 1];
        float scale[V], shift[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            scale[i] = (a.w ? load_param(a.w, (size_t)column * V + i, p.param_dtype) : 1.0f) * rstd;
            shift[i] = a.b ? load_param(a.b, (size_t)column * V + i, p.param_dtype) : 0.0f;
        }
        for (long long r = begin + at.row; r < end; r += at.tall) {
            float v[V];
            Channels<T, V>::load(x + r * p.x_row + (long long)column * V, v);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = activated(__builtin_fmaf(v[i] - mean, scale[i], shift[i]), p.activation);
            Channels<T, V>::store(y + r * p.y_row + (long long)column * V, v);
        }
    }
}

// ---------------------------------------------------------------- gradients
//
// With hat = (x - mean) rstd and f = dy act'(hat w + b): dw = sum f hat, db = sum f over batch and rows, and
// dx = rstd (f w - m1 - hat m2), m1 = E[f w], m2 = E[f w hat] over the group, which are sums over its channels of w times the entry's db and dw.

// The workspace: where its parts begin, in floats.
struct GradSpace {
    size_t sums;                   // [batch][f | f hat][channel], behind [batch][chunk][f | f hat][channel] at 0
    size_t means;                  // [batch][group][m1, m2]
    size_t floats;
};

__host__ __device__ GradSpace grad_space(const sys_group_norm_t& p, const NormShape& shape)
{
    GradSpace g;
    g.sums = (size_t)p.batch * shape.chunks * 2 * p.channels;
    g.means = g.sums + (size_t)p.batch * 2 * p.channels;
    g.floats = g.means + (size_t)p.batch * p.groups * 2;
    return g;
}

template <typename T, int V>
__global__ __launch_bounds__(kThreads) void norm_grad_sums_kernel(sys_group_norm_t p, NormArgs a, NormShape shape)
{
    const int b = blockIdx.x / shape.chunks, chunk = blockIdx.x - b * shape.chunks;
    const Lanes at(shape.columns);
    const long long begin = chunk * shape.chunk_rows, end = begin + shape.chunk_rows < p.rows ? begin + shape.chunk_rows : p.rows;
    const T* x = (const T*)a.x + b * p.x_batch;
    const T* dy = (const T*)a.dy + b * p.y_batch;
    float* to = a.workspace + ((size_t)b * shape.chunks + chunk) * 2 * p.channels;
    __shared__ float shared[V][kThreads];
    for (int c0 = 0; c0 < shape.columns; c0 += at.wide) {
        const int column = c0 + at.column;
        const bool there = at.there && column < shape.columns;
        float f_sum[V], hat_sum[V];
#pragma unroll
        for (int i = 0; i < V; ++i) f_sum[i] = hat_sum[i] = 0.0f;
        if (there) {
            const int group = column / shape.columns_a_group;
            const float mean = a.mean_in[(size_t)b * p.groups + group], rstd = a.rstd_in[(size_t)b * p.groups + group];
            float w[V], shift[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                w[i] = a.w ? load_param(a.w, (size_t)column * V + i, p.param_dtype) : 1.0f;
                shift[i] = a.b ? load_param(a.b, (size_t)column * V + i, p.param_dtype) : 0.0f;
            }
            for (long long r = begin + at.row; r < end; r += at.tall) {
                float v[V], f[V];
                Channels<T, V>::load(x + r * p.x_row + (long long)column * V, v);
                Channels<T, V>::load(dy + r * p.y_row + (long long)column * V, f);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float hat = (v[i] - mean) * rstd;
                    f[i] *= activated_grad(__builtin_fmaf(hat, w[i], shift[i]), p.activation);
                    f_sum[i] += f[i];
                    hat_sum[i] = __builtin_fmaf(f[i], hat, hat_sum[i]);
                }
            }
        }
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < V; ++i) shared[i][threadIdx.x] = which ? hat_sum[i] : f_sum[i];
            __syncthreads();
            if (at.row == 0 && there) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float s = shared[i][at.column];
                    for (int k = 1; k < at.tall; ++k) s += shared[i][k * at.wide + at.column];
                    to[(size_t)which * p.channels + (size_t)column * V + i] = s;
                }
            }
        }
    }
}

// Sums over the chunks: a lane an element of [batch][f | f hat][channel].
__global__ __launch_bounds__(kThreads) void norm_grad_chunks_kernel(sys_group_norm_t p, NormArgs a, NormShape shape)
{
    const long long at = (long long)blockIdx.x * kThreads + threadIdx.x, row = 2LL * p.channels;
    if (at >= p.batch * row) return;
    const long long b = at / row;
    const float* from = a.workspace + b * shape.chunks * row + (at - b * row);
    float s = 0.0f;
    for (int k = 0; k < shape.chunks; ++k) s += from[k * row];
    a.workspace[grad_space(p, shape).sums + at] = s;
}

// The first group_blocks workgroups: m1 and m2, a wavefront a group.  The others: dw and db, a lane a channel.
__global__ __launch_bounds__(kThreads) void norm_grad_means_kernel(sys_group_norm_t p, NormArgs a, NormShape shape, unsigned group_blocks)
{
    const GradSpace g = grad_space(p, shape);
    const float* sums = a.workspace + g.sums;
    if (blockIdx.x < group_blocks) {
        const long long at = ((long long)blockIdx.x * kThreads + threadIdx.x) >> 6;
        if (at >= (long long)p.batch * p.groups) return;
        const long long b = at / p.groups;
        const int channels = p.channels / p.groups, first = (int)(at - b * p.groups) * channels, lane = threadIdx.x & 63;
        const float* from = sums + b * 2 * p.channels;
        float m1 = 0.0f, m2 = 0.0f;
        for (int k = lane; k < channels; k += 64) {
            const float w = a.w ? load_param(a.w, first + k, p.param_dtype) : 1.0f;
            m1 = __builtin_fmaf(w, from[first + k], m1);
            m2 = __builtin_fmaf(w, from[p.channels + first + k], m2);
        }
        for (int k = 1; k < 64; k <<= 1) {
            m1 += __shfl_xor(m1, k);
            m2 += __shfl_xor(m2, k);
        }
        const float all = (float)((double)channels * (double)p.rows);
        if (lane == 0) {
            a.workspace[g.means + 2 * at] = m1 / all;
            a.workspace[g.means + 2 * at + 1] = m2 / all;
        }
        return;
    }
    const long long at = (long long)(blockIdx.x - group_blocks) * kThreads + threadIdx.x;
    if (at >= 2LL * p.channels) return;
    const bool is_w = at >= p.channels;
    void* to = is_w ? a.dw : a.db;
    if (!to) return;
    float s = 0.0f;
    for (int b = 0; b < p.batch; ++b) s += sums[b * 2LL * p.channels + at];
    store_param(to, at - (is_w ? p.channels : 0), p.param_dtype, s);
}

template <typename T, int V>
__global__ __launch_bounds__(kThreads) void norm_grad_apply_kernel(sys_group_norm_t p, NormArgs a, NormShape shape)
{
    const int b = blockIdx.x / shape.chunks, chunk = blockIdx.x - b * shape.chunks;
    const Lanes at(shape.columns);
    if (!at.there) return;
    const long long begin = chunk * shape.chunk_rows, end = begin + shape.chunk_rows < p.rows ? begin + shape.chunk_rows : p.rows;
    const T* x = (const T*)a.x + b * p.x_batch;
    const T* dy = (const T*)a.dy + b * p.y_batch;
    T* dx = (T*)a.dx + (size_t)b * p.rows * p.channels;
    const float* means = a.workspace + grad_space(p, shape).means + 2 * (size_t)b * p.groups;
    for (int column = at.column; column < shape.columns; column += at.wide) {
        const int group = column / shape.columns_a_group;
        const float mean = a.mean_in[(size_t)b * p.groups + group], rstd = a.rstd_in[(size_t)b * p.groups + group];
        const float m1 = means[2 * group], m2 = means[2 * group + 1];
        float w[V], shift[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            w[i] = a.w ? load_param(a.w, (size_t)column * V + i, p.param_dtype) : 1.0f;
            shift[i] = a.b ? load_param(a.b, (size_t)column * V + i, p.param_dtype) : 0.0f;
        }
        for (long long r = begin + at.row; r < end; r += at.tall) {
            float v[V], f[V];
            Channels<T, V>::load(x + r * p.x_row + (long long)column * V, v);
            Channels<T, V>::load(dy + r * p.y_row + (long long)column * V, f);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float hat = (v[i] - mean) * rstd;
                f[i] *= activated_grad(__builtin_fmaf(hat, w[i], shift[i]), p.activation);
                v[i] = rstd * (__builtin_fmaf(f[i], w[i], -m1) - hat * m2);
            }
            Channels<T, V>::store(dx + r * p.channels + (long long)column * V, v);
        }
    }
}

// ---------------------------------------------------------------- launches

int vector_of(const sys_group_norm_t& p)
{
    int v = p.dtype == SYS_F32 ? 4 : 8;
    while (p.channels / p.groups % v) v /= 2;
    return v;
}

NormShape shape_of(const sys_group_norm_t& p)
{
    NormShape s;
    const int v = vector_of(p);
    s.columns = p.channels / v;
    s.columns_a_group = s.columns / p.groups;
    // some 2048 workgroups, each of at least 16 rows a lane
    const long long tall = s.columns < kThreads ? kThreads / s.columns : 1;
    const long long most = (p.rows + 16 * tall - 1) / (16 * tall);
    long long chunks = p.batch > 0 ? (2048LL + p.batch - 1) / p.batch : 1;
    if (chunks > most) chunks = most;
    if (chunks < 1) chunks = 1;
    s.chunk_rows = (p.rows + chunks - 1) / chunks;
    s.chunks = (int)((p.rows + s.chunk_rows - 1) / s.chunk_rows);
    return s;
}

unsigned blocks_for(long long lanes) { return (unsigned)((lanes + kThreads - 1) / kThreads); }

template <typename T, int V>
hipError_t launch_forward(const sys_group_norm_t& p, const NormArgs& a, hipStream_t s)
{
    const NormShape shape = shape_of(p);
    const dim3 grid((unsigned)(shape.chunks * p.batch)), block(kThreads);
    hipLaunchKernelGGL((norm_moments_kernel<T, V>), grid, block, 0, s, p, a, shape);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((norm_statistics_kernel<T>), dim3(blocks_for(64LL * p.batch * p.groups)), block, 0, s, p, a, shape);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL((norm_apply_kernel<T, V>), grid, block, 0, s, p, a, shape);
    return hipGetLastError();
}

template <typename T, int V>
hipError_t launch_backward(const sys_group_norm_t& p, const NormArgs& a, hipStream_t s)
{
    const NormShape shape = shape_of(p);
    const dim3 grid((unsigned)(shape.chunks * p.batch)), block(kThreads);
    const unsigned group_blocks = blocks_for(64LL * p.batch * p.groups);
    hipError_t e;
    if (p.batch) {
        hipLaunchKernelGGL((norm_grad_sums_kernel<T, V>), grid, block, 0, s, p, a, shape);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        hipLaunchKernelGGL(norm_grad_chunks_kernel, dim3(blocks_for(2LL * p.batch * p.channels)), block, 0, s, p, a, shape);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    hipLaunchKernelGGL(norm_grad_means_kernel, dim3(group_blocks + blocks_for(2LL * p.channels)), block, 0, s, p, a, shape, group_blocks);
    if ((e = hipGetLastError()) != hipSuccess || !p.batch) return e;
    hipLaunchKernelGGL((norm_grad_apply_kernel<T, V>), grid, block, 0, s, p, a, shape);
    return hipGetLastError();
}

template <typename T, int V>
hipError_t launch_vector(bool grad, const sys_group_norm_t& p, const NormArgs& a, hipStream_t s)
{
    return grad ? launch_backward<T, V>(p, a, s) : launch_forward<T, V>(p, a, s);
}

template <typename T>
hipError_t launch_type(bool grad, const sys_group_norm_t& p, const NormArgs& a, hipStream_t s)
{
    switch (vector_of(p)) {
    case 1: return launch_vector<T, 1>(grad, p, a, s);
    case 2: return launch_vector<T, 2>(grad, p, a, s);
    case 4: return launch_vector<T, 4>(grad, p, a, s);
    default:
        if constexpr (sizeof(T) == 2) return launch_vector<T, 8>(grad, p, a, s);
        return hipErrorInvalidValue;
    }
}

hipError_t launch(bool grad, const sys_group_norm_t& p, const NormArgs& a, hipStream_t s)
{
    // (blocks of the small kernels: a wavefront a group, a lane a channel of a batch entry)
    if (64LL * p.batch * p.groups > 0x7fffffffLL * kThreads || (long long)shape_of(p).chunks * p.batch > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    switch (p.dtype) {
    case SYS_F32: return launch_type<float>(grad, p, a, s);
    case SYS_F16: return launch_type<f16_t>(grad, p, a, s);
    default: return launch_type<bf16_t>(grad, p, a, s);
    }
}

}  // namespace

hipError_t launch_group_norm(const sys_group_norm_t& p, const NormArgs& a, hipStream_t s) { return launch(false, p, a, s); }
hipError_t launch_group_norm_grad(const sys_group_norm_t& p, const NormArgs& a, hipStream_t s) { return launch(true, p, a, s); }

size_t group_norm_workspace(const sys_group_norm_t& p)
{
    const NormShape s = shape_of(p);
    return (size_t)p.batch * s.chunks * s.columns * sizeof(Moments) + (size_t)p.batch * p.groups * 2 * sizeof(float);
}

size_t group_norm_grad_workspace(const sys_group_norm_t& p) { return grad_space(p, shape_of(p)).floats * sizeof(float); }

}  // namespace sysconv
