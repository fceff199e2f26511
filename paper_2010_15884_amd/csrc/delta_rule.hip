// Gated delta rule, a position at a time: S_t = a_t S_{t-1} + k_t u_t^T, u_t = b_t (v_t - a_t S_{t-1}^T k_t), y_t = scale S_t^T q_t.
// Single tokens and short sequences; longer ones go through delta_chunk.hip.
//
// A workgroup holds the state of one head and 64 of its value columns in registers: V neighbouring columns a lane, 64 / V lanes a row, and the rows
// dealt to the groups of lanes in turn.  Both products with the state are taken of S_{t-1} in one sweep, S_t^T q = a S_{t-1}^T q + (k . q) u, so a
// position costs one sum over the rows (in the lane, over the wavefront's groups, over the wavefronts through LDS: one barrier).
// A position is four multiply-adds an element of the state against, for single tokens, 8 bytes of it: those are bound by memory.  64 tokens of 32 heads of 128 x 128
// take 55 us for 270 MB, 4.9 TB/s, a copy's rate.
#include "delta_tile.h"
#include "launch.h"

namespace sysconv {
namespace {

constexpr int kThreads = 256;
constexpr int kWavesOf = kThreads / 64;
constexpr int kColumns = 64;                       // of the values, a workgroup

template <typename T, int V, int KD>
__global__ __launch_bounds__(kThreads) void delta_step_kernel(sys_gated_delta_t p, DeltaArgs a, int blocks, int length, bool slotted)
{
    constexpr int kLanes = kColumns / V, kGroups = kThreads / kLanes, kRows = (KD + kGroups - 1) / kGroups;
    const int block = blockIdx.x % blocks, head = blockIdx.x / blocks % p.value_heads, b = blockIdx.x / blocks / p.value_heads;
    const int column = block * kColumns + (threadIdx.x % kLanes) * V, group = threadIdx.x / kLanes, wave = threadIdx.x >> 6;
    const bool there = column < p.value_dim;                           // (V divides it)
    const int key_head = head / (p.value_heads / p.key_heads);
    long long place = b;
    if (slotted && a.slots) place = a.slots[b];
    T* y = (T*)a.y + b * p.y_batch + head * p.value_dim + column;
    if (slotted && (place < 0 || place >= p.slots)) {
        const float zero[V] = {};
        if (group == 0 && there) Channels<T, V>::store(y, zero);
        return;
    }
    // a head's state as a buffer: rows and columns that are not there lie past its end, are zeros and not written
    const size_t base = ((size_t)place * p.value_heads + head) * p.key_dim * p.value_dim;
    const unsigned bytes = (unsigned)(p.key_dim * p.value_dim) * 4u;
    const unsigned offset = there ? (unsigned)(group * p.value_dim + column) * 4u : kNowhere, row_bytes = (unsigned)(kGroups * p.value_dim) * 4u;
    float s[kRows][V];
    {
        const __amdgpu_buffer_rsrc_t state = __builtin_amdgcn_make_buffer_rsrc((void*)(a.state + base), 0, a.state ? bytes : 0u, 0x00027000);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const unsigned at = there ? offset + i * row_bytes : kNowhere;
            if constexpr (V == 4) {
                const f4 v = __builtin_bit_cast(f4, __builtin_amdgcn_raw_buffer_load_b128(state, at, 0, 0));
#pragma unroll
                for (int j = 0; j < V; ++j) s[i][j] = v[j];
            } else {
                s[i][0] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(state, at, 0, 0));
            }
        }
    }
    const T* q = (const T*)a.q + b * p.q_batch + key_head * p.key_dim;
    const T* k = (const T*)a.k + b * p.k_batch + key_head * p.key_dim;
    const T* v = (const T*)a.v + b * p.v_batch + head * p.value_dim + (there ? column : 0);
    const T* delta = (const T*)a.delta + b * p.delta_batch + head;
    const T* beta = (const T*)a.beta + b * p.beta_batch + head;
    const float rate = a.a[head], bias = a.delta_bias ? a.delta_bias[head] : 0.0f;
    const int last = slotted ? 1 : sequence_length(a.lengths, b, length);

    // q and k of a position, three positions deep: the next one's are written while slower wavefronts still read the one before
    __shared__ float keys[3][KD], queries[3][KD];
    __shared__ float parts[2][kWavesOf][2 * kColumns + 1];
    const int mine = threadIdx.x % KD;
    const bool mine_is_q = threadIdx.x / KD == 1, mine_there = threadIdx.x < 2 * KD;
    auto fetch = [&](int t) -> float {
        return mine_there && mine < p.key_dim && t < last ? (float)(mine_is_q ? q[t * p.q_row + mine] : k[t * p.k_row + mine]) : 0.0f;
    };
    auto put = [&](int t, float value) {
        if (mine_there) (mine_is_q ? queries : keys)[t % 3][mine] = value;
    };
    if (last > 0) put(0, fetch(0));
    __syncthreads();
    for (int t = 0; t < last; ++t) {
        const float ahead = fetch(t + 1);
        float vt[V], step = (float)delta[t * p.delta_row] + bias, strength = (float)beta[t * p.beta_row];
        Channels<T, V>::load(v + t * p.v_row, vt);
        if (p.softplus) step = softplus(step);
        if (p.sigmoid) strength = sigmoid(strength);
        const float decay = fast_exp2(step * rate * kLog2e);
        float kt[kRows], sk[V] = {}, sq[V] = {}, kq = 0.0f;
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int row = group + i * kGroups;
            kt[i] = KD % kGroups == 0 || row < KD ? keys[t % 3][row] : 0.0f;
            const float qt = KD % kGroups == 0 || row < KD ? queries[t % 3][row] : 0.0f;
            kq = __builtin_fmaf(kt[i], qt, kq);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                sk[j] = __builtin_fmaf(s[i][j], kt[i], sk[j]);
                sq[j] = __builtin_fmaf(s[i][j], qt, sq[j]);
            }
        }
#pragma unroll
        for (int m = kLanes; m < 64; m <<= 1) {
            kq += __shfl_xor(kq, m);
#pragma unroll
            for (int j = 0; j < V; ++j) sk[j] += __shfl_xor(sk[j], m), sq[j] += __shfl_xor(sq[j], m);
        }
        if ((threadIdx.x & 63) < kLanes) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                parts[t & 1][wave][(threadIdx.x % kLanes) * V + j] = sk[j];
                parts[t & 1][wave][kColumns + (threadIdx.x % kLanes) * V + j] = sq[j];
            }
            if ((threadIdx.x & 63) == 0) parts[t & 1][wave][2 * kColumns] = kq;
        }
        put(t + 1, ahead);
        __syncthreads();
        kq = 0.0f;
#pragma unroll
        for (int j = 0; j < V; ++j) sk[j] = sq[j] = 0.0f;
#pragma unroll
        for (int w = 0; w < kWavesOf; ++w) {
            kq += parts[t & 1][w][2 * kColumns];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                sk[j] += parts[t & 1][w][(threadIdx.x % kLanes) * V + j];
                sq[j] += parts[t & 1][w][kColumns + (threadIdx.x % kLanes) * V + j];
            }
        }
        float u[V], out[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            u[j] = strength * __builtin_fmaf(-decay, sk[j], vt[j]);
            out[j] = p.scale * __builtin_fmaf(decay, sq[j], kq * u[j]);
        }
        if (group == 0 && there) Channels<T, V>::store(y + t * p.y_row, out);
#pragma unroll
        for (int i = 0; i < kRows; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) s[i][j] = __builtin_fmaf(decay, s[i][j], kt[i] * u[j]);
    }
    if (!slotted) {
        const float zero[V] = {};
        for (int t = last + group; t < length; t += kGroups)
            if (there) Channels<T, V>::store(y + t * p.y_row, zero);
    }
    if (a.state_out) {
        const __amdgpu_buffer_rsrc_t state = __builtin_amdgcn_make_buffer_rsrc((void*)(a.state_out + base), 0, bytes, 0x00027000);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const unsigned at = there ? offset + i * row_bytes : kNowhere;
            if constexpr (V == 4) {
                const f4 v = {s[i][0], s[i][1], s[i][2], s[i][3]};
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, v), state, at, 0, 0);
            } else {
                __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, s[i][0]), state, at, 0, 0);
            }
        }
    }
}

template <typename T, int V, int KD>
hipError_t launch_shape(bool step, const sys_gated_delta_t& p, const DeltaArgs& a, hipStream_t s)
{
    const int blocks = (p.value_dim + kColumns - 1) / kColumns;
    const long long all = (long long)blocks * p.value_heads * p.batch;
    if (all > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((delta_step_kernel<T, V, KD>), dim3((unsigned)all), dim3(kThreads), 0, s, p, a, blocks, step ? 1 : p.length, step);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_type(bool step, const sys_gated_delta_t& p, const DeltaArgs& a, hipStream_t s)
{
    if (p.value_dim % 4 == 0) return p.key_dim <= 64 ? launch_shape<T, 4, 64>(step, p, a, s) : launch_shape<T, 4, 128>(step, p, a, s);
    return p.key_dim <= 64 ? launch_shape<T, 1, 64>(step, p, a, s) : launch_shape<T, 1, 128>(step, p, a, s);
}

hipError_t launch(bool step, const sys_gated_delta_t& p, const DeltaArgs& a, hipStream_t s)
{
    switch (p.dtype) {
    case SYS_F32: return launch_type<float>(step, p, a, s);
    case SYS_F16: return launch_type<f16_t>(step, p, a, s);
    default: return launch_type<bf16_t>(step, p, a, s);
    }
}

}  // namespace

hipError_t launch_delta_step(const sys_gated_delta_t& p, const DeltaArgs& a, hipStream_t s) { return launch(true, p, a, s); }
hipError_t launch_delta_positions(const sys_gated_delta_t& p, const DeltaArgs& a, hipStream_t s) { return launch(false, p, a, s); }

}  // namespace sysconv
