// What the operators on channels-last sequences share (causal_conv.hip, selective_scan.hip, selective_scan_grad.hip, group_norm.hip):
// element types, loads and stores of several channels a lane, the activations, and sums over neighbouring lanes.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "sysconv.h"

namespace sysconv {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// V neighbouring channels of a row.  Rows may begin at any element, so the type asks for the alignment of one element only: the
// global loads and stores of this part take any byte address.
template <typename T, int V>
struct Channels {
    typedef T Vec __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    typedef float F __attribute__((ext_vector_type(V)));
    // as they lie in memory: half the registers of their values, for loads that are far ahead of their use
    typedef T Raw __attribute__((ext_vector_type(V)));
    static __device__ __forceinline__ Raw raw(const T* p) { return *(const Vec*)p; }
    static __device__ __forceinline__ void values(Raw v, float (&out)[V])
    {
        const F f = __builtin_convertvector(v, F);
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = f[i];
    }
    static __device__ __forceinline__ void load(const T* p, float (&out)[V]) { values(raw(p), out); }
    static __device__ __forceinline__ void store(T* p, const float (&in)[V])
    {
        F f;
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = in[i];
        *(Vec*)p = __builtin_convertvector(f, Vec);
    }
    static __device__ __forceinline__ void store_nt(T* p, const float (&in)[V])
    {
        F f;
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = in[i];
        __builtin_nontemporal_store(__builtin_convertvector(f, Vec), (Vec*)p);
    }
};

template <typename T>
struct Channels<T, 1> {
    typedef T Raw;
    static __device__ __forceinline__ Raw raw(const T* p) { return *p; }
    static __device__ __forceinline__ void values(Raw v, float (&out)[1]) { out[0] = (float)v; }
    static __device__ __forceinline__ void load(const T* p, float (&out)[1]) { out[0] = (float)*p; }
    static __device__ __forceinline__ void store(T* p, const float (&in)[1]) { *p = (T)in[0]; }
    static __device__ __forceinline__ void store_nt(T* p, const float (&in)[1]) { *p = (T)in[0]; }
};

// Channels of 16 bytes: what a lane loads at once.
template <typename T> constexpr int kLaneChannels = 16 / (int)sizeof(T);

// A parameter of one of the three types.
__device__ __forceinline__ float load_param(const void* p, size_t i, int dtype)
{
    if (dtype == SYS_F32) return ((const float*)p)[i];
    if (dtype == SYS_F16) return (float)((const f16_t*)p)[i];
    return (float)((const bf16_t*)p)[i];
}

// N neighbouring parameters from the i-th on, of T or fp32: one branch for all of them, loads of up to 16 bytes.
template <typename T, int N>
__device__ __forceinline__ void load_params(const void* p, size_t i, int dtype, float (&out)[N])
{
    constexpr int kMost = kLaneChannels<T>;
    if (sizeof(T) == 4 || dtype == SYS_F32) {
#pragma unroll
        for (int k = 0; k + 4 <= N; k += 4) Channels<float, 4>::load((const float*)p + i + k, *(float(*)[4])(out + k));
#pragma unroll
        for (int k = N / 4 * 4; k < N; ++k) out[k] = ((const float*)p)[i + k];
    } else {
#pragma unroll
        for (int k = 0; k + kMost <= N; k += kMost) Channels<T, kMost>::load((const T*)p + i + k, *(float(*)[kMost])(out + k));
#pragma unroll
        for (int k = N / kMost * kMost; k < N; ++k) out[k] = (float)((const T*)p)[i + k];
    }
}

__device__ __forceinline__ void store_param(void* p, size_t i, int dtype, float v)
{
    if (dtype == SYS_F32) ((float*)p)[i] = v;
    else if (dtype == SYS_F16) ((f16_t*)p)[i] = (f16_t)v;
    else ((bf16_t*)p)[i] = (bf16_t)v;
}

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float fast_rcp(float x) { return __builtin_amdgcn_rcpf(x); }

// 1 / (1 + e^-x): e^-x overflows to infinity where the result is below 2^-126, and its reciprocal is then 0.
__device__ __forceinline__ float sigmoid(float x) { return fast_rcp(1.0f + fast_exp2(-kLog2e * x)); }
__device__ __forceinline__ float silu(float x) { return x * sigmoid(x); }
__device__ __forceinline__ float silu_grad(float x)
{
    const float s = sigmoid(x);
    return s * __builtin_fmaf(x, 1.0f - s, 1.0f);
}

// log(1 + e^x) = max(x, 0) + log(1 + e), e = e^-|x| <= 1.  The logarithm of the rounded sum w = 1 + e misses what the sum
// lost, (1 + e) - w, which is added back (its factor 1/w differs from 1 only where that loss is below the result's own
// rounding); so the result keeps its relative accuracy down to e^x of the smallest normal number, where w = 1 and the loss is e.
__device__ __forceinline__ float softplus(float x)
{
    const float e = fast_exp2(-kLog2e * __builtin_fabsf(x));
    const float w = 1.0f + e;
    // (fmaxf drops a NaN, which comes back with e)
    return __builtin_fmaxf(x, 0.0f) + __builtin_fmaf(__builtin_amdgcn_logf(w), kLn2, e - (w - 1.0f));
}

// Sum of v over the 4 lanes of a quad (every lane gets it).
__device__ __forceinline__ float quad_sum(float v)
{
    v += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0xB1, 0xF, 0xF, true));   // lanes 1 0 3 2
    v += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x4E, 0xF, 0xF, true));   // lanes 2 3 0 1
    return v;
}

template <int CONTROL>
__device__ __forceinline__ float dpp(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CONTROL, 0xF, 0xF, true));
}

// Sums over the quad of four values a lane; lane j gets that of v[j].  Each step sends half of what a lane has to its neighbour.
__device__ __forceinline__ float quad_sums(const float (&v)[4])
{
    const bool odd = threadIdx.x & 1, high = threadIdx.x & 2;
    const float a = (odd ? v[1] : v[0]) + dpp<0xB1>(odd ? v[0] : v[1]);
    const float b = (odd ? v[3] : v[2]) + dpp<0xB1>(odd ? v[2] : v[3]);
    return (high ? b : a) + dpp<0x4E>(high ? a : b);
}

// v of lane J of the quad.
template <int J>
__device__ __forceinline__ float quad_take(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), J * 0x55, 0xF, 0xF, true));
}

// Workgroups go round the eight XCDs, each with an L2 of its own: workgroup i of n works at place(i), so that an XCD gets neighbouring places.
__device__ __forceinline__ unsigned xcd_place(unsigned i, unsigned n)
{
    const unsigned each = n / 8;
    return i < each * 8 ? (i & 7) * each + (i >> 3) : i;
}

// The positions of sequence b that exist: its length, held within the rows that there are.
__device__ __forceinline__ int sequence_length(const int* lengths, int b, int rows)
{
    if (!lengths) return rows;
    const int n = lengths[b];
    return n < 0 ? 0 : n > rows ? rows : n;
}

// ---------------------------------------------------------------- launch interface (arguments already validated)

struct CausalConvArgs {
    const void *x, *w, *bias, *state, *dy, *dstate_out;
    const int *lengths, *slots;
    void *y, *state_out, *dx, *dw, *dbias, *dstate;
    float* workspace;
};

struct ScanArgs {
    const void *u, *delta, *z, *b, *c, *dy;
    const float *a, *d, *delta_bias, *state, *dstate_out;
    const int *lengths, *slots;
    void *y, *du, *ddelta, *dz, *db, *dc;
    float *state_out, *da, *dd, *ddelta_bias, *dstate;
    float* workspace;
};

struct NormArgs {
    const void *x, *w, *b, *dy;
    const float *mean_in, *rstd_in;
    void *y, *dx, *dw, *db;
    float *mean, *rstd;
    float* workspace;
};

// The kernels that a call takes: rows a lane of the causal convolution, spans a chunk of the scan's gradients.
int causal_conv_rows_a_lane(const sys_causal_conv1d_t& p);
int scan_grad_spans(const sys_selective_scan_t& p);

hipError_t launch_causal_conv(const sys_causal_conv1d_t& p, const CausalConvArgs& a, hipStream_t s);
hipError_t launch_causal_conv_grad(const sys_causal_conv1d_t& p, const CausalConvArgs& a, hipStream_t s);
hipError_t launch_causal_conv_step(const sys_causal_conv1d_t& p, const CausalConvArgs& a, hipStream_t s);
size_t causal_conv_grad_workspace(const sys_causal_conv1d_t& p);

hipError_t launch_scan(const sys_selective_scan_t& p, const ScanArgs& a, hipStream_t s);
hipError_t launch_scan_grad(const sys_selective_scan_t& p, const ScanArgs& a, hipStream_t s);
hipError_t launch_scan_step(const sys_selective_scan_t& p, const ScanArgs& a, hipStream_t s);
size_t scan_workspace(const sys_selective_scan_t& p);
size_t scan_grad_workspace(const sys_selective_scan_t& p);

hipError_t launch_group_norm(const sys_group_norm_t& p, const NormArgs& a, hipStream_t s);
hipError_t launch_group_norm_grad(const sys_group_norm_t& p, const NormArgs& a, hipStream_t s);
size_t group_norm_workspace(const sys_group_norm_t& p);
size_t group_norm_grad_workspace(const sys_group_norm_t& p);

}  // namespace sysconv
