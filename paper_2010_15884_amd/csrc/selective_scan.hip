// Selective scan: h_t[n] = e^(s_t A[n]) h_{t-1}[n] + s_t u_t B_t[n],  y_t = (sum_n C_t[n] h_t[n] + D u_t) silu(z_t),
// s_t = softplus(delta_t + bias).  Prompts here, and single tokens; the gradients are in selective_scan_grad.hip.
//
// An element (position, channel, state) costs one exponential and four multiplies or multiply-adds, 25 clocks of a SIMD for 64
// elements (exp2 8.3, the others 4.2), against 8 bytes a (position, channel) in bf16: from about eight states on the vector ALUs
// are the bound.  The recurrence runs down the positions, so what can run side by side is batch x channels x states; where that
// leaves SIMDs idle the positions are cut into chunks: one launch finds each chunk's end state from a zero start, the next one starts
// every chunk from the states of those before it, combined in its prologue with e^(A sum s), and computes the outputs.
//
// Measured, bf16, 16 states, gated: one sequence of 4096 positions and channels (2^28 elements) 130 us; by the profiler 58 for the end states and 86 for
// the outputs, 5.2 and 7.9 vector instructions an element, VALUs 85 % busy, LDS 14 and 19; one sweep alone could take no less than 47.
// (The end state of the last chunk is worked out too, and not used.)
// Not faster, when it took 145: 8 or 32 positions a tile (151, 151), sixteen lanes a channel in one sweep without chunks (240 to 258: one wavefront a
// SIMD waits for every step), the scheduler set on instruction-level parallelism.
#include "launch.h"
#include "sequence.h"
#include "scan_tile.h"

namespace sysconv {
namespace {

// OUTPUTS false: the chunk's end state from zero and its sum of step sizes, into the workspace
// ([batch][chunk][channel][4 NS] and, behind those, [batch][chunk][channel]).
template <typename T, int NS, bool OUTPUTS>
__global__ __launch_bounds__(kScanThreads) void scan_kernel(sys_selective_scan_t p, ScanArgs a, ScanShape shape)
{
    constexpr int kOwn = kScanTile / 4;            // positions of a tile that a lane owns
    const ScanPlace at = scan_place(p, shape, a.lengths, blockIdx.x);
    const int part = threadIdx.x & 3, n0 = part * NS;
    const size_t all_chunks = (size_t)p.batch * shape.chunks;
    float* ends = a.workspace;
    float* sums = a.workspace + all_chunks * p.channels * (4 * NS);

    float decay[NS], h[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        const bool is = n0 + i < p.states;
        decay[i] = is ? a.a[(size_t)at.channel * p.states + n0 + i] * kLog2e : 0.0f;
        h[i] = is && OUTPUTS && a.state ? a.state[((size_t)at.batch * p.channels + at.channel) * p.states + n0 + i] : 0.0f;
    }
    if (OUTPUTS) {
        // the states behind the chunks before this one
        for (int k = 0; k < at.chunk; ++k) {
            const size_t row = ((size_t)at.batch * shape.chunks + k) * p.channels + at.channel;
            const float s = sums[row];
            float end[NS];
#pragma unroll
            for (int i = 0; i < NS; ++i) end[i] = ends[row * (4 * NS) + n0 + i];
#pragma unroll
            for (int i = 0; i < NS; ++i) h[i] = __builtin_fmaf(fast_exp2(s * decay[i]), h[i], end[i]);
        }
    }
    const float bias = a.delta_bias ? a.delta_bias[at.channel] : 0.0f;
    const float skip = OUTPUTS && a.d ? a.d[at.channel] : 0.0f;
    const int last = at.length < at.end ? at.length : at.end;      // positions that exist in this chunk end here
    const bool gated = OUTPUTS && a.z;
    RowBuffer<T> u((const T*)a.u + at.batch * p.u_batch, p.u_row, p.channels, at.begin, last);
    RowBuffer<T> delta((const T*)a.delta + at.batch * p.delta_batch, p.delta_row, p.channels, at.begin, last);
    RowBuffer<T> z(gated ? (const T*)a.z + at.batch * p.z_batch : nullptr, p.z_row, p.channels, at.begin, last);
    if (!gated) z.left = -1;
    RowBuffer<T> y(OUTPUTS ? (const T*)a.y + at.batch * p.y_batch : nullptr, p.y_row, p.channels, at.begin, last);
    unsigned u_at[kOwn], delta_at[kOwn], z_at[kOwn], y_at[kOwn];
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
        u_at[k] = u.offset(4 * k + part, at.channel);
        delta_at[k] = delta.offset(4 * k + part, at.channel);
        z_at[k] = z.offset(4 * k + part, at.channel);
        y_at[k] = at.there ? y.offset(4 * k + part, at.channel) : kNowhere;
    }
    __shared__ __attribute__((aligned(16))) float tile_b[2][kScanTile * 4 * NS], tile_c[OUTPUTS ? 2 : 1][kScanTile * 4 * NS];
    StateTile<T, NS> next_b((const T*)a.b + at.batch * p.b_batch + (size_t)at.group * p.states, p.b_row, p.states, at.begin, last);
    StateTile<T, NS> next_c((const T*)a.c + at.batch * p.c_batch + (size_t)at.group * p.states, p.c_row, p.states, at.begin, last);
    unsigned next_u[kOwn], next_delta[kOwn], next_z[kOwn];
    auto fetch = [&] {
        next_b.load();
        if (OUTPUTS) next_c.load();
        const __amdgpu_buffer_rsrc_t u_tile = u.tile(), delta_tile = delta.tile();
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            next_u[k] = buffer_load<T>(u_tile, u_at[k]);
            next_delta[k] = buffer_load<T>(delta_tile, delta_at[k]);
        }
        if (OUTPUTS) {
            const __amdgpu_buffer_rsrc_t z_tile = z.tile();
#pragma unroll
            for (int k = 0; k < kOwn; ++k) next_z[k] = buffer_load<T>(z_tile, z_at[k]);
        }
        u.next(), delta.next(), z.next();
    };
    float s_sum = 0.0f;
    fetch();
    for (int t0 = at.begin, turn = 0; t0 < last; t0 += kScanTile, turn ^= 1) {
        float own_u[kOwn], own_s[kOwn], own_z[kOwn], own_y[kOwn];
        next_b.store(tile_b[turn], t0);
        if (OUTPUTS) next_c.store(tile_c[turn], t0);
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            own_u[k] = loaded<T>(next_u[k]);
            own_z[k] = loaded<T>(next_z[k]);
            own_s[k] = loaded<T>(next_delta[k]) + bias;
        }
        if (p.softplus) {
#pragma unroll
            for (int k = 0; k < kOwn; ++k) own_s[k] = softplus(own_s[k]);
        }
        if (t0 + kScanTile > last) {
#pragma unroll
            for (int k = 0; k < kOwn; ++k) {
                const bool on = t0 + 4 * k + part < last;             // a position that is not there leaves the state as it is
                own_s[k] = on ? own_s[k] : 0.0f;
                own_u[k] = on ? own_u[k] : 0.0f;
            }
        }
        if (!OUTPUTS) {
#pragma unroll
            for (int k = 0; k < kOwn; ++k) s_sum += own_s[k];
        }
        __syncthreads();
        fetch();                                                       // (past the end: zeros)
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            const float s_own = own_s[k], x_own = own_s[k] * own_u[k];
            float sums_of[4];
            auto step = [&](auto lane) {
                constexpr int j = decltype(lane)::value;
                const float s = quad_take<j>(s_own), x = quad_take<j>(x_own);
                float bt[NS], ct[NS], sum = 0.0f;
                take<NS>(tile_b[turn] + (4 * k + j) * 4 * NS + n0, bt);
                if (OUTPUTS) take<NS>(tile_c[turn] + (4 * k + j) * 4 * NS + n0, ct);
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    h[i] = __builtin_fmaf(fast_exp2(s * decay[i]), h[i], x * bt[i]);
                    if (OUTPUTS) sum = __builtin_fmaf(ct[i], h[i], sum);
                }
                sums_of[j] = sum;
            };
            step(std::integral_constant<int, 0>());
            step(std::integral_constant<int, 1>());
            step(std::integral_constant<int, 2>());
            step(std::integral_constant<int, 3>());
            if (OUTPUTS) own_y[k] = quad_sums(sums_of);
        }
        if (OUTPUTS) {
            const __amdgpu_buffer_rsrc_t y_tile = y.tile();
#pragma unroll
            for (int k = 0; k < kOwn; ++k) {
                float out = __builtin_fmaf(skip, own_u[k], own_y[k]);
                if (gated) out *= silu(own_z[k]);
                buffer_store<T>(y_tile, y_at[k], (T)out);
            }
            y.next();
        }
        // the other buffer is written next; every wavefront has passed the barrier of this tile when it has read the one before
    }
    if (OUTPUTS) {
        T* rest = (T*)a.y + at.batch * p.y_batch + at.channel;
        for (int t = (at.begin > last ? at.begin : last) + part; t < at.end; t += 4)
            if (at.there) rest[t * p.y_row] = (T)0.0f;
        if (a.state_out && at.there && at.chunk == shape.chunks - 1) {
#pragma unroll
            for (int i = 0; i < NS; ++i)
                if (n0 + i < p.states) a.state_out[((size_t)at.batch * p.channels + at.channel) * p.states + n0 + i] = h[i];
        }
    } else if (at.there) {
        const size_t row = ((size_t)at.batch * shape.chunks + at.chunk) * p.channels + at.channel;
#pragma unroll
        for (int i = 0; i < NS; ++i) ends[row * (4 * NS) + n0 + i] = h[i];
        s_sum = quad_sum(s_sum);
        if (part == 0) sums[row] = s_sum;
    }
}

// ---------------------------------------------------------------- single tokens

// V neighbouring states a lane, `lanes` lanes (a power of two) a channel; the states are read and written once.  64 tokens of 4096 channels with 16
// states, 34 MB of states and 1 MB else: 11 us, 3.2 TB/s, with the VALUs three quarters busy, most of that with the indices' divisions; a call from the host 11.4.
template <typename T, int V>
__global__ __launch_bounds__(kScanThreads) void scan_step_kernel(sys_selective_scan_t p, ScanArgs a, int log_lanes)
{
    const long long at = ((long long)blockIdx.x * kScanThreads + threadIdx.x) >> log_lanes;
    const int lanes = 1 << log_lanes, part = threadIdx.x & (lanes - 1);
    const int r = (int)(at / p.channels);
    if (r >= p.batch) return;                      // (whole groups of lanes leave together)
    const int d = (int)(at - (long long)r * p.channels);
    const int slot = a.slots ? a.slots[r] : r;
    T* y = (T*)a.y + r * p.y_batch + d;
    if (slot < 0 || slot >= p.slots) {
        if (part == 0) *y = (T)0.0f;
        return;
    }
    const float u = (float)((const T*)a.u)[r * p.u_batch + d];
    float s = (float)((const T*)a.delta)[r * p.delta_batch + d] + (a.delta_bias ? a.delta_bias[d] : 0.0f);
    if (p.softplus) s = softplus(s);
    const int group = d / (p.channels / p.groups);
    const T* b = (const T*)a.b + r * p.b_batch + (size_t)group * p.states;
    const T* c = (const T*)a.c + r * p.c_batch + (size_t)group * p.states;
    const size_t base = ((size_t)slot * p.channels + d) * p.states;
    const float x = s * u;
    float sum = 0.0f;
    const int n = part * V;
    if (n < p.states) {
        float h[V], decay[V], bt[V], ct[V];
        Channels<float, V>::load(a.state + base + n, h);
        Channels<float, V>::load(a.a + (size_t)d * p.states + n, decay);
        Channels<T, V>::load(b + n, bt);
        Channels<T, V>::load(c + n, ct);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            h[i] = __builtin_fmaf(fast_exp2(s * (decay[i] * kLog2e)), h[i], x * bt[i]);
            sum = __builtin_fmaf(ct[i], h[i], sum);
        }
        Channels<float, V>::store(a.state_out + base + n, h);
    }
    for (int k = lanes >> 1; k; k >>= 1) sum += __shfl_xor(sum, k);
    if (part == 0) {
        float out = a.d ? __builtin_fmaf(a.d[d], u, sum) : sum;
        if (a.z) out *= silu((float)((const T*)a.z)[r * p.z_batch + d]);
        *y = (T)out;
    }
}

// ---------------------------------------------------------------- launches

ScanShape forward_shape(const sys_selective_scan_t& p, bool ragged)
{
    ScanShape s;
    s.channels_a_group = p.channels / p.groups;
    s.blocks_a_group = (s.channels_a_group + kScanChannels - 1) / kScanChannels;
    s.channel_blocks = s.blocks_a_group * p.groups;
    const long long workgroups = (long long)s.channel_blocks * p.batch;
    const int tiles = (p.length + kScanTile - 1) / kScanTile;
    // Chunks cost 1.65 times the work, so they begin where a wavefront a SIMD is not there; then sixteen wavefronts a CU, in chunks of at
    // least two tiles (one sequence of 4096 positions and channels, eight / sixteen / thirty-two a CU: 148 / 131 / 131 us; with / without chunks
    // 2 x 2048 x 4096 130 / 247, 4 x 2048 x 4096 246 / 248, 4 x 1024 x 4096 129 / 127, 6 x 1024 x 4096 197 / 171).  With lengths some chunks will be
    // empty (seven sequences of 0 .. 517 positions, eight / sixteen / thirty-two a CU: 48 / 36 / 30).
    long long chunks = workgroups >= 256 ? 1 : (ragged ? 2048 : 1024) / (workgroups ? workgroups : 1);
    if (chunks > tiles / 2) chunks = tiles / 2;
    if (chunks > 64) chunks = 64;
    if (chunks < 1) chunks = 1;
    const int tiles_a_chunk = tiles ? (int)((tiles + chunks - 1) / chunks) : 1;
    s.chunk_rows = tiles_a_chunk * kScanTile;
    s.chunks = tiles ? (tiles + tiles_a_chunk - 1) / tiles_a_chunk : 1;
    return s;
}

template <typename T, int NS>
hipError_t launch_forward(const sys_selective_scan_t& p, const ScanArgs& a, hipStream_t s)
{
    const ScanShape shape = forward_shape(p, a.lengths != nullptr);
    const long long blocks = (long long)shape.channel_blocks * shape.chunks * p.batch;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    if (shape.chunks > 1) {
        hipLaunchKernelGGL((scan_kernel<T, NS, false>), dim3((unsigned)blocks), dim3(kScanThreads), 0, s, p, a, shape);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((scan_kernel<T, NS, true>), dim3((unsigned)blocks), dim3(kScanThreads), 0, s, p, a, shape);
    return hipGetLastError();
}

template <typename T, int V>
hipError_t launch_token(const sys_selective_scan_t& p, const ScanArgs& a, hipStream_t s)
{
    int log_lanes = 0;
    while ((V << log_lanes) < p.states) ++log_lanes;
    const long long threads = ((long long)p.batch * p.channels) << log_lanes;
    const long long blocks = (threads + kScanThreads - 1) / kScanThreads;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((scan_step_kernel<T, V>), dim3((unsigned)blocks), dim3(kScanThreads), 0, s, p, a, log_lanes);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_type(bool step, const sys_selective_scan_t& p, const ScanArgs& a, hipStream_t s)
{
    if (step) return p.states % 4 == 0 ? launch_token<T, 4>(p, a, s) : launch_token<T, 1>(p, a, s);
    switch (scan_states_a_lane(p.states)) {
    case 1: return launch_forward<T, 1>(p, a, s);
    case 2: return launch_forward<T, 2>(p, a, s);
    case 4: return launch_forward<T, 4>(p, a, s);
    case 8: return launch_forward<T, 8>(p, a, s);
    default: return launch_forward<T, 16>(p, a, s);
    }
}

hipError_t launch(bool step, const sys_selective_scan_t& p, const ScanArgs& a, hipStream_t s)
{
    switch (p.dtype) {
    case SYS_F32: return launch_type<float>(step, p, a, s);
    case SYS_F16: return launch_type<f16_t>(step, p, a, s);
    default: return launch_type<bf16_t>(step, p, a, s);
    }
}

}  // namespace

hipError_t launch_scan(const sys_selective_scan_t& p, const ScanArgs& a, hipStream_t s)
{
    sys_selective_scan_t q = p;
    if (q.length == 1) q.y_row = q.channels;           // (a stride of no meaning; rows that are not there must lie behind this one)
    return launch(false, q, a, s);
}
hipError_t launch_scan_step(const sys_selective_scan_t& p, const ScanArgs& a, hipStream_t s) { return launch(true, p, a, s); }

size_t scan_workspace(const sys_selective_scan_t& p)
{
    const ScanShape s = forward_shape(p, true);         // (more chunks than without lengths)
    if (s.chunks == 1) return 0;
    return (size_t)p.batch * s.chunks * p.channels * (4 * scan_states_a_lane(p.states) + 1) * sizeof(float);
}

}  // namespace sysconv
