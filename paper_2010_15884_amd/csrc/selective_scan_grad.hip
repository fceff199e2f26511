// Gradients of the selective scan.  With a_t = e^(s_t A), x_t = s_t u_t and e_t = dy_t silu(z_t) (dy_t without a gate):
//
//   g_t  = C_t e_t + a_{t+1} g_{t+1}                       gradient of h_t, from the end (there: the gradient of state_out)
//   du_t = D e_t + s_t sum_n g_t B_t,   ds_t = u_t sum_n g_t B_t + sum_n A q_t,   q_t = g_t a_t h_{t-1},   ddelta_t = ds_t softplus'
//   dA   = sum_t q_t s_t,  dB_t = sum_d g_t x_t,  dC_t = sum_d h_t e_t,  dD = sum_t e_t u_t,  dz_t = dy_t (sum_n C_t h_t + D u_t) silu'(z_t)
//
// Both recurrences run along the positions, one from each end.  The positions are cut into chunks:
//   scan_ends_kernel    every chunk from a zero start: the state and sum s at its end and before each of its spans, and what its
//                       positions hand back to the chunk before it, sum_t (a_first .. a_t) C_t e_t -- with the running product, so that one sweep
//                       serves both directions;
//   scan_chain_kernel   along the chunks: the state before each, the gradient behind each;
//   scan_grad_kernel    every chunk's spans from the last to the first: the state before a span is that of the zero start plus e^(A sum s) times
//                       the chunk's; the span's states and decays go into registers, and the recurrence of the gradient runs over them;
//   scan_sums_kernel    adds up what the workgroups have summed over their channels (dB, dC) and their positions (dA, dD, ddelta_bias).
// Each sum has a fixed order.
//
// Bound by the vector ALUs.  4 x 2048 positions x 2048 channels, 16 states, gated, bf16 (2^28 elements): 337 us; by the profiler about 95 ends (10.8 vector
// instructions an element), 11 chain, 250 grad (24.6; the VALUs 88 % busy, 21 % of the LDS cycles bank conflicts that nothing here accounts for)
// and 17 sums; an exponential and fourteen multiply-adds an element are 110 us.
#include "launch.h"
#include "sequence.h"
#include "scan_tile.h"

namespace sysconv {
namespace {

// Positions of a span, whose states and decays are in registers at a time, 64 of each a lane at most; spans of a chunk at most.
template <int NS> constexpr int kSpan = NS <= 4 ? 16 : 64 / NS;
constexpr int kMostSpans = 8;
constexpr int kParts = 8;            // partial sums over channels in a workgroup: two a wavefront

struct GradShape : ScanShape {
    int spans;                       // of a chunk
};

GradShape backward_shape(const sys_selective_scan_t& p)
{
    GradShape s;
    s.channels_a_group = p.channels / p.groups;
    s.blocks_a_group = (s.channels_a_group + kScanChannels - 1) / kScanChannels;
    s.channel_blocks = s.blocks_a_group * p.groups;
    const int ns = scan_states_a_lane(p.states), span = ns <= 4 ? 16 : 64 / ns;
    // Long chunks leave the chain along them little to read and write; short ones leave work for all CUs: as long as there are two
    // workgroups a CU (16 states in bf16, eight / four / two a CU: 1 x 1024 positions x 2048 channels 81 / 69 / 64 us, 1 x 4096 x 2048 174 / 166 / 166,
    // 2 x 2048 x 4096 301 / 301 / 301).
    constexpr long long kEnough = 512LL * kMostSpans;
    const long long spans = ((long long)p.length + span - 1) / span, blocks = (long long)s.channel_blocks * p.batch;
    const long long all = (spans < kEnough ? spans : kEnough) * (blocks < kEnough ? blocks : kEnough);
    s.spans = all < 512 ? 1 : all > kEnough ? kMostSpans : (int)(all / 512);
    s.chunk_rows = s.spans * span;
    s.chunks = (int)((spans + s.spans - 1) / s.spans);
    return s;
}

// The workspace: where its parts begin, in floats.
struct Workspace {
    size_t back;                   // [batch][chunk][channel][width], behind the same for `ends` at 0
    size_t spans;                  // [batch][chunk][span 1 ..][channel][width]: the state before the span
    size_t sums;                   // [batch][chunk][span][channel]: sum s up to the span's end
    size_t params;                 // [batch][chunk][channel][width + 2]: dA, dD, ddelta_bias
    size_t states;                 // [channel block][batch][position][dB | dC][width]
    size_t floats;
};

__host__ __device__ Workspace workspace_of(const sys_selective_scan_t& p, const GradShape& shape, int width)
{
    Workspace w;
    const size_t rows = (size_t)p.batch * shape.chunks * p.channels;
    w.back = rows * width;
    w.spans = w.back + rows * width;
    w.sums = w.spans + rows * (shape.spans - 1) * width;
    w.params = w.sums + rows * shape.spans;
    w.states = w.params + rows * (width + 2);
    w.floats = w.states + (size_t)shape.channel_blocks * p.batch * p.length * 2 * width;
    return w;
}

// B or C of a chunk for LDS, [position][4 NS]: all of a lane's loads are under way before the first is used.  What is not there is read from a
// place that is, and stored as 0.
template <typename T, int NS>
struct ChunkStates {
    static constexpr int kEach = kMostSpans * kSpan<NS> * 4 * NS / kScanThreads;
    static_assert(kEach * kScanThreads == kMostSpans * kSpan<NS> * 4 * NS && kScanThreads % (4 * NS) == 0, "a lane keeps its state");
    T v[kEach];
    __device__ __forceinline__ ChunkStates(const sys_selective_scan_t& p, const void* from, long long batch_stride, long long row, const ScanPlace& at, int rows)
    {
        const int n = (int)threadIdx.x % (4 * NS);
        const T* column = (const T*)from + at.batch * batch_stride + (size_t)at.group * p.states + (n < p.states ? n : p.states - 1);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if (i * kScanThreads >= rows * 4 * NS) break;
            const int t = at.begin + (i * kScanThreads + (int)threadIdx.x) / (4 * NS);
            v[i] = column[(t < p.length ? t : p.length - 1) * row];
        }
    }
    __device__ __forceinline__ void store(float* lds, int states, const ScanPlace& at, int rows) const
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if (i * kScanThreads >= rows * 4 * NS) break;
            const int k = i * kScanThreads + (int)threadIdx.x;
            lds[k] = k % (4 * NS) < states && at.begin + k / (4 * NS) < at.length ? (float)v[i] : 0.0f;
        }
    }
};

// A lane's column of a tensor: positions 4k + part of a span.  One offset is kept; the others are added up where they are used, behind a wall
// that stops the compiler from keeping all of them in registers that the states need.
template <typename T, int OWN>
struct OwnColumn {
    RowBuffer<T> rows;
    unsigned at, step;
    __device__ __forceinline__ OwnColumn(const void* base, long long batch_stride, long long row, int channels, const ScanPlace& place, int end)
        : rows(base ? (const T*)base + place.batch * batch_stride : nullptr, row, channels, place.begin, end), at(rows.offset((int)(threadIdx.x & 3), place.channel)),
          step(rows.offset(4, 0))
    {
        if (!base) rows.left = -1;
    }
    __device__ __forceinline__ void load(int down, unsigned (&v)[OWN]) const
    {
        const __amdgpu_buffer_rsrc_t buffer = rows.tile(down);
        unsigned first = at;
        asm volatile("" : "+v"(first));
#pragma unroll
        for (int k = 0; k < OWN; ++k) v[k] = buffer_load<T>(buffer, first + k * step);
    }
    // positions from place.end on are not written, nor are channels that are not there
    __device__ __forceinline__ void store(const ScanPlace& place, int down, const float (&v)[OWN]) const
    {
        const __amdgpu_buffer_rsrc_t buffer = rows.tile(down);
        unsigned first = at;
        asm volatile("" : "+v"(first));
#pragma unroll
        for (int k = 0; k < OWN; ++k) buffer_store<T>(buffer, place.there ? first + k * step : kNowhere, (T)v[k]);
    }
};

// What the lanes of a wavefront have written to LDS can be read by its others from here on.  Its accesses are carried out in order, so this only keeps the compiler
// from moving them; no instruction comes of it.
__device__ __forceinline__ void wavefront_sees_lds()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <typename F>
__device__ __forceinline__ void four_steps(F&& f)
{
    f(std::integral_constant<int, 0>());
    f(std::integral_constant<int, 1>());
    f(std::integral_constant<int, 2>());
    f(std::integral_constant<int, 3>());
}

template <typename T, int NS>
__global__ __launch_bounds__(kScanThreads) void scan_ends_kernel(sys_selective_scan_t p, ScanArgs a, GradShape shape)
{
    constexpr int kS = kSpan<NS>, kRows = kMostSpans * kS, kWidth = 4 * NS, kOwn = kS / 4;
    const ScanPlace at = scan_place(p, shape, a.lengths, xcd_place(blockIdx.x, gridDim.x));
    const int part = threadIdx.x & 3, n0 = part * NS;
    const Workspace w = workspace_of(p, shape, kWidth);
    float *ends = a.workspace, *back = ends + w.back;
    const size_t entry = (size_t)at.batch * shape.chunks + at.chunk, row = entry * p.channels + at.channel;
    float* spans = ends + w.spans + (entry * (shape.spans - 1) * p.channels + at.channel) * kWidth + n0;
    float* sums = ends + w.sums + entry * shape.spans * p.channels + at.channel;
    __shared__ __attribute__((aligned(16))) float tile_b[kRows * kWidth], tile_c[kRows * kWidth];
    const ChunkStates<T, NS> states_b(p, a.b, p.b_batch, p.b_row, at, shape.chunk_rows), states_c(p, a.c, p.c_batch, p.c_row, at, shape.chunk_rows);
    const OwnColumn<T, kOwn> u(a.u, p.u_batch, p.u_row, p.channels, at, at.length), delta(a.delta, p.delta_batch, p.delta_row, p.channels, at, at.length);
    const OwnColumn<T, kOwn> dy(a.dy, p.y_batch, p.y_row, p.channels, at, at.length), z(a.z, p.z_batch, p.z_row, p.channels, at, at.length);
    unsigned next_u[kOwn], next_delta[kOwn], next_dy[kOwn], next_z[kOwn];
    auto fetch = [&](int down) {
        u.load(down, next_u);
        delta.load(down, next_delta);
        dy.load(down, next_dy);
        z.load(down, next_z);
    };
    fetch(0);
    const float bias = a.delta_bias ? a.delta_bias[at.channel] : 0.0f;
    float decay[NS], h[NS], product[NS], own_back[NS], s_sum = 0.0f;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        decay[i] = n0 + i < p.states ? a.a[(size_t)at.channel * p.states + n0 + i] * kLog2e : 0.0f;
        h[i] = own_back[i] = 0.0f;
        product[i] = 1.0f;
    }
    states_b.store(tile_b, p.states, at, shape.chunk_rows);
    states_c.store(tile_c, p.states, at, shape.chunk_rows);
    __syncthreads();
#pragma unroll 1
    for (int down = 0; down < shape.chunk_rows; down += kS) {
        float own_s[kOwn], own_x[kOwn], own_e[kOwn];
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            const bool on = at.begin + down + 4 * k + part < at.length;
            const float pre = loaded<T>(next_delta[k]) + bias;
            own_s[k] = on ? (p.softplus ? softplus(pre) : pre) : 0.0f;
            own_x[k] = on ? own_s[k] * loaded<T>(next_u[k]) : 0.0f;
            own_e[k] = on ? loaded<T>(next_dy[k]) : 0.0f;
            if (a.z) own_e[k] *= on ? silu(loaded<T>(next_z[k])) : 0.0f;
        }
        float span_sum = 0.0f;
#pragma unroll
        for (int k = 0; k < kOwn; ++k) span_sum += own_s[k];
        s_sum += quad_sum(span_sum);
        if (at.there && part == 0) *sums = s_sum;          // at the end of this span
        sums += p.channels;
        fetch(down + kS);                              // (past the end: zeros)
        if (down && at.there) {
            Channels<float, NS>::store(spans, h);
            spans += (size_t)p.channels * kWidth;
        }
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            four_steps([&](auto lane) {
                constexpr int j = decltype(lane)::value;
                const float s = quad_take<j>(own_s[k]), x = quad_take<j>(own_x[k]), e = quad_take<j>(own_e[k]);
                float bt[NS], ct[NS];
                take<NS>(tile_b + (down + 4 * k + j) * kWidth + n0, bt);
                take<NS>(tile_c + (down + 4 * k + j) * kWidth + n0, ct);
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    const float decayed = fast_exp2(s * decay[i]);
                    h[i] = __builtin_fmaf(decayed, h[i], x * bt[i]);
                    product[i] *= decayed;
                    own_back[i] = __builtin_fmaf(ct[i] * e, product[i], own_back[i]);
                }
            });
        }
    }
    if (!at.there) return;
    Channels<float, NS>::store(ends + row * kWidth + n0, h);
    Channels<float, NS>::store(back + row * kWidth + n0, own_back);
}

// A lane a (sequence, channel, state): the state before every chunk and the gradient behind it, in place of what the chunks left.
__global__ __launch_bounds__(kScanThreads) void scan_chain_kernel(sys_selective_scan_t p, ScanArgs a, GradShape shape, int width)
{
    const long long lane = (long long)blockIdx.x * kScanThreads + threadIdx.x;
    const int n = (int)(lane % width);
    const long long channel_of = lane / width;
    const int d = (int)(channel_of % p.channels);
    const long long b = channel_of / p.channels;
    if (b >= p.batch) return;
    const Workspace w = workspace_of(p, shape, width);
    float *ends = a.workspace, *back = ends + w.back;
    const float* sums = ends + w.sums;                 // of whole chunks: behind their last spans
    const bool is = n < p.states;
    const float decay = is ? a.a[(size_t)d * p.states + n] * kLog2e : 0.0f;
    const size_t state = ((size_t)b * p.channels + d) * p.states + n;
    const size_t first = ((size_t)b * shape.chunks) * p.channels + d;
    constexpr int kAhead = 8;                          // loads in flight
    float h = is && a.state ? a.state[state] : 0.0f;
    for (int k0 = 0; k0 < shape.chunks; k0 += kAhead) {
        float end[kAhead], factor[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const size_t row = first + (size_t)(k0 + k < shape.chunks ? k0 + k : k0) * p.channels;
            end[k] = ends[row * width + n];
            factor[k] = fast_exp2(sums[((row - d) * shape.spans + (shape.spans - 1) * (size_t)p.channels) + d] * decay);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (k0 + k >= shape.chunks) break;
            ends[(first + (size_t)(k0 + k) * p.channels) * width + n] = h;
            h = __builtin_fmaf(factor[k], h, end[k]);
        }
    }
    float g = is && a.dstate_out ? a.dstate_out[state] : 0.0f;
    for (int k0 = shape.chunks - 1; k0 >= 0; k0 -= kAhead) {
        float own[kAhead], factor[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const size_t row = first + (size_t)(k0 - k >= 0 ? k0 - k : k0) * p.channels;
            own[k] = back[row * width + n];
            factor[k] = fast_exp2(sums[((row - d) * shape.spans + (shape.spans - 1) * (size_t)p.channels) + d] * decay);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (k0 - k < 0) break;
            back[(first + (size_t)(k0 - k) * p.channels) * width + n] = g;
            g = __builtin_fmaf(factor[k], g, own[k]);
        }
    }
    if (is && a.dstate) a.dstate[state] = g;
}

// 16 values a lane, added up over the lanes whose numbers differ in bits 3 to 5: the lane keeps the values
// 8 bit5 + 4 bit4 + 2 bit3 + {0, 1}.  A swap of halves (or of rows of 16) between two registers puts what one half needs of both next to
// each other, so a step is a swap and an addition for two values.
__device__ __forceinline__ void add_over_channels(float (&v)[16], float (&out)[2])
{
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v[k]), __builtin_bit_cast(unsigned, v[k + 8]), false, false);
        const unsigned r0 = r[0], r1 = r[1];       // (a bit_cast of r[1] itself takes r[0])
        v[k] = __builtin_bit_cast(float, r0) + __builtin_bit_cast(float, r1);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v[k]), __builtin_bit_cast(unsigned, v[k + 4]), false, false);
        const unsigned r0 = r[0], r1 = r[1];       // (a bit_cast of r[1] itself takes r[0])
        v[k] = __builtin_bit_cast(float, r0) + __builtin_bit_cast(float, r1);
    }
    const bool high = threadIdx.x & 8;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const float give = high ? v[k] : v[k + 2], keep = high ? v[k + 2] : v[k];
        out[k] = keep + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, give), 0x128, 0xF, 0xF, true));   // lane ^ 8 of the row
    }
}

template <typename T, int NS, bool GATE>
__global__ __launch_bounds__(kScanThreads) void scan_grad_kernel(sys_selective_scan_t p, ScanArgs a, GradShape shape)
{
    constexpr int kS = kSpan<NS>, kRows = kMostSpans * kS, kWidth = 4 * NS, kOwn = kS / 4;
    const unsigned block = xcd_place(blockIdx.x, gridDim.x);
    const ScanPlace at = scan_place(p, shape, a.lengths, block);
    const int part = threadIdx.x & 3, n0 = part * NS, wave = threadIdx.x >> 6, own_channel = threadIdx.x >> 2;
    const Workspace w = workspace_of(p, shape, kWidth);
    const float *ends = a.workspace, *back = ends + w.back;
    const size_t entry = (size_t)at.batch * shape.chunks + at.chunk, row = entry * p.channels + at.channel;
    const float* spans = ends + w.spans + (entry * (shape.spans - 1) * p.channels + at.channel) * kWidth + n0;
    const float* sums = ends + w.sums + entry * shape.spans * p.channels + at.channel;
    typedef float F4 __attribute__((ext_vector_type(4)));
    __shared__ __attribute__((aligned(16))) float tile_b[kRows * kWidth], tile_c[kRows * kWidth];
    // s, x and e of a span: written by the lane that owns a position, read by the four of its channel, which are of one wavefront (no barrier of the workgroup)
    __shared__ F4 steps[kS][kScanChannels];
    __shared__ __attribute__((aligned(16))) float parts[kParts][kS * 2 * kWidth];   // sums over channels: [position][dB | dC][state]

    const ChunkStates<T, NS> states_b(p, a.b, p.b_batch, p.b_row, at, shape.chunk_rows), states_c(p, a.c, p.c_batch, p.c_row, at, shape.chunk_rows);
    const OwnColumn<T, kOwn> u(a.u, p.u_batch, p.u_row, p.channels, at, at.length), delta(a.delta, p.delta_batch, p.delta_row, p.channels, at, at.length);
    const OwnColumn<T, kOwn> dy(a.dy, p.y_batch, p.y_row, p.channels, at, at.length), z(GATE ? a.z : nullptr, p.z_batch, p.z_row, p.channels, at, at.length);
    const long long values = (long long)p.length * p.channels;
    const OwnColumn<T, kOwn> du(a.du, values, p.channels, p.channels, at, at.end), ddelta(a.ddelta, values, p.channels, p.channels, at, at.end);
    const OwnColumn<T, kOwn> dz(GATE ? a.dz : nullptr, values, p.channels, p.channels, at, at.end);
    unsigned next_u[kOwn], next_delta[kOwn], next_dy[kOwn], next_z[kOwn];
    float next_state[NS], next_sum;
    auto fetch = [&](int span) {
        u.load(span * kS, next_u);
        delta.load(span * kS, next_delta);
        dy.load(span * kS, next_dy);
        z.load(span * kS, next_z);
        if (span) {                                    // (the first span begins with the chunk's state)
            Channels<float, NS>::load(spans + (size_t)(span - 1) * p.channels * kWidth, next_state);
            next_sum = sums[(size_t)(span - 1) * p.channels];
        }
    };
    fetch(shape.spans - 1);
    const float bias = a.delta_bias ? a.delta_bias[at.channel] : 0.0f, skip = a.d ? a.d[at.channel] : 0.0f;
    float decay[NS], h0[NS], carry[NS], d_a[NS];
    Channels<float, NS>::load(ends + row * kWidth + n0, h0);
    Channels<float, NS>::load(back + row * kWidth + n0, carry);
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        decay[i] = n0 + i < p.states ? a.a[(size_t)at.channel * p.states + n0 + i] * kLog2e : 0.0f;
        h0[i] = at.there ? h0[i] : 0.0f;               // (a channel that is not there adds nothing to the sums)
        carry[i] = at.there ? carry[i] : 0.0f;
        d_a[i] = 0.0f;
    }
    states_b.store(tile_b, p.states, at, shape.chunk_rows);
    states_c.store(tile_c, p.states, at, shape.chunk_rows);
    __syncthreads();

    float d_skip = 0.0f, d_bias = 0.0f;
#pragma unroll 1
    for (int span = shape.spans - 1; span >= 0; --span) {
        const int t_span = at.begin + span * kS;
        float state[kS + 1][NS], decayed[kS][NS];
        float own_s[kOwn], own_e[kOwn], own_u[kOwn], own_slope[kOwn], own_dz[kOwn];
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            const bool on = at.there && t_span + 4 * k + part < at.length;
            const float pre = loaded<T>(next_delta[k]) + bias;
            own_s[k] = on ? (p.softplus ? softplus(pre) : pre) : 0.0f;
            own_slope[k] = p.softplus ? sigmoid(pre) : 1.0f;
            own_u[k] = on ? loaded<T>(next_u[k]) : 0.0f;
            own_e[k] = on ? loaded<T>(next_dy[k]) : 0.0f;
            if (GATE) {
                const float gate = on ? loaded<T>(next_z[k]) : 0.0f, open = sigmoid(gate);
                own_dz[k] = own_e[k] * open * __builtin_fmaf(gate, 1.0f - open, 1.0f);
                own_e[k] *= gate * open;
            }
            steps[4 * k + part][own_channel] = F4{own_s[k], own_s[k] * own_u[k], own_e[k], 0.0f};
        }
        wavefront_sees_lds();
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            const float from_start = at.there ? next_state[i] : 0.0f;
            state[0][i] = span ? __builtin_fmaf(fast_exp2(next_sum * decay[i]), h0[i], from_start) : h0[i];
        }
        fetch(span ? span - 1 : 0);                    // (the first span's come once more, and are not used)
        // the states of this span
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            float sums_of[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const F4 step = steps[4 * k + j][own_channel];
                float bt[NS], ct[NS], sum = 0.0f;
                take<NS>(tile_b + (span * kS + 4 * k + j) * kWidth + n0, bt);
                if (GATE) take<NS>(tile_c + (span * kS + 4 * k + j) * kWidth + n0, ct);
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    decayed[4 * k + j][i] = fast_exp2(step[0] * decay[i]);
                    state[4 * k + j + 1][i] = __builtin_fmaf(decayed[4 * k + j][i], state[4 * k + j][i], step[1] * bt[i]);
                    if (GATE) sum = __builtin_fmaf(ct[i], state[4 * k + j + 1][i], sum);
                }
                sums_of[j] = sum;
            }
            if (GATE) own_dz[k] *= __builtin_fmaf(skip, own_u[k], quad_sums(sums_of));
        }
        if (GATE) {
#pragma unroll
            for (int k = 0; k < kOwn; ++k) own_dz[k] = t_span + 4 * k + part < at.length ? own_dz[k] : 0.0f;
            dz.store(at, span * kS, own_dz);
        }
        // and the gradient, from its end
        constexpr int kBatch = NS >= 8 ? 1 : 8 / NS;         // positions whose 16 values are added up together
        float values_of[NS == 16 ? 2 : 1][16], own_du[kOwn], own_ddelta[kOwn];
#pragma unroll
        for (int k = kOwn - 1; k >= 0; --k) {
            float gb_of[4], qa_of[4];
#pragma unroll
            for (int j = 3; j >= 0; --j) {
                const int t = 4 * k + j;                     // within the span
                const F4 step = steps[t][own_channel];
                const float s = step[0], x = step[1], e = step[2];
                float bt[NS], ct[NS], gb = 0.0f, qa = 0.0f;
                take<NS>(tile_b + (span * kS + t) * kWidth + n0, bt);
                take<NS>(tile_c + (span * kS + t) * kWidth + n0, ct);
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    const float g = __builtin_fmaf(ct[i], e, carry[i]);
                    if constexpr (NS == 16) {
                        values_of[0][i] = g * x;
                        values_of[1][i] = state[t + 1][i] * e;
                    } else {
                        values_of[0][(t % kBatch) * 2 * NS + i] = g * x;
                        values_of[0][(t % kBatch) * 2 * NS + NS + i] = state[t + 1][i] * e;
                    }
                    gb = __builtin_fmaf(g, bt[i], gb);
                    carry[i] = g * decayed[t][i];
                    const float q = carry[i] * state[t][i];
                    d_a[i] = __builtin_fmaf(q, s, d_a[i]);
                    qa = __builtin_fmaf(q, decay[i], qa);
                }
                gb_of[j] = gb;
                qa_of[j] = qa;
                if (t % kBatch == 0) {
                    const int high = ((threadIdx.x >> 5) & 1) * 8 + ((threadIdx.x >> 4) & 1) * 4 + ((threadIdx.x >> 3) & 1) * 2;
                    float* to = parts[wave * 2 + ((threadIdx.x >> 2) & 1)];
#pragma unroll
                    for (int set = 0; set < (NS == 16 ? 2 : 1); ++set) {
                        float sum[2];
                        add_over_channels(values_of[set], sum);
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            const int v = high + m;
                            if constexpr (NS == 16) to[(t * 2 + set) * kWidth + n0 + v] = sum[m];
                            else to[((t + v / (2 * NS)) * 2 + (v / NS) % 2) * kWidth + n0 + v % NS] = sum[m];
                        }
                    }
                }
            }
            const bool on = at.there && t_span + 4 * k + part < at.length;
            const float gb = quad_sums(gb_of), qa = quad_sums(qa_of);
            const float ds = __builtin_fmaf(gb, own_u[k], qa * kLn2);            // (decay is A log2 e)
            own_ddelta[k] = on ? ds * own_slope[k] : 0.0f;
            own_du[k] = on ? __builtin_fmaf(gb, own_s[k], skip * own_e[k]) : 0.0f;
            d_skip = __builtin_fmaf(own_e[k], own_u[k], d_skip);
            d_bias += own_ddelta[k];
        }
        du.store(at, span * kS, own_du);
        ddelta.store(at, span * kS, own_ddelta);
        __syncthreads();
        {
            const int channel_block = block % shape.channel_blocks;
            float* to = a.workspace + w.states + (((size_t)channel_block * p.batch + at.batch) * p.length + t_span) * (2 * kWidth);
            for (int k = threadIdx.x; k < kS * 2 * kWidth; k += kScanThreads) {
                if (t_span + k / (2 * kWidth) >= at.end) break;
                float sum = parts[0][k];
#pragma unroll
                for (int m = 1; m < kParts; ++m) sum += parts[m][k];
                to[k] = sum;
            }
        }
        __syncthreads();
    }
    d_skip = quad_sum(d_skip);
    d_bias = quad_sum(d_bias);
    if (!at.there) return;
    float* to = a.workspace + w.params + row * (kWidth + 2);
#pragma unroll
    for (int i = 0; i < NS; ++i) to[n0 + i] = d_a[i];
    if (part == 0) {
        to[kWidth] = d_skip;
        to[kWidth + 1] = d_bias;
    }
}

// The first `state_blocks` workgroups: dB and dC, a lane an element.  The others: dA, dD and ddelta_bias, 16 columns x 16 shares of the
// sequences and chunks a workgroup.
template <typename T>
__global__ __launch_bounds__(kScanThreads) void scan_sums_kernel(sys_selective_scan_t p, ScanArgs a, GradShape shape, int width, unsigned state_blocks)
{
    const Workspace w = workspace_of(p, shape, width);
    if (blockIdx.x < state_blocks) {
        const long long i = (long long)blockIdx.x * kScanThreads + threadIdx.x;
        const long long all = (long long)p.batch * p.length * p.groups * p.states;
        if (i >= 2 * all) return;
        const bool is_c = i >= all;
        long long rest = is_c ? i - all : i;
        const long long to = rest;
        const int n = (int)(rest % p.states);
        rest /= p.states;
        const int group = (int)(rest % p.groups);
        rest /= p.groups;                              // batch * length + t
        const int b = (int)(rest / p.length), t = (int)(rest - (long long)b * p.length);
        float s = 0.0f;
        if (t < sequence_length(a.lengths, b, p.length)) {
            for (int k = 0; k < shape.blocks_a_group; ++k)
                s += a.workspace[w.states + ((((size_t)(group * shape.blocks_a_group + k) * p.batch + b) * p.length + t) * 2 + is_c) * width + n];
        }
        ((T*)(is_c ? a.dc : a.db))[to] = (T)s;
        return;
    }
    const int columns = width + 2;
    const long long column = (long long)(blockIdx.x - state_blocks) * 16 + (threadIdx.x & 15);
    const int share = threadIdx.x >> 4;
    const bool there = column < (long long)p.channels * columns;
    float s = 0.0f;
    if (there)
        for (int k = share; k < p.batch * shape.chunks; k += 16) s += a.workspace[w.params + (size_t)k * p.channels * columns + column];
    __shared__ float shared[16][16];
    shared[share][threadIdx.x & 15] = s;
    __syncthreads();
    if (share || !there) return;
    for (int k = 1; k < 16; ++k) s += shared[k][threadIdx.x];
    const int d = (int)(column / columns), n = (int)(column - (long long)d * columns);
    if (n < p.states) a.da[(size_t)d * p.states + n] = s;
    else if (n == width && a.dd) a.dd[d] = s;
    else if (n == width + 1 && a.ddelta_bias) a.ddelta_bias[d] = s;
}

template <typename T, int NS>
hipError_t launch_states(const sys_selective_scan_t& p, const ScanArgs& a, hipStream_t s)
{
    const GradShape shape = backward_shape(p);
    const long long blocks = (long long)shape.channel_blocks * shape.chunks * p.batch;
    const long long chains = ((long long)p.batch * p.channels * (4 * NS) + kScanThreads - 1) / kScanThreads;
    const long long state_blocks = (2LL * p.batch * p.length * p.groups * p.states + kScanThreads - 1) / kScanThreads;
    const long long param_blocks = ((long long)p.channels * (4 * NS + 2) + 15) / 16;
    if (blocks > 0x7fffffffLL || chains > 0x7fffffffLL || state_blocks + param_blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    hipError_t e;
    if (blocks) {
        hipLaunchKernelGGL((scan_ends_kernel<T, NS>), dim3((unsigned)blocks), dim3(kScanThreads), 0, s, p, a, shape);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (chains) {
        hipLaunchKernelGGL(scan_chain_kernel, dim3((unsigned)chains), dim3(kScanThreads), 0, s, p, a, shape, 4 * NS);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (blocks) {
        if (a.z) hipLaunchKernelGGL((scan_grad_kernel<T, NS, true>), dim3((unsigned)blocks), dim3(kScanThreads), 0, s, p, a, shape);
        else hipLaunchKernelGGL((scan_grad_kernel<T, NS, false>), dim3((unsigned)blocks), dim3(kScanThreads), 0, s, p, a, shape);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    hipLaunchKernelGGL((scan_sums_kernel<T>), dim3((unsigned)(state_blocks + param_blocks)), dim3(kScanThreads), 0, s, p, a, shape, 4 * NS, (unsigned)state_blocks);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_type(const sys_selective_scan_t& p, const ScanArgs& a, hipStream_t s)
{
    switch (scan_states_a_lane(p.states)) {
    case 1: return launch_states<T, 1>(p, a, s);
    case 2: return launch_states<T, 2>(p, a, s);
    case 4: return launch_states<T, 4>(p, a, s);
    case 8: return launch_states<T, 8>(p, a, s);
    default: return launch_states<T, 16>(p, a, s);
    }
}

}  // namespace

int scan_grad_spans(const sys_selective_scan_t& p) { return backward_shape(p).spans; }

hipError_t launch_scan_grad(const sys_selective_scan_t& p, const ScanArgs& a, hipStream_t s)
{
    switch (p.dtype) {
    case SYS_F32: return launch_type<float>(p, a, s);
    case SYS_F16: return launch_type<f16_t>(p, a, s);
    default: return launch_type<bf16_t>(p, a, s);
    }
}

size_t scan_grad_workspace(const sys_selective_scan_t& p)
{
    return workspace_of(p, backward_shape(p), 4 * scan_states_a_lane(p.states)).floats * sizeof(float);
}

}  // namespace sysconv
