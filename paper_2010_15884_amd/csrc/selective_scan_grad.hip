// Gradients of the selective scan.  With a_t = e^(s_t A), x_t = s_t u_t and e_t = dy_t silu(z_t) (dy_t without a gate):
//
//   g_t  = C_t e_t + a_{t+1} g_{t+1}                       gradient of h_t, from the end (there: the gradient of state_out)
//   du_t = D e_t + s_t sum_n g_t B_t,   ds_t = u_t sum_n g_t B_t + sum_n A q_t,   q_t = g_t a_t h_{t-1},   ddelta_t = ds_t softplus'
//   dA   = sum_t q_t s_t,  dB_t = sum_d g_t x_t,  dC_t = sum_d h_t e_t,  dD = sum_t e_t u_t,  dz_t = dy_t (sum_n C_t h_t + D u_t) silu'(z_t)
//
// Both recurrences run along the positions, one from each end.  The positions are cut into chunks:
//   scan_ends_kernel    every chunk from a zero start: the state at its end, sum s, and what its positions hand back to the one before
//                       it, sum_t (a_first .. a_t) C_t e_t -- with the running product, so one sweep serves both directions;
//   scan_chain_kernel   along the chunks: the state before each, the gradient behind each;
//   scan_grad_kernel    every chunk again, from those: the states forward, a copy every few positions; then, backwards, these few
//                       positions' states and decays once more into registers and the recurrence of the gradient over them;
//   scan_sums_kernel    adds up what the workgroups have summed over their channels (dB, dC) and their positions (dA, dD, ddelta_bias).
// Each sum has a fixed order.
#include "launch.h"
#include "sequence.h"
#include "scan_tile.h"

namespace sysconv {
namespace {

// Positions whose states and decays are in registers at a time: 64 of each a lane at most; and those of a chunk.
template <int NS> constexpr int kSpan = NS <= 4 ? 16 : 64 / NS;
template <int NS> constexpr int kChunk = 4 * kSpan<NS>;
constexpr int kParts = 8;            // partial sums over channels in a workgroup: two a wavefront

int chunk_rows_of(int states)
{
    const int ns = scan_states_a_lane(states);
    return 4 * (ns <= 4 ? 16 : 64 / ns);
}

ScanShape backward_shape(const sys_selective_scan_t& p)
{
    ScanShape s;
    s.channels_a_group = p.channels / p.groups;
    s.blocks_a_group = (s.channels_a_group + kScanChannels - 1) / kScanChannels;
    s.channel_blocks = s.blocks_a_group * p.groups;
    s.chunk_rows = chunk_rows_of(p.states);
    s.chunks = (p.length + s.chunk_rows - 1) / s.chunk_rows;
    return s;
}

// The workspace: where its parts begin, in floats.
struct Workspace {
    size_t back;                   // [batch][chunk][channel][width], behind the same for `ends` at 0
    size_t sums;                   // [batch][chunk][channel]
    size_t params;                 // [batch][chunk][channel][width + 2]: dA, dD, ddelta_bias
    size_t states;                 // [channel block][batch][position][dB | dC][width]
    size_t floats;
};

__host__ __device__ Workspace workspace_of(const sys_selective_scan_t& p, const ScanShape& shape, int width)
{
    Workspace w;
    const size_t rows = (size_t)p.batch * shape.chunks * p.channels;
    w.back = rows * width;
    w.sums = w.back + rows * width;
    w.params = w.sums + rows;
    w.states = w.params + rows * (width + 2);
    w.floats = w.states + (size_t)shape.channel_blocks * p.batch * p.length * 2 * width;
    return w;
}

// What a lane owns of four positions 4k + part.
struct Own {
    float u, s, pre, dy, z;
};

template <typename T>
struct Columns {
    const T *u, *delta, *z, *dy;
    float bias;
    __device__ __forceinline__ Columns(const sys_selective_scan_t& p, const ScanArgs& a, const ScanPlace& at)
        : u((const T*)a.u + at.batch * p.u_batch + at.channel), delta((const T*)a.delta + at.batch * p.delta_batch + at.channel),
          z(a.z ? (const T*)a.z + at.batch * p.z_batch + at.channel : nullptr), dy((const T*)a.dy + at.batch * p.y_batch + at.channel),
          bias(a.delta_bias ? a.delta_bias[at.channel] : 0.0f)
    {
    }
    __device__ __forceinline__ Own load(const sys_selective_scan_t& p, const ScanPlace& at, int t) const
    {
        Own o = {};
        const bool on = at.there && t < at.length && t < at.end;
        if (on) {
            o.u = (float)u[t * p.u_row];
            o.pre = (float)delta[t * p.delta_row] + bias;
            o.dy = (float)dy[t * p.y_row];
            if (z) o.z = (float)z[t * p.z_row];
            o.s = p.softplus ? softplus(o.pre) : o.pre;
        }
        return o;
    }
};

// B and C of a chunk in LDS, [position][4 NS].
template <typename T, int NS>
__device__ __forceinline__ void load_states(const sys_selective_scan_t& p, const void* from, long long batch_stride, long long row, const ScanPlace& at, float* lds)
{
    const T* rows = (const T*)from + at.batch * batch_stride + (size_t)at.group * p.states;
    for (int k = threadIdx.x; k < kChunk<NS> * 4 * NS; k += kScanThreads) {
        const int t = at.begin + k / (4 * NS), n = k % (4 * NS);
        lds[k] = t < at.length && n < p.states ? (float)rows[t * row + n] : 0.0f;
    }
}

template <typename F>
__device__ __forceinline__ void four_steps(F&& f)
{
    f(std::integral_constant<int, 0>());
    f(std::integral_constant<int, 1>());
    f(std::integral_constant<int, 2>());
    f(std::integral_constant<int, 3>());
}

template <typename F>
__device__ __forceinline__ void four_steps_back(F&& f)
{
    f(std::integral_constant<int, 3>());
    f(std::integral_constant<int, 2>());
    f(std::integral_constant<int, 1>());
    f(std::integral_constant<int, 0>());
}

template <typename T, int NS>
__global__ __launch_bounds__(kScanThreads) void scan_ends_kernel(sys_selective_scan_t p, ScanArgs a, ScanShape shape)
{
    const ScanPlace at = scan_place(p, shape, a.lengths, blockIdx.x);
    const int part = threadIdx.x & 3, n0 = part * NS;
    const Workspace w = workspace_of(p, shape, 4 * NS);
    float *ends = a.workspace, *back = ends + w.back, *sums = ends + w.sums;
    __shared__ __attribute__((aligned(16))) float tile_b[kChunk<NS> * 4 * NS], tile_c[kChunk<NS> * 4 * NS];
    load_states<T, NS>(p, a.b, p.b_batch, p.b_row, at, tile_b);
    load_states<T, NS>(p, a.c, p.c_batch, p.c_row, at, tile_c);
    const Columns<T> columns(p, a, at);
    float decay[NS], h[NS], product[NS], own_back[NS], s_sum = 0.0f;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        decay[i] = n0 + i < p.states ? a.a[(size_t)at.channel * p.states + n0 + i] * kLog2e : 0.0f;
        h[i] = own_back[i] = 0.0f;
        product[i] = 1.0f;
    }
    __syncthreads();
    for (int k = 0; k < kChunk<NS> / 4; ++k) {
        const Own o = columns.load(p, at, at.begin + 4 * k + part);
        const float e_own = a.z ? o.dy * silu(o.z) : o.dy, x_own = o.s * o.u;
        s_sum += o.s;
        four_steps([&](auto lane) {
            constexpr int j = decltype(lane)::value;
            const float s = quad_take<j>(o.s), x = quad_take<j>(x_own), e = quad_take<j>(e_own);
            float bt[NS], ct[NS];
            take<NS>(tile_b + (4 * k + j) * 4 * NS + n0, bt);
            take<NS>(tile_c + (4 * k + j) * 4 * NS + n0, ct);
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                const float decayed = fast_exp2(s * decay[i]);
                h[i] = __builtin_fmaf(decayed, h[i], x * bt[i]);
                product[i] *= decayed;
                own_back[i] = __builtin_fmaf(ct[i] * e, product[i], own_back[i]);
            }
        });
    }
    if (!at.there) return;
    const size_t row = ((size_t)at.batch * shape.chunks + at.chunk) * p.channels + at.channel;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        ends[row * (4 * NS) + n0 + i] = h[i];
        back[row * (4 * NS) + n0 + i] = own_back[i];
    }
    s_sum = quad_sum(s_sum);
    if (part == 0) sums[row] = s_sum;
}

// A lane a (sequence, channel, state): the state before every chunk and the gradient behind it, in place of what the chunks left.
__global__ __launch_bounds__(kScanThreads) void scan_chain_kernel(sys_selective_scan_t p, ScanArgs a, ScanShape shape, int width)
{
    const long long lane = (long long)blockIdx.x * kScanThreads + threadIdx.x;
    const int n = (int)(lane % width);
    const long long channel_of = lane / width;
    const int d = (int)(channel_of % p.channels);
    const long long b = channel_of / p.channels;
    if (b >= p.batch) return;
    const Workspace w = workspace_of(p, shape, width);
    float *ends = a.workspace, *back = ends + w.back, *sums = ends + w.sums;
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
            factor[k] = fast_exp2(sums[row] * decay);
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
            factor[k] = fast_exp2(sums[row] * decay);
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
__global__ __launch_bounds__(kScanThreads) void scan_grad_kernel(sys_selective_scan_t p, ScanArgs a, ScanShape shape)
{
    constexpr int kS = kSpan<NS>, kRows = kChunk<NS>, kWidth = 4 * NS, kSpans = kRows / kS;
    const ScanPlace at = scan_place(p, shape, a.lengths, blockIdx.x);
    const int part = threadIdx.x & 3, n0 = part * NS, wave = threadIdx.x >> 6;
    const Workspace w = workspace_of(p, shape, kWidth);
    const float *ends = a.workspace, *back = ends + w.back;
    __shared__ __attribute__((aligned(16))) float tile_b[kRows * kWidth], tile_c[kRows * kWidth];
    __shared__ __attribute__((aligned(16))) float kept[kSpans][NS][kScanThreads];             // the state before every span
    __shared__ float kept_s[kRows / 4][kScanThreads], kept_x[kRows / 4][kScanThreads];        // what this lane owns
    __shared__ __attribute__((aligned(16))) float parts[kParts][kS * 2 * kWidth];             // sums over channels: [position][dB | dC][state]
    load_states<T, NS>(p, a.b, p.b_batch, p.b_row, at, tile_b);
    load_states<T, NS>(p, a.c, p.c_batch, p.c_row, at, tile_c);
    const Columns<T> columns(p, a, at);
    const size_t row = ((size_t)at.batch * shape.chunks + at.chunk) * p.channels + at.channel;
    float decay[NS], h[NS], carry[NS], d_a[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        decay[i] = n0 + i < p.states ? a.a[(size_t)at.channel * p.states + n0 + i] * kLog2e : 0.0f;
        h[i] = at.there ? ends[row * kWidth + n0 + i] : 0.0f;
        carry[i] = at.there ? back[row * kWidth + n0 + i] : 0.0f;
        d_a[i] = 0.0f;
    }
    const float skip = a.d ? a.d[at.channel] : 0.0f;
    __syncthreads();

    // forwards: the state before every span
#pragma unroll 1
    for (int span = 0; span < kSpans; ++span) {
#pragma unroll
        for (int i = 0; i < NS; ++i) kept[span][i][threadIdx.x] = h[i];
#pragma unroll 1
        for (int k = span * (kS / 4); k < (span + 1) * (kS / 4); ++k) {
            const Own o = columns.load(p, at, at.begin + 4 * k + part);
            const float x_own = o.s * o.u;
            kept_s[k][threadIdx.x] = o.s;
            kept_x[k][threadIdx.x] = x_own;
            if (span == kSpans - 1) continue;
            four_steps([&](auto lane) {
                constexpr int j = decltype(lane)::value;
                const float s = quad_take<j>(o.s), x = quad_take<j>(x_own);
                float bt[NS];
                take<NS>(tile_b + (4 * k + j) * kWidth + n0, bt);
#pragma unroll
                for (int i = 0; i < NS; ++i) h[i] = __builtin_fmaf(fast_exp2(s * decay[i]), h[i], x * bt[i]);
            });
        }
    }

    float d_skip = 0.0f, d_bias = 0.0f;
#pragma unroll 1
    for (int span = kSpans - 1; span >= 0; --span) {
        const int t_span = at.begin + span * kS;
        float state[kS + 1][NS], decayed[kS][NS];
        float own_s[kS / 4], own_x[kS / 4], own_e[kS / 4];
        Own own[kS / 4];
#pragma unroll
        for (int i = 0; i < NS; ++i) state[0][i] = kept[span][i][threadIdx.x];
        // the states of this span
#pragma unroll
        for (int k = 0; k < kS / 4; ++k) {
            const int t = t_span + 4 * k + part;
            own[k] = columns.load(p, at, t);
            own_s[k] = kept_s[span * (kS / 4) + k][threadIdx.x];
            own_x[k] = kept_x[span * (kS / 4) + k][threadIdx.x];
            own_e[k] = GATE ? own[k].dy * silu(own[k].z) : own[k].dy;
            float own_y = 0.0f;
            four_steps([&](auto lane) {
                constexpr int j = decltype(lane)::value;
                const float s = quad_take<j>(own_s[k]), x = quad_take<j>(own_x[k]);
                float bt[NS], ct[NS], sum = 0.0f;
                take<NS>(tile_b + (span * kS + 4 * k + j) * kWidth + n0, bt);
                if (GATE) take<NS>(tile_c + (span * kS + 4 * k + j) * kWidth + n0, ct);
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    decayed[4 * k + j][i] = fast_exp2(s * decay[i]);
                    state[4 * k + j + 1][i] = __builtin_fmaf(decayed[4 * k + j][i], state[4 * k + j][i], x * bt[i]);
                    if (GATE) sum = __builtin_fmaf(ct[i], state[4 * k + j + 1][i], sum);
                }
                if (GATE) {
                    sum = quad_sum(sum);
                    own_y = part == j ? sum : own_y;
                }
            });
            if (GATE && at.there && t < at.end) {
                const float y = __builtin_fmaf(skip, own[k].u, own_y);
                ((T*)a.dz)[((size_t)at.batch * p.length + t) * p.channels + at.channel] = (T)(t < at.length ? own[k].dy * y * silu_grad(own[k].z) : 0.0f);
            }
        }
        // and the gradient, from its end
        constexpr int kBatch = NS >= 8 ? 1 : 8 / NS;         // positions whose 16 values are added up together
        float values[NS == 16 ? 2 : 1][16];
#pragma unroll
        for (int k = kS / 4 - 1; k >= 0; --k) {
            float own_gb = 0.0f, own_qa = 0.0f;
            four_steps_back([&](auto lane) {
                constexpr int j = decltype(lane)::value;
                const int t = 4 * k + j;                     // within the span
                const float s = quad_take<j>(own_s[k]), x = quad_take<j>(own_x[k]), e = quad_take<j>(own_e[k]);
                float bt[NS], ct[NS], gb = 0.0f, qa = 0.0f;
                take<NS>(tile_b + (span * kS + t) * kWidth + n0, bt);
                take<NS>(tile_c + (span * kS + t) * kWidth + n0, ct);
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    const float g = __builtin_fmaf(ct[i], e, carry[i]);
                    if constexpr (NS == 16) {
                        values[0][i] = g * x;
                        values[1][i] = state[t + 1][i] * e;
                    } else {
                        values[0][(t % kBatch) * 2 * NS + i] = g * x;
                        values[0][(t % kBatch) * 2 * NS + NS + i] = state[t + 1][i] * e;
                    }
                    gb = __builtin_fmaf(g, bt[i], gb);
                    carry[i] = g * decayed[t][i];
                    const float q = carry[i] * state[t][i];
                    d_a[i] = __builtin_fmaf(q, s, d_a[i]);
                    qa = __builtin_fmaf(q, decay[i], qa);
                }
                gb = quad_sum(gb);
                qa = quad_sum(qa);
                own_gb = part == j ? gb : own_gb;
                own_qa = part == j ? qa : own_qa;
                if (t % kBatch == 0) {
                    const int high = ((threadIdx.x >> 5) & 1) * 8 + ((threadIdx.x >> 4) & 1) * 4 + ((threadIdx.x >> 3) & 1) * 2;
                    float* to = parts[wave * 2 + ((threadIdx.x >> 2) & 1)];
#pragma unroll
                    for (int set = 0; set < (NS == 16 ? 2 : 1); ++set) {
                        float sum[2];
                        add_over_channels(values[set], sum);
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            const int v = high + m;
                            if constexpr (NS == 16) to[(t * 2 + set) * kWidth + n0 + v] = sum[m];
                            else to[((t + v / (2 * NS)) * 2 + (v / NS) % 2) * kWidth + n0 + v % NS] = sum[m];
                        }
                    }
                }
            });
            const int t = t_span + 4 * k + part;
            const float ds = own_gb * own[k].u + own_qa * kLn2;                  // (decay is A log2 e)
            const float ddelta = p.softplus ? ds * sigmoid(own[k].pre) : ds;
            const bool on = at.there && t < at.length && t < at.end;
            d_skip += on ? own_e[k] * own[k].u : 0.0f;
            d_bias += on ? ddelta : 0.0f;
            if (at.there && t < at.end) {
                const size_t to = ((size_t)at.batch * p.length + t) * p.channels + at.channel;
                ((T*)a.du)[to] = (T)(on ? __builtin_fmaf(own_gb, own_s[k], skip * own_e[k]) : 0.0f);
                ((T*)a.ddelta)[to] = (T)(on ? ddelta : 0.0f);
            }
        }
        __syncthreads();
        {
            const int channel_block = blockIdx.x % shape.channel_blocks;
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
__global__ __launch_bounds__(kScanThreads) void scan_sums_kernel(sys_selective_scan_t p, ScanArgs a, ScanShape shape, int width, unsigned state_blocks)
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
    const ScanShape shape = backward_shape(p);
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
