// Norm of every head of queries and keys, with the rotation of positions in the same pass: z = x w r, r = 1 / sqrt(E[x^2] + eps) or
// 1 / sqrt(sum x^2 + eps); pairs (a, b) of the first `rotary` entries become (a c - b s, b c + a s).  Forward and gradients.
//
// Both tensors go through one launch.  A head lies with `parts` neighbouring lanes, each of which holds kSlots pairs of pieces of V entries
// that are turned with each other (or a first and a second half of what is not turned), so that no entry is needed in another lane; a wavefront runs `heads` heads
// of one token side by side and walks through the rest of them with the next ones' loads in flight: the tables' rows and the weights are
// loaded once a token.
// Bound by memory: 16-bit entries cost 4 bytes in the forward pass and some five vector instructions.  8192 tokens of 36 heads of 128 in bf16 take 32 us (4.9 TB/s, a
// copy's rate), the gradients of 18 heads of 256 62 us (56 and 5 for the join of the weights' sums by the profiler; 4.1 TB/s over the first; eight wavefronts a CU, which wait for 59 % of
// their time and keep the vector units busy for half of it), 32 tokens of 40 heads 4 us, a launch.
#include "launch.h"
#include "sequence.h"

namespace sysconv {
namespace {

constexpr int kThreads = 256;
constexpr int kWavesOf = kThreads / 64;

// How a call is laid on the chip.
struct NormPlan {
    int slots;                         // pairs of pieces of a head
    int turned;                        // of them, those that are turned
    int parts_log;                     // lanes a head
    int heads_log;                     // heads side by side
    int splits;                        // wavefronts that share a token's heads
    int each;                          // heads of one of them
    int all_heads;
    long long tokens;
    unsigned blocks;
};

// Sum over 2^log neighbouring lanes, every one of which gets it.
__device__ __forceinline__ float lanes_sum(float v, int log)
{
    if (log > 0) v += dpp<0xB1>(v);                // lanes 1 0 3 2
    if (log > 1) v += dpp<0x4E>(v);                // lanes 2 3 0 1
    if (log > 2) v += dpp<0x141>(v);               // the other half of 8
    if (log > 3) v += dpp<0x140>(v);               // the other half of 16
    if (log > 4) v += __shfl_xor(v, 16);
    if (log > 5) v += __shfl_xor(v, 32);
    return v;
}

// A lane's entries: where the pieces of its slots begin, and which row entries of the tables turn them.
template <int V, int S>
struct Slots {
    int first[S], second[S], angle[2][S];
    unsigned there, pairs, turned;     // a bit a slot: it exists, with a second piece, and is turned
    __device__ __forceinline__ Slots(const sys_head_norm_t& p, const NormPlan& n, int part) : there(0), pairs(0), turned(0)
    {
        const int tail = p.dim - p.rotary, half = (tail + 1) / 2;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const int s = part + (i << n.parts_log);
            const bool turn = s < n.turned, both = V == 1 && p.interleaved;
            const int f = turn ? (both ? 2 * s : s * V) : p.rotary + (s - n.turned) * V;
            const int g = turn ? (both ? 2 * s + 1 : p.rotary / 2 + s * V) : f + half;
            const bool is = s < n.slots, second_is = is && (turn || g < p.dim);
            first[i] = is ? f : 0;
            second[i] = second_is ? g : first[i];
            angle[0][i] = turn ? (p.interleaved && V > 1 ? f / 2 : s * V) : 0;
            angle[1][i] = turn ? g / 2 : 0;        // (interleaved pieces alone)
            there |= (unsigned)is << i, pairs |= (unsigned)second_is << i, turned |= (unsigned)turn << i;
        }
    }
    __device__ __forceinline__ bool is(int i) const { return there >> i & 1; }
    __device__ __forceinline__ bool has_second(int i) const { return pairs >> i & 1; }
    __device__ __forceinline__ bool turns(int i) const { return turned >> i & 1; }
};

// Cosines and sines of a lane's pairs at a row of the tables: [piece][pair] for interleaved pieces, else [0][entry].
template <int V, int S>
struct Angles {
    float c[S][V], s[S][V];
    __device__ __forceinline__ void load(const sys_head_norm_t& p, const HeadNormArgs& a, const Slots<V, S>& at, long long row)
    {
        const float* cosine = a.cosine + row * (p.rotary / 2);
        const float* sine = a.sine + row * (p.rotary / 2);
#pragma unroll
        for (int i = 0; i < S; ++i)
            if (at.turns(i)) {
                if (V > 1 && p.interleaved) {
                    constexpr int H = V > 1 ? V / 2 : 1;
                    Channels<float, H>::load(cosine + at.angle[0][i], *(float(*)[H])c[i]);
                    Channels<float, H>::load(sine + at.angle[0][i], *(float(*)[H])s[i]);
                    if (V > 1) {
                        Channels<float, H>::load(cosine + at.angle[1][i], *(float(*)[H])(c[i] + V / 2));
                        Channels<float, H>::load(sine + at.angle[1][i], *(float(*)[H])(s[i] + V / 2));
                    }
                } else {
                    Channels<float, V>::load(cosine + at.angle[0][i], c[i]);
                    Channels<float, V>::load(sine + at.angle[0][i], s[i]);
                }
            }
    }
    // sign -1: back
    __device__ __forceinline__ void turn(bool interleaved, int i, float sign, float (&x)[V], float (&y)[V]) const
    {
        if (V > 1 && interleaved) {
#pragma unroll
            for (int j = 0; j + 1 < V; j += 2) {
                const float a = x[j], b = x[j + 1], sa = sign * s[i][j / 2];
                x[j] = __builtin_fmaf(-b, sa, a * c[i][j / 2]), x[j + 1] = __builtin_fmaf(a, sa, b * c[i][j / 2]);
                const float d = y[j], e = y[j + 1], sd = sign * s[i][(V + j) / 2];
                y[j] = __builtin_fmaf(-e, sd, d * c[i][(V + j) / 2]), y[j + 1] = __builtin_fmaf(d, sd, e * c[i][(V + j) / 2]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float a = x[j], b = y[j], sa = sign * s[i][j];
                x[j] = __builtin_fmaf(-b, sa, a * c[i][j]), y[j] = __builtin_fmaf(a, sa, b * c[i][j]);
            }
        }
    }
};

// A token and the heads of it that a group of lanes walks through.
struct TokenPlace {
    long long token;
    int b, t, head, last, step;        // heads head, head + step, .. below last
    bool there;                        // within the sequence, and with a position
    long long row;                     // of the tables
};

__device__ __forceinline__ TokenPlace token_place(const sys_head_norm_t& p, const HeadNormArgs& a, const NormPlan& n, long long wave)
{
    TokenPlace at;
    const int lane = threadIdx.x & 63;
    const int tokens_log = 6 - n.parts_log - n.heads_log;              // side by side
    const int split = n.splits > 1 ? (int)(wave % n.splits) : 0;
    if (n.splits > 1) wave /= n.splits;
    at.token = (wave << tokens_log) + (lane >> (n.parts_log + n.heads_log));
    at.step = 1 << n.heads_log;
    at.head = split * n.each + ((lane >> n.parts_log) & (at.step - 1));
    at.last = split * n.each + n.each < n.all_heads ? split * n.each + n.each : n.all_heads;
    if (at.token >= n.tokens) {
        at.token = n.tokens - 1;
        at.last = 0;                                                   // nothing of it is stored
    }
    at.b = p.batch == 1 ? 0 : (int)(at.token / p.length);
    at.t = (int)(at.token - (long long)at.b * p.length);
    at.there = at.t < sequence_length(a.lengths, at.b, p.length);
    at.row = at.t;
    if (p.rotary && a.positions) {
        at.row = a.positions[at.token];
        at.there = at.there && at.row >= 0 && at.row < p.positions;
    }
    return at;
}

template <typename T, int V, int S>
__global__ __launch_bounds__(kThreads) void head_norm_kernel(sys_head_norm_t p, HeadNormArgs a, NormPlan n)
{
    const int part = threadIdx.x & ((1 << n.parts_log) - 1);
    const TokenPlace at = token_place(p, a, n, (long long)blockIdx.x * kWavesOf + (threadIdx.x >> 6));
    const Slots<V, S> slots(p, n, part);
    Angles<V, S> angles;
    if (at.there && p.rotary) angles.load(p, a, slots, at.row);
    float w[2][S][V];
    const void* w_of = nullptr;
    bool weights_loaded = false;
    const float share = p.norm == SYS_NORM_RMS ? 1.0f / (float)p.dim : 1.0f;
    const T* q = (const T*)a.q + at.b * p.q_batch + at.t * p.q_row;
    const T* k = (const T*)a.k + at.b * p.k_batch + at.t * p.k_row;
    T* yq = (T*)a.yq + at.b * p.yq_batch + at.t * p.yq_row;
    T* yk = (T*)a.yk + at.b * p.yk_batch + at.t * p.yk_row;
    typedef typename Channels<T, V>::Raw Raw;
    Raw next[2][S];
    auto fetch = [&](int head) {
        if (at.there && head < at.last) {
            const T* x = head < p.q_heads ? q + head * p.dim : k + (head - p.q_heads) * p.dim;
#pragma unroll
            for (int i = 0; i < S; ++i) {
                next[0][i] = Channels<T, V>::raw(x + slots.first[i]);
                next[1][i] = Channels<T, V>::raw(x + slots.second[i]);
            }
        }
    };
    fetch(at.head);
    for (int head = at.head; head < at.last; head += at.step) {
        float x[2][S][V], sum = 0.0f;
        if (at.there) {
#pragma unroll
            for (int i = 0; i < S; ++i) {
                Channels<T, V>::values(next[0][i], x[0][i]);
                Channels<T, V>::values(next[1][i], x[1][i]);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    if (S > 1 || V == 1) {
                        x[0][i][j] = slots.is(i) ? x[0][i][j] : 0.0f;
                        x[1][i][j] = slots.has_second(i) ? x[1][i][j] : 0.0f;
                    }
                    sum = __builtin_fmaf(x[0][i][j], x[0][i][j], sum);
                    sum = __builtin_fmaf(x[1][i][j], x[1][i][j], sum);
                }
                if (S == 1 && V > 1 && !slots.is(i)) sum = 0.0f;
            }
        }
        fetch(head + at.step);
        const bool is_q = head < p.q_heads;
        const void* weights = is_q ? a.wq : a.wk;
        if (!weights_loaded || weights != w_of) {
            weights_loaded = true, w_of = weights;
#pragma unroll
            for (int i = 0; i < S; ++i)
                if (weights) {
                    load_params<T, V>(weights, slots.first[i], p.param_dtype, w[0][i]);
                    load_params<T, V>(weights, slots.second[i], p.param_dtype, w[1][i]);
                } else {
#pragma unroll
                    for (int j = 0; j < V; ++j) w[0][i][j] = w[1][i][j] = 1.0f;
                }
        }
        sum = lanes_sum(sum, n.parts_log);
        // (the square root and the quotient are off by a unit each)
        const float r = 1.0f / __builtin_sqrtf(__builtin_fmaf(sum, share, p.eps));
        T* y = is_q ? yq + head * p.dim : yk + (head - p.q_heads) * p.dim;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            float f[V], g[V];
#pragma unroll
            for (int j = 0; j < V; ++j) f[j] = at.there ? x[0][i][j] * r * w[0][i][j] : 0.0f, g[j] = at.there ? x[1][i][j] * r * w[1][i][j] : 0.0f;
            if (at.there && slots.turns(i)) angles.turn(p.interleaved, i, 1.0f, f, g);
            if (slots.is(i)) {
                Channels<T, V>::store(y + slots.first[i], f);
                if (slots.has_second(i)) Channels<T, V>::store(y + slots.second[i], g);
            }
        }
    }
}

// Gradients.  With n = x r: dz = dy turned back, dw = sum dz n, dn = dz w, dx = r (dn - n share (n . dn)).  A wavefront goes through tokens in
// steps of the launch and keeps the sums of its columns in registers; they are joined in a workgroup and then over workgroups, in a fixed order.
template <typename T, int V, int S>
__global__ __launch_bounds__(kThreads) void head_norm_grad_kernel(sys_head_norm_t p, HeadNormArgs a, NormPlan n, long long waves)
{
    const int part = threadIdx.x & ((1 << n.parts_log) - 1);
    const Slots<V, S> slots(p, n, part);
    const float share = p.norm == SYS_NORM_RMS ? 1.0f / (float)p.dim : 1.0f;
    typedef typename Channels<T, V>::Raw Raw;
    float dw[2][2][S][V] = {};                                          // [q or k][piece]
    for (long long wave = (long long)blockIdx.x * kWavesOf + (threadIdx.x >> 6); wave < waves; wave += (long long)gridDim.x * kWavesOf) {
        const TokenPlace at = token_place(p, a, n, wave);
        Angles<V, S> angles;
        if (at.there && p.rotary) angles.load(p, a, slots, at.row);
        const T* q = (const T*)a.q + at.b * p.q_batch + at.t * p.q_row;
        const T* k = (const T*)a.k + at.b * p.k_batch + at.t * p.k_row;
        const T* dyq = (const T*)a.dyq + at.b * p.yq_batch + at.t * p.yq_row;
        const T* dyk = (const T*)a.dyk + at.b * p.yk_batch + at.t * p.yk_row;
        T* dq = (T*)a.yq + at.token * p.q_heads * p.dim;
        T* dk = (T*)a.yk + at.token * p.k_heads * p.dim;
        Raw next[4][S];
        auto fetch = [&](int head) {
            if (at.there && head < at.last) {
                const bool is_q = head < p.q_heads;
                const T* x = is_q ? q + head * p.dim : k + (head - p.q_heads) * p.dim;
                const T* dy = is_q ? dyq + head * p.dim : dyk + (head - p.q_heads) * p.dim;
#pragma unroll
                for (int i = 0; i < S; ++i) {
                    next[0][i] = Channels<T, V>::raw(x + slots.first[i]);
                    next[1][i] = Channels<T, V>::raw(x + slots.second[i]);
                    next[2][i] = Channels<T, V>::raw(dy + slots.first[i]);
                    next[3][i] = Channels<T, V>::raw(dy + slots.second[i]);
                }
            }
        };
        // the heads of q, then those of k: the sums' registers are named at compile time
        int head = at.head;
        fetch(head);
        auto run = [&](auto which) {
            constexpr int K = decltype(which)::value;
            const int last = K == 0 && p.q_heads < at.last ? p.q_heads : at.last;
            const void* weights = K ? a.wk : a.wq;
            float w[2][S][V];
#pragma unroll
            for (int i = 0; i < S; ++i)
                if (weights) {
                    load_params<T, V>(weights, slots.first[i], p.param_dtype, w[0][i]);
                    load_params<T, V>(weights, slots.second[i], p.param_dtype, w[1][i]);
                } else {
#pragma unroll
                    for (int j = 0; j < V; ++j) w[0][i][j] = w[1][i][j] = 1.0f;
                }
            for (; head < last; head += at.step) {
                float x[2][S][V], z[2][S][V], sum = 0.0f, dot = 0.0f;
                if (at.there) {
#pragma unroll
                    for (int i = 0; i < S; ++i) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            Channels<T, V>::values(next[h][i], x[h][i]);
                            Channels<T, V>::values(next[2 + h][i], z[h][i]);
                        }
                        if (slots.turns(i)) angles.turn(p.interleaved, i, -1.0f, z[0][i], z[1][i]);
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            if (S > 1 || V == 1) {
                                x[0][i][j] = slots.is(i) ? x[0][i][j] : 0.0f;
                                x[1][i][j] = slots.has_second(i) ? x[1][i][j] : 0.0f;
                                z[0][i][j] = slots.is(i) ? z[0][i][j] : 0.0f;
                                z[1][i][j] = slots.has_second(i) ? z[1][i][j] : 0.0f;
                            }
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                sum = __builtin_fmaf(x[h][i][j], x[h][i][j], sum);
                                dot = __builtin_fmaf(x[h][i][j], z[h][i][j] * w[h][i][j], dot);
                            }
                        }
                    }
                }
                fetch(head + at.step);
                if (S == 1 && V > 1 && !slots.is(0)) sum = dot = 0.0f;  // (a lane without entries has another's, whose products nobody takes)
                sum = lanes_sum(sum, n.parts_log);
                dot = lanes_sum(dot, n.parts_log);
                const float r = 1.0f / __builtin_sqrtf(__builtin_fmaf(sum, share, p.eps));
                const float along = r * r * (share * dot);              // of x: n share (n . dn) = x along
                T* dx = K ? dk + (head - p.q_heads) * p.dim : dq + head * p.dim;
#pragma unroll
                for (int i = 0; i < S; ++i) {
                    float f[2][V] = {};
                    if (at.there) {
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int j = 0; j < V; ++j) {
                                dw[K][h][i][j] = __builtin_fmaf(z[h][i][j], x[h][i][j] * r, dw[K][h][i][j]);
                                f[h][j] = r * __builtin_fmaf(-x[h][i][j], along, z[h][i][j] * w[h][i][j]);
                            }
                    }
                    if (slots.is(i)) {
                        Channels<T, V>::store(dx + slots.first[i], f[0]);
                        if (slots.has_second(i)) Channels<T, V>::store(dx + slots.second[i], f[1]);
                    }
                }
            }
        };
        run(std::integral_constant<int, 0>());
        run(std::integral_constant<int, 1>());
    }
    if (!a.dwq && !a.dwk) return;
    __shared__ float joined[kWavesOf][SYS_MAX_HEAD_DIM];
    float* out = a.workspace + (size_t)blockIdx.x * 2 * p.dim;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < S; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float v = dw[k][h][i][j];
                    for (int m = 1 << n.parts_log; m < 64; m <<= 1) v += __shfl_xor(v, m);
                    if ((threadIdx.x & 63) >> n.parts_log == 0 && (h ? slots.has_second(i) : slots.is(i)))
                        joined[threadIdx.x >> 6][(h ? slots.second[i] : slots.first[i]) + j] = v;
                }
        __syncthreads();
        for (int c = threadIdx.x; c < p.dim; c += kThreads) {
            float v = joined[0][c];
#pragma unroll
            for (int m = 1; m < kWavesOf; ++m) v += joined[m][c];
            out[k * p.dim + c] = v;
        }
    }
}

// The workgroups' sums of a column, [blocks][2][dim]: 16 columns a workgroup (64 bytes of a row), 64 lanes a column, joined in a fixed order.
constexpr int kJoinColumns = 16, kJoinThreads = 1024;
__global__ __launch_bounds__(kJoinThreads) void head_norm_join_kernel(sys_head_norm_t p, HeadNormArgs a, int blocks)
{
    constexpr int kRows = kJoinThreads / kJoinColumns;
    const int column = blockIdx.x * kJoinColumns + threadIdx.x % kJoinColumns, first = threadIdx.x / kJoinColumns;
    const bool there = column < 2 * p.dim;
    float v = 0.0f;
#pragma unroll 8
    for (int i = first; i < blocks; i += kRows) v += there ? a.workspace[(size_t)i * 2 * p.dim + column] : 0.0f;
    // over the four rows of lanes of a wavefront, then over wavefronts
    v += __shfl_xor(v, 16);
    v += __shfl_xor(v, 32);
    __shared__ float sums[kJoinThreads / 64][kJoinColumns];
    if ((threadIdx.x & 63) < kJoinColumns) sums[threadIdx.x >> 6][threadIdx.x & 63] = v;
    __syncthreads();
    if (threadIdx.x >= kJoinColumns || !there) return;
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < kJoinThreads / 64; ++i) v += sums[i][threadIdx.x];
    void* out = column < p.dim ? a.dwq : a.dwk;
    if (out) store_param(out, column < p.dim ? column : column - p.dim, p.param_dtype, v);
}

// ---------------------------------------------------------------- launches

// Workgroups of the gradients, at most: as many as the registers of an instance leave resident, so that none starts behind the others.  Whole calls on 8192 tokens, one behind the
// other, us with 512, 768, 1024 and 256: 18 heads of 256 in bf16 (V = 8, 199 registers) 60, 72, 67, 77; of 36 heads of 128 62, 76, 70, 80; of 72 heads of 72 (V = 4, 133) 105, 92, 112, 166;
// of 36 heads of 128 in fp32 (V = 4 as well) 97, 99, 111, 111; of 50 heads of 50 (V = 1, 91) 101, 90, 82, 169; of 16 heads of 200 in fp32 (V = 1, S = 4) 93, 107, 96, 133.
constexpr int kGradBlocks = 1024;
template <int V, int S> constexpr int kResidentBlocks = V * S == 1 ? kGradBlocks : V == 4 ? 768 : 512;

template <int V, int S>
NormPlan plan_of(const sys_head_norm_t& p, bool grad)
{
    NormPlan n = {};
    n.turned = p.rotary / 2 / V;
    n.slots = n.turned + ((p.dim - p.rotary + 1) / 2 + V - 1) / V;
    while ((1 << n.parts_log) * S < n.slots) ++n.parts_log;
    n.all_heads = p.q_heads + p.k_heads;
    while (n.parts_log + n.heads_log < 6 && (1 << n.heads_log) < n.all_heads) ++n.heads_log;
    n.tokens = (long long)p.batch * p.length;
    const int side = 1 << (6 - n.parts_log - n.heads_log);
    const long long waves = (n.tokens + side - 1) / side;
    // few tokens: their heads go to several wavefronts
    const int turns = (n.all_heads + (1 << n.heads_log) - 1) >> n.heads_log;
    n.splits = 1;
    if (!grad)
        while (n.splits < turns && waves * n.splits < 2048) ++n.splits;
    const int each = (turns + n.splits - 1) / n.splits;
    n.each = each << n.heads_log;
    n.splits = (turns + each - 1) / each;
    return n;
}

template <typename T, int V, int S>
hipError_t launch_shape(bool grad, const sys_head_norm_t& p, const HeadNormArgs& a, hipStream_t s)
{
    const NormPlan n = plan_of<V, S>(p, grad);
    const int side = 1 << (6 - n.parts_log - n.heads_log);
    const long long waves = (n.tokens + side - 1) / side * n.splits;
    long long blocks = (waves + kWavesOf - 1) / kWavesOf;
    if (!grad) {
        if (blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
        hipLaunchKernelGGL((head_norm_kernel<T, V, S>), dim3((unsigned)blocks), dim3(kThreads), 0, s, p, a, n);
        return hipGetLastError();
    }
    if (blocks > kResidentBlocks<V, S>) blocks = kResidentBlocks<V, S>;
    if (blocks) {
        hipLaunchKernelGGL((head_norm_grad_kernel<T, V, S>), dim3((unsigned)blocks), dim3(kThreads), 0, s, p, a, n, waves);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!a.dwq && !a.dwk) return hipSuccess;
    hipLaunchKernelGGL(head_norm_join_kernel, dim3((unsigned)(2 * p.dim + kJoinColumns - 1) / kJoinColumns), dim3(kJoinThreads), 0, s, p, a, (int)blocks);
    return hipGetLastError();
}

// Pieces of V entries: the turned halves and the halves of the rest are whole numbers of them.
bool pieces_of(const sys_head_norm_t& p, int v) { return p.rotary / 2 % v == 0 && (p.dim - p.rotary) % (2 * v) == 0; }

template <typename T>
hipError_t launch_type(bool grad, const sys_head_norm_t& p, const HeadNormArgs& a, hipStream_t s)
{
    constexpr int V = kLaneChannels<T>;
    if (pieces_of(p, V)) return launch_shape<T, V, 1>(grad, p, a, s);
    if (sizeof(T) == 2 && p.dim <= 512 && pieces_of(p, 4)) return launch_shape<T, 4, 1>(grad, p, a, s);
    if (p.dim <= 128) return launch_shape<T, 1, 1>(grad, p, a, s);
    return launch_shape<T, 1, 4>(grad, p, a, s);
}

hipError_t launch(bool grad, const sys_head_norm_t& p, const HeadNormArgs& a, hipStream_t s)
{
    switch (p.dtype) {
    case SYS_F32: return launch_type<float>(grad, p, a, s);
    case SYS_F16: return launch_type<f16_t>(grad, p, a, s);
    default: return launch_type<bf16_t>(grad, p, a, s);
    }
}

}  // namespace

hipError_t launch_head_norm(const sys_head_norm_t& p, const HeadNormArgs& a, hipStream_t s) { return launch(false, p, a, s); }
hipError_t launch_head_norm_grad(const sys_head_norm_t& p, const HeadNormArgs& a, hipStream_t s) { return launch(true, p, a, s); }

// Sums of the weights' gradients of every workgroup.
size_t head_norm_grad_workspace(const sys_head_norm_t& p)
{
    return p.batch && p.length ? (size_t)kGradBlocks * 2 * p.dim * sizeof(float) : 0;
}

}  // namespace sysconv
