// Group norm with an activation, channels last: y = act((x - mean) rstd w + b), statistics over the rows of a batch entry and the
// channels of a group.  Bound by memory: some ten operations a value beside its bytes.
//
// Two ways.  Where a group's rows fit the registers of a workgroup (or of a part of a wavefront: a token, a small image) they are
// read once, wait there for the group's sums, and are written once (norm_resident_kernel, norm_grad_resident_kernel).  Else a first
// launch sums up chunks of rows channel by channel, one or two small ones combine them, and a last one reads the rows again.
//
// Squares are never summed as they come, so a mean far from zero costs no digits of the variance: what a lane has seen of the group's mean is taken
// off its values, some differences at a time give their own mean and sum of squared distances, and these are put together as n = n1 + n2,
// mean = mean1 + d n2/n, M2 = M2_1 + M2_2 + d^2 n1 n2/n with d = mean2 - mean1, or for many at once as mean = sum n_i mean_i / n,
// M2 = sum M2_i + n_i (mean_i - mean)^2.  Means stay in two parts until they have been subtracted: rounded to 32 bits they would bring their own size
// into d.  No one value is taken off all the others, for it may be far from them, and its size would stay in the mean's last digit.
//
// Measured, bf16: 16 x 4096 x 512 in 32 groups with SiLU 31.8 us, 4.2 TB/s of x and y (a copy of as many bytes: 22; every CU holds one unit,
// so all load, then all store, in pieces of 64 bytes); 8192 rows of 64 x 64 channels 26.6, 5.0 TB/s, their gradients 50, 4.0 TB/s of x, dy
// and dx; gradients of 8 x 4096 x 320 in 32 groups, f16, in chunks 33.0, by the profiler about 15 sums, 7 combining and 14 dx.  Chunks of few wide groups
// are far from their bytes: 1 x 16384 x 2048 in one group 1780 us, nearly all of it one workgroup that adds up [chunk][channel] (4 x 4096 x 320 in 32
// groups: 17.4).
#include <type_traits>

#include "launch.h"
#include "sequence.h"

namespace sysconv {
namespace {

constexpr int kThreads = 256;

struct Moments {
    float n, mean, m2;
};

__device__ __forceinline__ Moments merged(Moments a, Moments b)
{
    const float n = a.n + b.n;
    const float share = n > 0.0f ? b.n * fast_rcp(n) : 0.0f, d = b.mean - a.mean;
    return {n, b.n > 0.0f ? __builtin_fmaf(d, share, a.mean) : a.mean, b.n > 0.0f ? a.m2 + b.m2 + d * d * a.n * share : a.m2};
}

template <int V, int ACTIVATION>
__device__ __forceinline__ void activate(float (&v)[V])
{
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = ACTIVATION == SYS_ACT_SILU ? silu(v[k]) : ACTIVATION == SYS_ACT_RELU && v[k] <= 0.0f ? 0.0f : v[k];   // (a NaN stays)
}

// work(integral_constant) of the activation: one branch for a lane's rows (a branch for each value had taken 2 us of 35).
template <typename F>
__device__ __forceinline__ void by_activation(int activation, F&& work)
{
    if (activation == SYS_ACT_SILU) work(std::integral_constant<int, SYS_ACT_SILU>());
    else if (activation == SYS_ACT_RELU) work(std::integral_constant<int, SYS_ACT_RELU>());
    else work(std::integral_constant<int, SYS_ACT_NONE>());
}

// 1 / sqrt(v) to an ulp or so; the instruction takes no v below the smallest normal number.  (A quotient, a root and a quotient rounded by the book had
// been a fifth of the instructions for rows of 64 x 64 channels.)
__device__ __forceinline__ float inverse_root(float v)
{
    const bool tiny = v < 0x1p-100f;
    return __builtin_amdgcn_rsqf(tiny ? v * 0x1p64f : v) * (tiny ? 0x1p32f : 1.0f);
}

// The groups of V neighbouring channels, one division for all of them; counted from `from` on.
template <int V, typename Index>
__device__ __forceinline__ void groups_of(int channel, int channels_a_group, Index from, Index (&group)[V])
{
    int g = channel / channels_a_group, in_group = channel - g * channels_a_group;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        group[i] = from + g;
        const bool next = ++in_group == channels_a_group;
        g += next;
        in_group = next ? 0 : in_group;
    }
}

// w and b of V channels, 1 and 0 without them.
template <typename T, int V>
__device__ __forceinline__ void load_affine(const sys_group_norm_t& p, const NormArgs& a, int channel, float (&w)[V], float (&b)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] = 1.0f, b[i] = 0.0f;
    if (a.w) load_params<T, V>(a.w, (size_t)channel, p.param_dtype, w);
    if (a.b) load_params<T, V>(a.b, (size_t)channel, p.param_dtype, b);
}

// ================================================================ rows that stay in registers

// A unit -- a batch entry and `tile` neighbouring groups -- has 2^log_unit lanes, 1 to 1024: a part of a wavefront or a whole workgroup.
// From the lowest bits of the lane up: lane of the group (V channels each, rounded up to a power of two), group of the tile, row.
// A lane has its channels in `items` rows.
struct ResidentShape {
    int log_group, log_tile, log_unit, threads;     // lanes a group; groups a tile; lanes a unit; lanes a workgroup
    int items, tiles;                               // tiles: of a batch entry
    int columns_a_group;                            // lanes of a group that hold channels
    int entries, units;                             // batch entries a unit has at a time; units of the launch
    int slices, rounds;                             // gradients: units of a tile, and how often each takes its entries
};

struct ResidentLane {
    int unit, tile_group, group, row, tall, channel;
    bool there;
    __device__ __forceinline__ ResidentLane(const sys_group_norm_t& p, const ResidentShape& s, int units, unsigned place)
    {
        const int in_unit = threadIdx.x & ((1 << s.log_unit) - 1), in_group = in_unit & ((1 << s.log_group) - 1);
        const int index = place * (blockDim.x >> s.log_unit) + (threadIdx.x >> s.log_unit);
        unit = index < units ? index : units - 1;
        tile_group = (in_unit >> s.log_group) & ((1 << s.log_tile) - 1);
        row = in_unit >> (s.log_group + s.log_tile);
        tall = 1 << (s.log_unit - s.log_group - s.log_tile);
        const int g = unit % s.tiles * (1 << s.log_tile) + tile_group;
        there = index < units && in_group < s.columns_a_group && g < p.groups;
        group = g < p.groups ? g : p.groups - 1;
        const int channels = p.channels / p.groups, v = channels / s.columns_a_group;
        channel = group * channels + (in_group < s.columns_a_group ? in_group : 0) * v;
    }
};

// Rows of a lane, `tall` apart; past the last one that row again, which is not used.  No load depends on a branch, so what is made of the
// first rows need not wait for the last ones.
template <typename T, int V, int ITEMS>
struct ResidentRows {
    typename Channels<T, V>::Raw raw[ITEMS];
    __device__ __forceinline__ void load(const T* from, long long row_stride, int rows, int row, int tall)
    {
        int r = row < rows ? row : rows - 1;
        from += r * row_stride;
        const long long step = tall * row_stride;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            raw[i] = Channels<T, V>::raw(from);
            r += tall;
            from += r < rows ? step : 0;
        }
    }
};

// The same rows, to be worked on once more: without this the compiler keeps what it made of them the first time, in registers that are not there.
template <typename Raw>
__device__ __forceinline__ void forget(Raw& raw)
{
    if constexpr (sizeof(Raw) == 2) {
        unsigned v = __builtin_bit_cast(unsigned short, raw);
        asm volatile("" : "+v"(v));
        raw = __builtin_bit_cast(Raw, (unsigned short)v);
    } else if constexpr (sizeof(Raw) == 4) {
        unsigned v = __builtin_bit_cast(unsigned, raw);
        asm volatile("" : "+v"(v));
        raw = __builtin_bit_cast(Raw, v);
    } else {
        typedef unsigned Words __attribute__((ext_vector_type(sizeof(Raw) / 4)));
        Words v = __builtin_bit_cast(Words, raw);
        asm volatile("" : "+v"(v));
        raw = __builtin_bit_cast(Raw, v);
    }
}

// v + v of lane ^ (1 << BIT).
template <int BIT>
__device__ __forceinline__ float add_lane(float v)
{
    if constexpr (BIT == 0) return v + dpp<0xB1>(v);                    // quad_perm 1 0 3 2
    else if constexpr (BIT == 1) return v + dpp<0x4E>(v);               // quad_perm 2 3 0 1
    else if constexpr (BIT == 2) return v + dpp<0x1B>(dpp<0x141>(v));   // the half row mirrored, and every quad of it
    else if constexpr (BIT == 3) return v + dpp<0x128>(v);              // the row turned by 8
    else {
        const unsigned u = __builtin_bit_cast(unsigned, v);
        unsigned low, high;
        if constexpr (BIT == 4) {
            const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
            low = r[0], high = r[1];
        } else {
            const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
            low = r[0], high = r[1];
        }
        return __builtin_bit_cast(float, low) + __builtin_bit_cast(float, high);
    }
}

// Sums over the lanes of a wavefront that share a unit and a group; every lane gets them.
template <int N>
__device__ __forceinline__ void sum_lanes(const ResidentShape& s, float (&v)[N])
{
    const int wide = s.log_group + s.log_tile;
    auto add = [&](auto bit) {
        constexpr int kBit = decltype(bit)::value;
        if (kBit >= s.log_unit || (kBit >= s.log_group && kBit < wide)) return;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = add_lane<kBit>(v[i]);
    };
    add(std::integral_constant<int, 0>()), add(std::integral_constant<int, 1>()), add(std::integral_constant<int, 2>());
    add(std::integral_constant<int, 3>()), add(std::integral_constant<int, 4>()), add(std::integral_constant<int, 5>());
}

constexpr int kMostTile = 32;                       // groups a tile

// Units of more than a wavefront: what the wavefronts have goes through LDS, [entry][wavefront][group of the tile].  Every wavefront of the
// workgroup has to come here.
template <int ENTRIES, int MOST, typename M>
__device__ __forceinline__ void put_wavefront(const ResidentShape& s, int tile_group, const M (&m)[ENTRIES], M (&shared)[ENTRIES][MOST])
{
    const unsigned lane = threadIdx.x & 63;
    __syncthreads();                                // (what was here before has been read)
    if (lane < (1u << (s.log_group + s.log_tile)) && (lane & ((1u << s.log_group) - 1)) == 0) {
#pragma unroll
        for (int e = 0; e < ENTRIES; ++e) shared[e][((threadIdx.x >> 6) << s.log_tile) + tile_group] = m[e];
    }
    __syncthreads();
}

// work(e, what a wavefront put there) for the wavefronts of the unit, in their order.
template <int ENTRIES, int MOST, typename M, typename F>
__device__ __forceinline__ void each_wavefront(const ResidentShape& s, int tile_group, const M (&shared)[ENTRIES][MOST], F&& work)
{
    const int waves = 1 << (s.log_unit - 6), first = (threadIdx.x >> s.log_unit) * waves;
    for (int k = 0; k < waves; ++k) {
#pragma unroll
        for (int e = 0; e < ENTRIES; ++e) work(e, shared[e][((first + k) << s.log_tile) + tile_group]);
    }
}

// n values, their mean (origin + mean: the mean of some of them, and where the mean of all lies from there), and the sum of squared distances from it.
struct PartMoments {
    float n, origin, mean, m2;
};

// Moments of a lane's rows: all of `items`, or all but the last one.
template <typename T, int V, int ITEMS>
__device__ __forceinline__ PartMoments lane_moments(const ResidentRows<T, V, ITEMS>& rows, bool there, bool whole, int items)
{
    PartMoments m = {0.0f, 0.0f, 0.0f, 0.0f};
    float head[V];
    Channels<T, V>::values(rows.raw[0], head);
#pragma unroll
    for (int k = 0; k < V; ++k) m.origin = __builtin_fmaf(head[k], 1.0f / V, m.origin);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        if (ITEMS > 1 && i >= items) continue;
        float v[V], sum = 0.0f, square = 0.0f;
        Channels<T, V>::values(rows.raw[i], v);
#pragma unroll
        for (int k = 0; k < V; ++k) sum += v[k] - m.origin;
        const float mean = sum * (1.0f / V);
#pragma unroll
        for (int k = 0; k < V; ++k) square = __builtin_fmaf((v[k] - m.origin) - mean, (v[k] - m.origin) - mean, square);
        if (i == 0) {                               // (a lane without any row is put right below)
            m.mean = mean;
            m.m2 = square;
            continue;
        }
        const float on = i + 1 < items || whole ? 1.0f : 0.0f, d = mean - m.mean;
        m.mean = __builtin_fmaf(d, on * (1.0f / (i + 1)), m.mean);
        m.m2 = __builtin_fmaf(on, __builtin_fmaf(d * d, (float)V * i / (i + 1), square), m.m2);
    }
    m.n = there ? (float)(V * (items - !whole)) : 0.0f;
    if (m.n == 0.0f) m = {0.0f, 0.0f, 0.0f, 0.0f};
    return m;
}

// A unit has ENTRIES batch entries in a row; with one row a lane (ITEMS 1: tokens) several, whose loads and sums run side by side.
template <typename T, int V, int ITEMS, int ENTRIES>
__global__ __launch_bounds__(1024) void norm_resident_kernel(sys_group_norm_t p, NormArgs a, ResidentShape s)
{
    __shared__ PartMoments shared[ENTRIES][ITEMS == 1 ? 16 : 16 * kMostTile];         // (one row a lane is a row in all, whose units of several wavefronts are one group)
    const ResidentLane at(p, s, s.units, xcd_place(blockIdx.x, gridDim.x));
    const int b0 = at.unit / s.tiles * ENTRIES;
    ResidentRows<T, V, ITEMS> rows[ENTRIES];
#pragma unroll
    for (int e = 0; e < ENTRIES; ++e) rows[e].load((const T*)a.x + (b0 + e < p.batch ? b0 + e : p.batch - 1) * p.x_batch + at.channel, p.x_row, (int)p.rows, at.row, at.tall);
    float w[V], shift[V];
    load_affine<T, V>(p, a, at.channel, w, shift);
    const bool whole = at.row + (s.items - 1) * at.tall < (int)p.rows;
    PartMoments m[ENTRIES];
#pragma unroll
    for (int e = 0; e < ENTRIES; ++e) m[e] = lane_moments<T, V, ITEMS>(rows[e], at.there, whole, s.items);
    // the mean of several means, then the sum of squared distances from it and where the mean lies from there (in 32 bits it was rounded on the way),
    // over the lanes; and the same of the wavefronts
    float n[1] = {m[0].n}, mean_of[ENTRIES], sums[2 * ENTRIES];
    sum_lanes(s, n);
    const float share = n[0] > 0.0f ? 1.0f / n[0] : 0.0f;
#pragma unroll
    for (int e = 0; e < ENTRIES; ++e) mean_of[e] = m[e].n * share * (m[e].origin + m[e].mean);
    sum_lanes(s, mean_of);
#pragma unroll
    for (int e = 0; e < ENTRIES; ++e) {
        const float d = (m[e].origin - mean_of[e]) + m[e].mean;
        sums[2 * e] = m[e].n * d;
        sums[2 * e + 1] = __builtin_fmaf(m[e].n * d, d, m[e].m2);
    }
    sum_lanes(s, sums);
#pragma unroll
    for (int e = 0; e < ENTRIES; ++e) m[e] = {n[0], mean_of[e], sums[2 * e] * share, __builtin_fmaf(sums[2 * e] * share, -sums[2 * e], sums[2 * e + 1])};
    const float all = (float)p.rows * (float)(p.channels / p.groups);
    if (s.log_unit > 6) {
        put_wavefront(s, at.tile_group, m, shared);
        // (distances from the first wavefront's mean: their squares are at most 16, the wavefronts, times the sum that is left of them)
        const int first_wave = (threadIdx.x >> s.log_unit) << (s.log_unit - 6);
#pragma unroll
        for (int e = 0; e < ENTRIES; ++e) mean_of[e] = shared[e][(first_wave << s.log_tile) + at.tile_group].origin, sums[2 * e] = sums[2 * e + 1] = 0.0f;
        each_wavefront(s, at.tile_group, shared, [&](int e, const PartMoments& o) {
            const float d = (o.origin - mean_of[e]) + o.mean;
            sums[2 * e] = __builtin_fmaf(o.n, d, sums[2 * e]);
            sums[2 * e + 1] += __builtin_fmaf(o.n * d, d, o.m2);
        });
#pragma unroll
        for (int e = 0; e < ENTRIES; ++e) m[e] = {all, mean_of[e], sums[2 * e] * (1.0f / all), __builtin_fmaf(sums[2 * e] * (1.0f / all), -sums[2 * e], sums[2 * e + 1])};
    }
#pragma unroll
    for (int e = 0; e < ENTRIES; ++e) {
        if (!at.there || b0 + e >= p.batch) continue;
        const float m2 = m[e].m2 < 0.0f ? 0.0f : m[e].m2;                   // (of equal values it may be, by roundings; a NaN stays)
        const float mean = m[e].origin + m[e].mean, rstd = inverse_root(__builtin_fmaf(m2, 1.0f / all, p.eps));
        if (at.row == 0 && at.channel == at.group * (p.channels / p.groups)) {
            const size_t group = (size_t)(b0 + e) * p.groups + at.group;
            if (a.mean) a.mean[group] = mean;
            if (a.rstd) a.rstd[group] = rstd;
        }
        T* y = (T*)a.y + (b0 + e) * p.y_batch + at.row * p.y_row + at.channel;
        const long long step = at.tall * p.y_row;
        float scale[V];
#pragma unroll
        for (int k = 0; k < V; ++k) scale[k] = w[k] * rstd;
        by_activation(p.activation, [&](auto activation) {
            int items = s.items;
            T* to = y;
            // (else the rows' addresses are made all at once, and the comparisons kept from the loop above, in registers that are not there)
            if (ITEMS > 1) asm volatile("" : "+s"(items), "+v"(to));
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                if (ITEMS > 1 && i >= items) continue;
                if (i + 1 == items && !whole) continue;
                float v[V];
                if (ITEMS > 1) forget(rows[e].raw[i]);
                Channels<T, V>::values(rows[e].raw[i], v);
#pragma unroll
                for (int k = 0; k < V; ++k) v[k] = __builtin_fmaf(v[k] - mean, scale[k], shift[k]);
                activate<V, decltype(activation)::value>(v);
                Channels<T, V>::store_nt(to, v);
                to += step;
                if (ITEMS > 1) asm volatile("" : "+v"(to));
            }
        });
    }
}

// Gradients: with hat = (x - mean) rstd and f = dy act'(hat w + b): dw = sum f hat, db = sum f over batch and rows, and
// dx = rstd (f w - m1 - hat m2), m1 = E[f w], m2 = E[f w hat] over the group.

struct Pair {
    float a, b;
};

template <int ACTIVATION>
__device__ __forceinline__ float activation_grad(float v)
{
    return ACTIVATION == SYS_ACT_SILU ? silu_grad(v) : ACTIVATION == SYS_ACT_RELU ? (v > 0.0f ? 1.0f : 0.0f) : 1.0f;
}

// f and hat of V channels of a row.
template <int V, int ACTIVATION>
__device__ __forceinline__ void row_grad(const float (&x)[V], const float (&dy)[V], float mean, float rstd, const float (&w)[V], const float (&shift)[V], float (&f)[V], float (&hat)[V])
{
#pragma unroll
    for (int k = 0; k < V; ++k) {
        hat[k] = (x[k] - mean) * rstd;
        f[k] = dy[k] * activation_grad<ACTIVATION>(__builtin_fmaf(hat[k], w[k], shift[k]));
    }
}

// A unit goes through the batch entries of its slice, ENTRIES at a time, and adds up dw and db of its channels: [slice][f | f hat][channel] in the
// workspace.
template <typename T, int V, int ITEMS, int ENTRIES>
__global__ __launch_bounds__(512) void norm_grad_resident_kernel(sys_group_norm_t p, NormArgs a, ResidentShape s)
{
    __shared__ Pair shared[ENTRIES][8 * kMostTile];
    __shared__ float sums[512];
    const ResidentLane at(p, s, s.units, xcd_place(blockIdx.x, gridDim.x));
    const int slice = at.unit / s.tiles;
    const T *x = (const T*)a.x + at.channel, *dy = (const T*)a.dy + at.channel;
    float w[V], shift[V], f_sum[V], hat_sum[V];
    load_affine<T, V>(p, a, at.channel, w, shift);
#pragma unroll
    for (int k = 0; k < V; ++k) f_sum[k] = hat_sum[k] = 0.0f;
    const float share = 1.0f / ((float)p.rows * (float)(p.channels / p.groups));
    const bool whole = at.row + (s.items - 1) * at.tall < (int)p.rows;
    // as many rounds for every unit, so that all wavefronts of a workgroup meet at its barriers
    for (int round = 0; round < s.rounds; ++round) {
        const int b0 = (round * s.slices + slice) * ENTRIES;
        ResidentRows<T, V, ITEMS> rows_x[ENTRIES], rows_dy[ENTRIES];
        float mean[ENTRIES], rstd[ENTRIES];
#pragma unroll
        for (int e = 0; e < ENTRIES; ++e) {
            const int b = b0 + e < p.batch ? b0 + e : p.batch - 1;
            rows_x[e].load(x + b * p.x_batch, p.x_row, (int)p.rows, at.row, at.tall);
            rows_dy[e].load(dy + b * p.y_batch, p.y_row, (int)p.rows, at.row, at.tall);
            mean[e] = a.mean_in[(size_t)b * p.groups + at.group];
            rstd[e] = a.rstd_in[(size_t)b * p.groups + at.group];
        }
        float m[2 * ENTRIES];                       // sums of f w and of f w hat
#pragma unroll
        for (int e = 0; e < 2 * ENTRIES; ++e) m[e] = 0.0f;
        by_activation(p.activation, [&](auto activation) {
#pragma unroll
            for (int e = 0; e < ENTRIES; ++e) {
                const bool there = at.there && b0 + e < p.batch;
#pragma unroll
                for (int i = 0; i < ITEMS; ++i) {
                    if (ITEMS > 1 && i >= s.items) continue;
                    float v[V], g[V], f[V], hat[V];
                    Channels<T, V>::values(rows_x[e].raw[i], v);
                    Channels<T, V>::values(rows_dy[e].raw[i], g);
                    row_grad<V, decltype(activation)::value>(v, g, mean[e], rstd[e], w, shift, f, hat);
                    if (there && (i + 1 < s.items || whole)) {
#pragma unroll
                        for (int k = 0; k < V; ++k) {
                            f_sum[k] += f[k];
                            hat_sum[k] = __builtin_fmaf(f[k], hat[k], hat_sum[k]);
                            m[2 * e] = __builtin_fmaf(f[k], w[k], m[2 * e]);
                            m[2 * e + 1] = __builtin_fmaf(f[k] * w[k], hat[k], m[2 * e + 1]);
                        }
                    }
                }
            }
        });
        sum_lanes(s, m);
        if (s.log_unit > 6) {
            Pair pair[ENTRIES];
#pragma unroll
            for (int e = 0; e < ENTRIES; ++e) pair[e] = {m[2 * e], m[2 * e + 1]}, m[2 * e] = m[2 * e + 1] = 0.0f;
            put_wavefront(s, at.tile_group, pair, shared);
            each_wavefront(s, at.tile_group, shared, [&](int e, const Pair& o) { m[2 * e] += o.a, m[2 * e + 1] += o.b; });
        }
#pragma unroll
        for (int e = 0; e < ENTRIES; ++e) {
            if (!at.there || b0 + e >= p.batch) continue;
            const float m1 = m[2 * e] * share, m2 = m[2 * e + 1] * share;
            T* dx = (T*)a.dx + ((size_t)(b0 + e) * p.rows + at.row) * p.channels + at.channel;
            const long long step = (long long)at.tall * p.channels;
            by_activation(p.activation, [&](auto activation) {
#pragma unroll
                for (int i = 0; i < ITEMS; ++i) {
                    if (ITEMS > 1 && i >= s.items) continue;
                    if (i + 1 == s.items && !whole) continue;
                    float v[V], g[V], f[V], hat[V];
                    if (ITEMS * ENTRIES > 1) {
                        forget(rows_x[e].raw[i]);
                        forget(rows_dy[e].raw[i]);
                    }
                    Channels<T, V>::values(rows_x[e].raw[i], v);
                    Channels<T, V>::values(rows_dy[e].raw[i], g);
                    row_grad<V, decltype(activation)::value>(v, g, mean[e], rstd[e], w, shift, f, hat);
#pragma unroll
                    for (int k = 0; k < V; ++k) v[k] = rstd[e] * (__builtin_fmaf(f[k], w[k], -m1) - hat[k] * m2);
                    Channels<T, V>::store_nt(dx + i * step, v);
                }
            });
        }
    }
    if (!a.dw && !a.db) return;
    // over the rows of the unit: the upper bits of the lane
    const int wide = s.log_group + s.log_tile;
    float* to = a.workspace + (size_t)slice * 2 * p.channels + at.channel;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        for (int which = 0; which < 2; ++which) {
            float v = which ? hat_sum[k] : f_sum[k];
            for (int bit = wide; bit < s.log_unit && bit < 6; ++bit) v += __shfl_xor(v, 1 << bit);
            if (s.log_unit > 6 && wide < s.log_unit) {
                __syncthreads();
                sums[threadIdx.x] = v;
                __syncthreads();
                const int step = wide < 6 ? 64 : 1 << wide, first = threadIdx.x & ~((1 << s.log_unit) - 1);
                if (at.row == 0) {
                    for (int t = step; t < (1 << s.log_unit); t += step) v += sums[first + (threadIdx.x & ((1 << wide) - 1)) + t];
                }
            }
            if (at.there && at.row == 0) to[(size_t)which * p.channels + k] = v;
        }
    }
}

// ================================================================ rows that are read twice

struct NormShape {
    int columns;                   // lanes a row, of V channels (the last one begins earlier where channels are no multiple of V)
    int chunks;                    // of the rows, a workgroup each
    long long chunk_rows;
};

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

// Rows of a lane that are on their way together.
constexpr int kNormRows = 8;

// Mean and sum of squared distances of every channel in a chunk of rows: [batch][chunk][mean | m2][channel].
template <typename T, int V>
__global__ __launch_bounds__(kThreads) void norm_moments_kernel(sys_group_norm_t p, NormArgs a, NormShape shape)
{
    const int b = blockIdx.x / shape.chunks, chunk = blockIdx.x - b * shape.chunks;
    const Lanes at(shape.columns);
    const long long begin = chunk * shape.chunk_rows, end = begin + shape.chunk_rows < p.rows ? begin + shape.chunk_rows : p.rows;
    const T* x = (const T*)a.x + b * p.x_batch;
    float* to = a.workspace + ((size_t)b * shape.chunks + chunk) * 2 * p.channels;
    __shared__ float shared_n[kThreads], shared_mean[V][kThreads], shared_m2[V][kThreads];
    for (int c0 = 0; c0 < shape.columns; c0 += at.wide) {
        const bool there = at.there && c0 + at.column < shape.columns;
        const int column = c0 + at.column < shape.columns ? c0 + at.column : shape.columns - 1;
        const int channel = column * V + V <= p.channels ? column * V : p.channels - V;
        float n = 0.0f, mean[V], rest[V], m2[V];    // the mean: mean + rest
#pragma unroll
        for (int i = 0; i < V; ++i) mean[i] = rest[i] = m2[i] = 0.0f;
        if (there) {
            const T* from = x + channel;
            for (long long r = begin + at.row; r < end; r += (long long)at.tall * kNormRows) {
                typename Channels<T, V>::Raw raw[kNormRows];
#pragma unroll
                for (int k = 0; k < kNormRows; ++k) {
                    const long long row = r + (long long)k * at.tall;
                    raw[k] = Channels<T, V>::raw(from + (row < end ? row : r) * p.x_row);
                }
                if (n == 0.0f) Channels<T, V>::values(raw[0], mean);      // (of no rows: taken off the first ones, it moves to their mean with them)
                float count = 0.0f, sum[V], square[V];
#pragma unroll
                for (int i = 0; i < V; ++i) sum[i] = square[i] = 0.0f;
#pragma unroll
                for (int k = 0; k < kNormRows; ++k) {
                    const float on = r + (long long)k * at.tall < end ? 1.0f : 0.0f;
                    float v[V];
                    Channels<T, V>::values(raw[k], v);
                    count += on;
#pragma unroll
                    for (int i = 0; i < V; ++i) sum[i] = __builtin_fmaf(on, v[i] - mean[i], sum[i]);       // (the row that stands in for one that is not there is in the sum)
                }
                const float inverse = fast_rcp(count);
#pragma unroll
                for (int i = 0; i < V; ++i) sum[i] *= inverse;
#pragma unroll
                for (int k = 0; k < kNormRows; ++k) {
                    const float on = r + (long long)k * at.tall < end ? 1.0f : 0.0f;
                    float v[V];
                    Channels<T, V>::values(raw[k], v);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float d = (v[i] - mean[i]) - sum[i];
                        square[i] = __builtin_fmaf(on * d, d, square[i]);
                    }
                }
                const float all = n + count, share = count * fast_rcp(all);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float d = sum[i] - rest[i];
                    m2[i] += square[i] + d * d * n * share;
                    const float step = __builtin_fmaf(d, share, rest[i]), now = mean[i] + step;
                    rest[i] = (mean[i] - now) + step;
                    mean[i] = now;
                }
                n = all;
            }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) mean[i] += rest[i];
        // the rows of the workgroup, by halves
        for (int tall = at.tall; tall > 1;) {
            const int half = (tall + 1) / 2;
            __syncthreads();
            if (at.row >= half && at.row < tall) {
                shared_n[threadIdx.x] = n;
#pragma unroll
                for (int i = 0; i < V; ++i) shared_mean[i][threadIdx.x] = mean[i], shared_m2[i][threadIdx.x] = m2[i];
            }
            __syncthreads();
            if (at.row + half < tall) {
                const int other = threadIdx.x + half * at.wide;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const Moments m = merged(Moments{n, mean[i], m2[i]}, Moments{shared_n[other], shared_mean[i][other], shared_m2[i][other]});
                    mean[i] = m.mean;
                    m2[i] = m.m2;
                }
                n += shared_n[other];
            }
            tall = half;
        }
        if (there && at.row == 0) {
            Channels<float, V>::store(to + channel, mean);
            Channels<float, V>::store(to + p.channels + channel, m2);
        }
    }
}

// Sum over the lanes of a workgroup; every lane gets it.
__device__ __forceinline__ double workgroup_sum(double v, double (&shared)[kThreads / 64])
{
    for (int k = 1; k < 64; k <<= 1) v += __shfl_xor(v, k);
    __syncthreads();                                // (what was here before has been read)
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
    __syncthreads();
    v = shared[0];
    for (int k = 1; k < kThreads / 64; ++k) v += shared[k];
    return v;
}

// mean and rstd of every group, a workgroup each: [batch][group] pairs behind the chunks' sums, and the caller's arrays.  The entries are thousands to
// a lane for few wide groups, so their sums are in 64 bits: in 32 they had cost rstd 22 units of 2^-24 (1 x 16384 x 2048 in one group).  Taking
// one entry's mean off the others leaves the squares 2^-53 of their own size, which is at most the number of values times that of the variance.
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_statistics_kernel(sys_group_norm_t p, NormArgs a, NormShape shape)
{
    constexpr int kEntries = 8;                     // of a lane on their way together
    const int b = blockIdx.x / p.groups, group = blockIdx.x - b * p.groups;
    const int channels = p.channels / p.groups;
    const float* from = a.workspace + (size_t)b * shape.chunks * 2 * p.channels + (size_t)group * channels;
    const double all = (double)p.rows * channels, chunk_rows = (double)shape.chunk_rows, last_rows = (double)(p.rows - (shape.chunks - 1) * shape.chunk_rows);
    const double origin = *from;
    // a group's entries in [chunk][channel], dealt out to the lanes: 256 channels side by side, or those of several chunks
    const int wide = channels < kThreads ? channels : kThreads, tall = kThreads / wide, row = (int)threadIdx.x / wide, first = (int)threadIdx.x - row * wide;
    double sum = 0.0, squares = 0.0;
    for (int chunk = row < tall ? row : shape.chunks, c = first; chunk < shape.chunks;) {
        float mean[kEntries], m2[kEntries];
        double rows[kEntries];
#pragma unroll
        for (int k = 0; k < kEntries; ++k) {
            const bool there = chunk < shape.chunks;
            const float* entry = there ? from + (size_t)chunk * 2 * p.channels + c : from;
            mean[k] = entry[0];
            m2[k] = entry[p.channels];
            rows[k] = !there ? 0.0 : chunk + 1 < shape.chunks ? chunk_rows : last_rows;
            c += wide;
            if (c >= channels) c = first, chunk += tall;
        }
#pragma unroll
        for (int k = 0; k < kEntries; ++k) {
            const double d = mean[k] - origin;
            sum += rows[k] * d;
            squares += rows[k] > 0.0 ? rows[k] * d * d + m2[k] : 0.0;
        }
    }
    __shared__ double shared[kThreads / 64];
    sum = workgroup_sum(sum, shared);
    squares = workgroup_sum(squares, shared);
    if (threadIdx.x) return;
    const double m2 = squares - sum * (sum / all);
    const float rstd = inverse_root((float)((m2 < 0.0 ? 0.0 : m2 / all) + p.eps));       // (of equal values it may be, by roundings; a NaN stays)
    const float mean = (float)(origin + sum / all);
    float* to = a.workspace + (size_t)p.batch * shape.chunks * 2 * p.channels + 2 * (size_t)blockIdx.x;
    to[0] = mean;
    to[1] = rstd;
    if (a.mean) a.mean[blockIdx.x] = mean;
    if (a.rstd) a.rstd[blockIdx.x] = rstd;
}

template <typename T, int V>
__global__ __launch_bounds__(kThreads) void norm_apply_kernel(sys_group_norm_t p, NormArgs a, NormShape shape)
{
    const int b = blockIdx.x / shape.chunks, chunk = blockIdx.x - b * shape.chunks;
    const Lanes at(shape.columns);
    if (!at.there) return;
    const int channels = p.channels / p.groups;
    const long long begin = chunk * shape.chunk_rows, end = begin + shape.chunk_rows < p.rows ? begin + shape.chunk_rows : p.rows;
    const float* statistics = a.workspace + (size_t)p.batch * shape.chunks * 2 * p.channels + 2 * (size_t)b * p.groups;
    for (int column = at.column; column < shape.columns; column += at.wide) {
        const int channel = column * V + V <= p.channels ? column * V : p.channels - V;
        const T* x = (const T*)a.x + b * p.x_batch + channel;
        T* y = (T*)a.y + b * p.y_batch + channel;
        float mean[V], scale[V], shift[V];
        load_affine<T, V>(p, a, channel, scale, shift);
        int group[V];
        groups_of<V>(channel, channels, 0, group);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            mean[i] = statistics[2 * group[i]];
            scale[i] *= statistics[2 * group[i] + 1];
        }
        by_activation(p.activation, [&](auto activation) {
            for (long long r = begin + at.row; r < end; r += (long long)at.tall * kNormRows) {
                typename Channels<T, V>::Raw raw[kNormRows];
#pragma unroll
                for (int k = 0; k < kNormRows; ++k) {
                    const long long row = r + (long long)k * at.tall;
                    raw[k] = Channels<T, V>::raw(x + (row < end ? row : r) * p.x_row);
                }
#pragma unroll
                for (int k = 0; k < kNormRows; ++k) {
                    const long long row = r + (long long)k * at.tall;
                    if (row >= end) continue;
                    float v[V];
                    Channels<T, V>::values(raw[k], v);
#pragma unroll
                    for (int i = 0; i < V; ++i) v[i] = __builtin_fmaf(v[i] - mean[i], scale[i], shift[i]);
                    activate<V, decltype(activation)::value>(v);
                    Channels<T, V>::store_nt(y + row * p.y_row, v);
                }
            }
        });
    }
}

// m1 and m2 are sums over a group's channels of w times the batch entry's sums of f and f hat, which dw and db are made of as well.
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

// rows of x and of dy on their way together (8 x 4096 x 320, f16, kernels for sums + dx: 14.9 + 13.7 us; with the first loads before the constants
// of the channels, 2 / 4 / 6 / 8 rows: 15.1 + 13.9 / 20.4 + 16.8 / 20.5 + 18.9 / 26 + 21, as their registers leave two wavefronts a SIMD or one)
constexpr int kGradRows = 4;

// Those rows; past the end the first one again.
template <typename T, int V>
struct GradRows {
    typename Channels<T, V>::Raw x[kGradRows], dy[kGradRows];
    __device__ __forceinline__ void load(const sys_group_norm_t& p, const T* from_x, const T* from_dy, long long r, int tall, long long end)
    {
#pragma unroll
        for (int k = 0; k < kGradRows; ++k) {
            const long long row = r + (long long)k * tall < end ? r + (long long)k * tall : r;
            x[k] = Channels<T, V>::raw(from_x + row * p.x_row);
            dy[k] = Channels<T, V>::raw(from_dy + row * p.y_row);
        }
    }
};

// Constants of a lane's channels in the gradients: hat = (x - mean) rstd is not formed, the activation's argument is (x - mean) scale + shift with
// scale = rstd w.
template <typename T, int V>
struct GradLane {
    float mean[V], scale[V], shift[V];
    __device__ __forceinline__ GradLane(const sys_group_norm_t& p, const NormArgs& a, const size_t (&group)[V], int channel)
    {
        load_affine<T, V>(p, a, channel, scale, shift);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            mean[i] = a.mean_in[group[i]];
            scale[i] *= a.rstd_in[group[i]];
        }
    }
    // f and x - mean of a row
    template <int ACTIVATION, typename Raw>
    __device__ __forceinline__ void row(Raw x, Raw dy, float (&f)[V], float (&away)[V]) const
    {
        forget(x), forget(dy);
        Channels<T, V>::values(x, away);
        Channels<T, V>::values(dy, f);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            away[i] -= mean[i];
            f[i] *= activation_grad<ACTIVATION>(__builtin_fmaf(away[i], scale[i], shift[i]));
        }
    }
};

template <typename T, int V>
__global__ __launch_bounds__(kThreads) void norm_grad_sums_kernel(sys_group_norm_t p, NormArgs a, NormShape shape)
{
    const int b = blockIdx.x / shape.chunks, chunk = blockIdx.x - b * shape.chunks;
    const Lanes at(shape.columns);
    const long long begin = chunk * shape.chunk_rows, end = begin + shape.chunk_rows < p.rows ? begin + shape.chunk_rows : p.rows;
    float* to = a.workspace + ((size_t)b * shape.chunks + chunk) * 2 * p.channels;
    __shared__ float shared[V][kThreads];
    for (int c0 = 0; c0 < shape.columns; c0 += at.wide) {
        const bool there = at.there && c0 + at.column < shape.columns;
        const int column = c0 + at.column < shape.columns ? c0 + at.column : shape.columns - 1;
        const int channel = column * V + V <= p.channels ? column * V : p.channels - V;
        float f_sum[V], hat_sum[V];
#pragma unroll
        for (int i = 0; i < V; ++i) f_sum[i] = hat_sum[i] = 0.0f;
        if (there) {
            size_t group[V];
            groups_of<V>(channel, p.channels / p.groups, (size_t)b * p.groups, group);
            const T* x = (const T*)a.x + b * p.x_batch + channel;
            const T* dy = (const T*)a.dy + b * p.y_batch + channel;
            GradRows<T, V> rows;
            const GradLane<T, V> lane(p, a, group, channel);
            by_activation(p.activation, [&](auto activation) {
                for (long long r = begin + at.row; r < end; r += (long long)at.tall * kGradRows) {
                    rows.load(p, x, dy, r, at.tall, end);
#pragma unroll
                    for (int k = 0; k < kGradRows; ++k) {
                        if (r + (long long)k * at.tall >= end) continue;
                        float f[V], away[V];
                        lane.template row<decltype(activation)::value>(rows.x[k], rows.dy[k], f, away);
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            f_sum[i] += f[i];
                            hat_sum[i] = __builtin_fmaf(f[i], away[i], hat_sum[i]);
                        }
                    }
                }
            });
#pragma unroll
            for (int i = 0; i < V; ++i) hat_sum[i] *= a.rstd_in[group[i]];
        }
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < V; ++i) shared[i][threadIdx.x] = which ? hat_sum[i] : f_sum[i];
            // the rows of the workgroup, by halves
            for (int tall = at.tall; tall > 1;) {
                const int half = (tall + 1) / 2;
                __syncthreads();
                if (at.row + half < tall) {
#pragma unroll
                    for (int i = 0; i < V; ++i) shared[i][threadIdx.x] += shared[i][threadIdx.x + half * at.wide];
                }
                tall = half;
            }
            if (at.row == 0 && there) {
                float v[V];
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] = shared[i][threadIdx.x];
                Channels<float, V>::store(to + (size_t)which * p.channels + channel, v);
            }
        }
    }
}

// Sums over `parts` rows of [part][f | f hat][channel] of 16 columns, 16 shares of the parts a workgroup, in one order; in the first 16 lanes.
__device__ __forceinline__ float sum_parts(const float* from, int parts, int columns, int column)
{
    const int share = threadIdx.x >> 4;
    float s = 0.0f;
    if (column < columns)
        for (int k = share; k < parts; k += 16) s += from[(size_t)k * columns + column];
    __shared__ float shared[16][16];
    shared[share][threadIdx.x & 15] = s;
    __syncthreads();
    if (!share)
        for (int k = 1; k < 16; ++k) s += shared[k][threadIdx.x];
    return s;
}

__device__ __forceinline__ void store_affine(const sys_group_norm_t& p, const NormArgs& a, int column, float s)
{
    void* out = column >= p.channels ? a.dw : a.db;
    if (out) store_param(out, column >= p.channels ? column - p.channels : column, p.param_dtype, s);
}

// dw and db.
__global__ __launch_bounds__(kThreads) void norm_grad_affine_kernel(sys_group_norm_t p, NormArgs a, int parts)
{
    const int columns = 2 * p.channels, column = blockIdx.x * 16 + (threadIdx.x & 15);
    const float s = sum_parts(a.workspace, parts, columns, column);
    if (threadIdx.x < 16 && column < columns) store_affine(p, a, column, s);
}

// The chunks of every batch entry into one.
__global__ __launch_bounds__(kThreads) void norm_grad_chunks_kernel(sys_group_norm_t p, NormArgs a, NormShape shape, int blocks_an_entry)
{
    const int b = blockIdx.x / blocks_an_entry, columns = 2 * p.channels, column = (blockIdx.x - b * blocks_an_entry) * 16 + (threadIdx.x & 15);
    const float s = sum_parts(a.workspace + (size_t)b * shape.chunks * columns, shape.chunks, columns, column);
    if (threadIdx.x < 16 && column < columns) a.workspace[grad_space(p, shape).sums + (size_t)b * columns + column] = s;
}

// The first group_blocks workgroups: m1 and m2, a wavefront a group.  The others: dw and db.
__global__ __launch_bounds__(kThreads) void norm_grad_means_kernel(sys_group_norm_t p, NormArgs a, NormShape shape, unsigned group_blocks)
{
    const GradSpace g = grad_space(p, shape);
    const float* sums = a.workspace + g.sums;
    if (blockIdx.x >= group_blocks) {
        const int columns = 2 * p.channels, column = (blockIdx.x - group_blocks) * 16 + (threadIdx.x & 15);
        const float s = sum_parts(sums, p.batch, columns, column);
        if (threadIdx.x < 16 && column < columns) store_affine(p, a, column, s);
        return;
    }
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
    const float all = (float)channels * (float)p.rows;
    if (lane == 0) {
        a.workspace[g.means + 2 * at] = m1 / all;
        a.workspace[g.means + 2 * at + 1] = m2 / all;
    }
}

template <typename T, int V>
__global__ __launch_bounds__(kThreads) void norm_grad_apply_kernel(sys_group_norm_t p, NormArgs a, NormShape shape)
{
    const int b = blockIdx.x / shape.chunks, chunk = blockIdx.x - b * shape.chunks;
    const Lanes at(shape.columns);
    if (!at.there) return;
    const long long begin = chunk * shape.chunk_rows, end = begin + shape.chunk_rows < p.rows ? begin + shape.chunk_rows : p.rows;
    const float* means = a.workspace + grad_space(p, shape).means;
    for (int column = at.column; column < shape.columns; column += at.wide) {
        const int channel = column * V + V <= p.channels ? column * V : p.channels - V;
        const T* x = (const T*)a.x + b * p.x_batch + channel;
        const T* dy = (const T*)a.dy + b * p.y_batch + channel;
        T* dx = (T*)a.dx + (size_t)b * p.rows * p.channels + channel;
        GradRows<T, V> rows;
        size_t group[V];
        groups_of<V>(channel, p.channels / p.groups, (size_t)b * p.groups, group);
        const GradLane<T, V> lane(p, a, group, channel);
        float rstd[V], m1[V], m2[V];                // (rstd^2 m2 may pass what fp32 holds where dx does not)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            rstd[i] = a.rstd_in[group[i]];
            m1[i] = means[2 * group[i]];
            m2[i] = means[2 * group[i] + 1] * rstd[i];
        }
        by_activation(p.activation, [&](auto activation) {
            for (long long r = begin + at.row; r < end; r += (long long)at.tall * kGradRows) {
                rows.load(p, x, dy, r, at.tall, end);
#pragma unroll
                for (int k = 0; k < kGradRows; ++k) {
                    const long long row = r + (long long)k * at.tall;
                    if (row >= end) continue;
                    float f[V], away[V];
                    lane.template row<decltype(activation)::value>(rows.x[k], rows.dy[k], f, away);
#pragma unroll
                    for (int i = 0; i < V; ++i) f[i] = __builtin_fmaf(f[i], lane.scale[i], rstd[i] * __builtin_fmaf(away[i], -m2[i], -m1[i]));
                    Channels<T, V>::store_nt(dx + row * p.channels, f);
                }
            }
        });
    }
}

// ================================================================ launches

// Channels a lane: 16 bytes, or what divides the channels of a group.
int group_vector(const sys_group_norm_t& p)
{
    int v = p.dtype == SYS_F32 ? 4 : 8;
    while (p.channels / p.groups % v) v /= 2;
    return v;
}

int most_channels(const sys_group_norm_t& p) { return p.dtype == SYS_F32 ? 4 : 8; }

int log2_up(long long n)
{
    int l = 0;
    while ((1LL << l) < n) ++l;
    return l;
}

// Rows of a lane that are held: at most 64 registers for x, 32 each for x and dy.
constexpr int most_items(int bytes, bool grad) { return (bytes > 8 ? 16 : 32) >> grad; }

// Whether a call's rows stay in registers, and how they lie there.
bool resident_shape(const sys_group_norm_t& p, bool grad, ResidentShape* out)
{
    ResidentShape s;
    const int v = group_vector(p), element = p.dtype == SYS_F32 ? 4 : 2;
    s.columns_a_group = p.channels / p.groups / v;
    s.log_group = log2_up(s.columns_a_group);
    const int most_log = grad ? 9 : 10;                    // 512 lanes leave 256 registers, 1024 leave 128
    if (s.log_group > most_log) return false;
    // Where the unit is more than a wavefront, a part of a row of at least 64 bytes (16 x 4096 x 512 in 32 groups, bf16, 32 / 64 / 128 bytes: 59 / 31 /
    // 47 us) -- but not at the price of more than 16 rows a lane while there are few units (4 and 8 x 1024 x 320 in 32 groups: 12.5 and 12.7 us
    // with 80 bytes, 9.2 and 9.7 with 40; 16 x 1024 x 320: 13.7 and 15.2).
    s.log_tile = 0;
    const long long lanes = p.rows << s.log_group;
    const int most = most_items(v * element, grad);
    if (lanes > 64) {
        while (s.log_group + s.log_tile < 6 && s.log_tile < 5 && (p.channels / p.groups * element << s.log_tile) < 64 && (1 << s.log_tile) < p.groups
               && (p.rows <= 16LL << (most_log - s.log_group - s.log_tile - 1) || (long long)p.batch * p.groups >> (s.log_tile + 1) >= 128))
            ++s.log_tile;
    }
    const int wide = s.log_group + s.log_tile;
    // up to four rows a lane, then the whole workgroup, then as many rows as there are registers for
    s.log_unit = wide + log2_up((p.rows + 3) / 4);
    if (s.log_unit > most_log) s.log_unit = most_log;
    const long long tall = 1LL << (s.log_unit - wide);
    const long long items = (p.rows + tall - 1) / tall;
    const bool thin = lanes > 64 && (1 << s.log_tile) < p.groups && (p.channels / p.groups * element << s.log_tile) < 64;
    if (items > (thin && most > 16 ? 16 : most)) return false;     // (4 x 4096 x 320 in 32 groups, 32 rows a lane: 29 us, in chunks 17)
    s.items = (int)items;
    s.tiles = (p.groups + (1 << s.log_tile) - 1) >> s.log_tile;
    s.threads = s.log_unit > 8 ? 1 << s.log_unit : kThreads;
    // Entries at a time, where a lane has one row of each and wavefronts are left (rows of 64 x 64 channels, one / four entries, 2048 rows 9.8 / 8.6 us,
    // 4096 18 / 14, 8192 25 / 26).
    const long long waves = (((long long)p.batch * s.tiles) << s.log_unit) >> 6;
    s.entries = items == 1 && waves >= 4 * 4096 ? 4 : 1;
    const long long turns = ((long long)p.batch + s.entries - 1) / s.entries;
    // Gradients: eight wavefronts a CU where lanes hold 16 bytes of several rows, or one row (whose sums of dw and db are soon more than it), else
    // sixteen, and no more sums of dw and db than that (eight / sixteen / twenty-four a CU: 8192 x 64 x 64 channels 50 / 63 / 67 us, 8192 x 32 x 10
    // 21 / 28 / 37, 256 x 256 x 256 in 32 groups 31 / 39 / 44; 4096 x 16 x 320 in 32 groups 80 / 61 / 58, 512 x 64 x 320 39 / 27 / 28).
    const long long grad_waves = items == 1 || v * element == 16 ? 2048 : 4096;
    long long slices = grad ? (grad_waves * 64 >> s.log_unit) / s.tiles : turns;
    slices = slices < 1 ? 1 : slices > turns ? turns : slices;
    s.slices = (int)slices;
    s.rounds = (int)((turns + slices - 1) / slices);
    s.units = (int)(slices * s.tiles);
    *out = s;
    return true;
}

NormShape shape_of(const sys_group_norm_t& p)
{
    NormShape s;
    const int v = p.channels >= most_channels(p) ? most_channels(p) : 1;
    s.columns = (p.channels + v - 1) / v;
    // some 2048 workgroups, each of at least eight rows a lane (gradients of 8 x 4096 x 320 when it was chosen, four / eight / sixteen: 18 + 16 / 16.5 + 14.6 / 19 + 18 us)
    const long long tall = (s.columns < kThreads ? kThreads / s.columns : 1) * 8;
    const long long most = (p.rows + tall - 1) / tall;
    long long chunks = p.batch > 0 ? (2048LL + p.batch - 1) / p.batch : 1;
    if (chunks > most) chunks = most;
    if (chunks < 1) chunks = 1;
    s.chunk_rows = (p.rows + chunks - 1) / chunks;
    s.chunks = (int)((p.rows + s.chunk_rows - 1) / s.chunk_rows);
    return s;
}

unsigned blocks_for(long long lanes) { return (unsigned)((lanes + kThreads - 1) / kThreads); }

unsigned affine_blocks(const sys_group_norm_t& p) { return (unsigned)((2LL * p.channels + 15) / 16); }

unsigned resident_blocks(const ResidentShape& s) { return (unsigned)((((long long)s.units << s.log_unit) + s.threads - 1) / s.threads); }

template <typename T, int V, int ITEMS, int ENTRIES>
hipError_t launch_resident(const sys_group_norm_t& p, const NormArgs& a, const ResidentShape& s, hipStream_t stream)
{
    hipLaunchKernelGGL((norm_resident_kernel<T, V, ITEMS, ENTRIES>), dim3(resident_blocks(s)), dim3(s.threads), 0, stream, p, a, s);
    return hipGetLastError();
}

template <typename T, int V, int ITEMS, int ENTRIES>
hipError_t launch_grad_resident(const sys_group_norm_t& p, const NormArgs& a, const ResidentShape& s, hipStream_t stream)
{
    hipLaunchKernelGGL((norm_grad_resident_kernel<T, V, ITEMS, ENTRIES>), dim3(resident_blocks(s)), dim3(s.threads), 0, stream, p, a, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || (!a.dw && !a.db)) return e;
    hipLaunchKernelGGL(norm_grad_affine_kernel, dim3(affine_blocks(p)), dim3(kThreads), 0, stream, p, a, s.slices);
    return hipGetLastError();
}

template <typename T, int V>
hipError_t launch_items(bool grad, const sys_group_norm_t& p, const NormArgs& a, const ResidentShape& s, hipStream_t stream)
{
    if (s.entries > 1) return grad ? launch_grad_resident<T, V, 1, 4>(p, a, s, stream) : launch_resident<T, V, 1, 4>(p, a, s, stream);
    if (s.items == 1) return grad ? launch_grad_resident<T, V, 1, 1>(p, a, s, stream) : launch_resident<T, V, 1, 1>(p, a, s, stream);
    if (s.items <= 4) return grad ? launch_grad_resident<T, V, 4, 1>(p, a, s, stream) : launch_resident<T, V, 4, 1>(p, a, s, stream);
    if (s.items <= 8) return grad ? launch_grad_resident<T, V, 8, 1>(p, a, s, stream) : launch_resident<T, V, 8, 1>(p, a, s, stream);
    if (s.items <= 16 && !grad) return launch_resident<T, V, 16, 1>(p, a, s, stream);
    if constexpr (most_items(V * (int)sizeof(T), false) > 16) return grad ? launch_grad_resident<T, V, 16, 1>(p, a, s, stream) : launch_resident<T, V, 32, 1>(p, a, s, stream);
    return hipErrorInvalidValue;                           // (resident_shape has no such shape)
}

template <typename T, int V>
hipError_t launch_chunks(bool grad, const sys_group_norm_t& p, const NormArgs& a, hipStream_t s)
{
    const NormShape shape = shape_of(p);
    const dim3 grid((unsigned)(shape.chunks * p.batch)), block(kThreads);
    const unsigned group_blocks = blocks_for(64LL * p.batch * p.groups);
    hipError_t e;
    if (!grad) {
        hipLaunchKernelGGL((norm_moments_kernel<T, V>), grid, block, 0, s, p, a, shape);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        hipLaunchKernelGGL((norm_statistics_kernel<T>), dim3((unsigned)(p.batch * p.groups)), block, 0, s, p, a, shape);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        hipLaunchKernelGGL((norm_apply_kernel<T, V>), grid, block, 0, s, p, a, shape);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((norm_grad_sums_kernel<T, V>), grid, block, 0, s, p, a, shape);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(norm_grad_chunks_kernel, dim3(affine_blocks(p) * (unsigned)p.batch), block, 0, s, p, a, shape, (int)affine_blocks(p));
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(norm_grad_means_kernel, dim3(group_blocks + (a.dw || a.db ? affine_blocks(p) : 0)), block, 0, s, p, a, shape, group_blocks);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL((norm_grad_apply_kernel<T, V>), grid, block, 0, s, p, a, shape);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_type(bool grad, const sys_group_norm_t& p, const NormArgs& a, hipStream_t s)
{
    ResidentShape r;
    if (resident_shape(p, grad, &r)) {
        switch (group_vector(p)) {
        case 1: return launch_items<T, 1>(grad, p, a, r, s);
        case 2: return launch_items<T, 2>(grad, p, a, r, s);
        case 4: return launch_items<T, 4>(grad, p, a, r, s);
        default:
            if constexpr (sizeof(T) == 2) return launch_items<T, 8>(grad, p, a, r, s);
            return hipErrorInvalidValue;
        }
    }
    return p.channels >= kLaneChannels<T> ? launch_chunks<T, kLaneChannels<T>>(grad, p, a, s) : launch_chunks<T, 1>(grad, p, a, s);
}

hipError_t launch(bool grad, const sys_group_norm_t& p, const NormArgs& a, hipStream_t s)
{
    const long long most = 0x7fffffffLL;
    if (!p.batch) {                                        // (only the gradients come here: sums of nothing)
        if (!a.dw && !a.db) return hipSuccess;
        hipLaunchKernelGGL(norm_grad_affine_kernel, dim3(affine_blocks(p)), dim3(kThreads), 0, s, p, a, 0);
        return hipGetLastError();
    }
    ResidentShape r;
    if (resident_shape(p, grad, &r) ? ((long long)p.batch * r.tiles << r.log_unit) > most * kThreads || (long long)p.batch * r.tiles > most
                                    : 64LL * p.batch * p.groups > most * kThreads || (long long)shape_of(p).chunks * p.batch > most
                                          || (long long)affine_blocks(p) * p.batch > most)
        return hipErrorInvalidConfiguration;
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
    ResidentShape r;
    if (!p.batch || resident_shape(p, false, &r)) return 0;
    return ((size_t)p.batch * shape_of(p).chunks * 2 * p.channels + (size_t)p.batch * p.groups * 2) * sizeof(float);
}

size_t group_norm_grad_workspace(const sys_group_norm_t& p)
{
    ResidentShape r;
    if (!p.batch) return 0;
    if (resident_shape(p, true, &r)) return (size_t)r.slices * 2 * p.channels * sizeof(float);
    return grad_space(p, shape_of(p)).floats * sizeof(float);
}

}  // namespace sysconv
