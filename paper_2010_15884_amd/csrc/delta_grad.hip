// Gradients of the gated delta rule in chunks of 64 positions (delta_tile.h has the forward formulas, the precision and the layout).
//
// With dO the gradient of the outputs times `scale`, dS' that of the state behind a chunk, and E = e^(G_end - G):
//   dU = P^T dO + E (K dS'),   Z = X^T dU,   dV = b Z,   dS = e^(G_end) dS' + Q^T (e^G dO) - K^T (e^G b Z)
// which is a sweep over the chunks from the last to the first, like the one forwards and laid out like it; it leaves dS' and Z, the sweep forwards S
// and U.  Then all chunks side by side: with the ratios of decays r_ij = e^(G_i - G_j) and
//   B_ij = r_ij dO_i . U_j  (j <= i),   C_ij = -r_ij Z_i . U_j  (j < i),
//   dQ = e^G (dO S^T) + B K,   Kr = -e^G (Z S^T) + C K,   Kc = E (U dS'^T) + B^T Q + (b C)^T K,   dK = b Kr + Kc,
//   db_i = Z_i . V_i + k_i . Kr_i,   and the logarithm of a decay gets the sum of the gradients dG of the sums G from its position on.
// The shares of B and C in dG_i cancel between a row and a column of the two positions' entry: with
//   H_ij = B_ij q_i . k_j + b_i C_ij k_i . k_j  (j < i)  they are the row's sum less the column's, of the same numbers and in 64 bits (what a row's sum is
// rounded by would reach all positions before it: dA off by 2e-6 of itself),
// and what else there is comes from the products with the states: q_i . (e^G S dO)_i + b_i k_i . (-e^G S Z)_i from the position on, E_i k_i . (dS' U_i) up
// to it, e^(G_end) <S, dS'> for all; sums over the positions of a chunk are in 64 bits.
//
// Four sequences of 2048, 8 key heads and 16 value heads of 128 in bf16 (22000 us as torch operators): 499 us.  By the profiler, under which they add up to 5 % more, 48 us for the chunks'
// matrices, 109 for the sweep forwards, 141 for the one backwards, 215 for the chunks' gradients, 6 + 5 for what gates and rates get.  S, dS', U and Z are 400 MB that are written and read once: the sweep
// forwards takes 75 us without its stores, and the chunks' gradients read 546 MB at 2.5 TB/s over the launch, more while they go through the columns.
#include "delta_tile.h"
#include "launch.h"

namespace sysconv {
namespace {

template <typename T, int KD, int NT>
__global__ __launch_bounds__(kSweepThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void delta_back_kernel(sys_gated_delta_t p, DeltaArgs a, DeltaShape shape,
                                                                                                             DeltaPlanes w)
{
    constexpr int NX = kInputParts<T>, KS = KD / 32, TW = KD / 64;
    constexpr bool kAtOnce = NX * NT <= 2;         // there are registers for all operands of a product
    const unsigned place = xcd_place(blockIdx.x, gridDim.x);
    const int tile = place % shape.tiles, rest = place / shape.tiles, head = rest % p.value_heads, b = rest / p.value_heads;
    const int key_head = head / (p.value_heads / p.key_heads);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) & 3, lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const bool chain = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8) == 0;
    const int last = sequence_length(a.lengths, b, p.length), chunks = (last + kChunk - 1) / kChunk, top = chunks > 0 ? chunks - 1 : 0;
    const int first_step = wave >> 1;              // of X^T and P^T: what lies below their diagonals is zero
    const int my_row = tile_row(wave, 4 * g);
    int column[NT];
    bool there[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) column[n] = (tile * NT + n) * 16 + r, there[n] = column[n] < p.value_dim;

    __shared__ Operands<KS, 3, NT> states;
    __shared__ Operands<2, 3, NT> misses, writes, weighted;
    __shared__ Operands<2, NX, NT> outs;
    // P^T dO and Q^T (e^G dO) of the next chunk, Z of this one
    __shared__ f4 of_outs[4][NT][64], of_queries[4 * TW][NT][64], zs[4][NT][64];

    const size_t vc = ((size_t)b * p.value_heads + head) * shape.chunks, kc = ((size_t)b * p.key_heads + key_head) * shape.chunks;
    const long long dv_row = (long long)p.value_heads * p.value_dim;
    if (chain) {
        const size_t state_base = ((size_t)b * p.value_heads + head) * p.key_dim * p.value_dim;
        const unsigned state_bytes = (unsigned)(p.key_dim * p.value_dim) * 4u;
        f4 s[TW][NT];
        {
            const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc((void*)(a.dstate_out + state_base), 0, a.dstate_out ? state_bytes : 0u, 0x00027000);
#pragma unroll
            for (int i = 0; i < TW; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const unsigned row = tile_row(TW * wave + i, 4 * g) + e;
                        s[i][n][e] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(from, there[n] ? (row * p.value_dim + column[n]) * 4u : kNowhere, 0, 0));
                    }
        }
        auto put_state = [&] {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if constexpr (TW == 2) states.put(wave, n, lane, s[0][n], s[1][n]);
                else states.put_half(wave, n, lane, s[0][n]);
            }
        };
        b8 ka[KS][NX], kta[TW][2][NX], xa[2][3];
        f4 next_gamma, next_left, next_strength;
        float next_end;
        auto fetch_keys = [&](int c) {
#pragma unroll
            for (int i = 0; i < KS; ++i)
#pragma unroll
                for (int n = 0; n < NX; ++n) ka[i][n] = operand(w.k + ((kc + c) * NX + n) * kChunk * KD, KS, wave, i, lane);
            const float* from = w.scalars + (vc + c) * kScalars * kChunk;
            next_gamma = *(const f4*)(from + kGamma * kChunk + my_row);
            next_left = *(const f4*)(from + kLeft * kChunk + my_row);
            next_strength = *(const f4*)(from + kStrength * kChunk + my_row);
            next_end = from[kGamma * kChunk + kChunk - 1];
        };
        auto fetch_inverse = [&](int c) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (i >= first_step) {
#pragma unroll
                    for (int n = 0; n < 3; ++n) xa[i][n] = operand(w.xt + ((vc + c) * 3 + n) * kSquare, 2, wave, i, lane);
                }
        };
        auto fetch_transposed = [&](int c) {
#pragma unroll
            for (int i = 0; i < TW; ++i)
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int n = 0; n < NX; ++n) kta[i][m][n] = operand(w.kt + ((kc + c) * NX + n) * kChunk * KD, 2, TW * wave + i, m, lane);
        };
        if (chunks > 0) {
            fetch_keys(top), fetch_inverse(top), fetch_transposed(top);
            put_state();
            lds_barrier();
        }
        for (int c = top; c >= 0 && chunks > 0; --c) {
            const int next = c > 0 ? c - 1 : 0;
            lds_barrier();
            // dU
            f4 ks[NT][3] = {};
            {
                b8 parts[KS][NT][3];
#pragma unroll
                for (int i = 0; i < KS; ++i)
#pragma unroll
                    for (int n = 0; n < NT; ++n) states.take(i, n, lane, parts[i][n]);
                if (kAtOnce) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < KS; ++i)
#pragma unroll
                    for (int n = 0; n < NT; ++n) multiply_apart<2>(ka[i], parts[i][n], ks[n]);
            }
            const f4 gamma = next_gamma, left = next_left, strength = next_strength;
            const float end = next_end;
#pragma unroll
            for (int n = 0; n < NT; ++n) misses.put_half(wave, n, lane, of_outs[wave][n][lane] + left * joined(ks[n]));
            fetch_keys(next);
            lds_barrier();
            // Z
            f4 z[NT][3] = {};
            {
                b8 parts[2][NT][3];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int n = 0; n < NT; ++n) misses.take(i, n, lane, parts[i][n]);
                if (kAtOnce) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (i >= first_step) {
#pragma unroll
                        for (int n = 0; n < NT; ++n) multiply_apart<2>(xa[i], parts[i][n], z[n]);
                    }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const f4 sum = joined(z[n]);
                writes.put_half(wave, n, lane, -(gamma * strength * sum));
                zs[wave][n][lane] = sum;
            }
            fetch_inverse(next);
            lds_barrier();
            // dS before the chunk
            {
                b8 parts[2][NT][3];
                f4 more[TW][NT][3] = {};
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int n = 0; n < NT; ++n) writes.take(m, n, lane, parts[m][n]);
#pragma unroll
                for (int i = 0; i < TW; ++i)
#pragma unroll
                    for (int n = 0; n < NT; ++n) more[i][n][1] = of_queries[TW * wave + i][n][lane];
                if (kAtOnce) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int i = 0; i < TW; ++i) more[i][n][0] = s[i][n] * end;
#pragma unroll
                    for (int m = 0; m < 2; ++m)
#pragma unroll
                        for (int i = 0; i < TW; ++i) multiply_apart<2>(kta[i][m], parts[m][n], more[i][n]);
#pragma unroll
                    for (int i = 0; i < TW; ++i) s[i][n] = joined(more[i][n]);
                }
            }
            put_state();
            fetch_transposed(next);
        }
        if (a.dstate) {
            const __amdgpu_buffer_rsrc_t to = __builtin_amdgcn_make_buffer_rsrc((void*)(a.dstate + state_base), 0, state_bytes, 0x00027000);
#pragma unroll
            for (int i = 0; i < TW; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const unsigned row = tile_row(TW * wave + i, 4 * g) + e;
                        const float value = s[i][n][e];
                        __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, value), to, there[n] ? (row * p.value_dim + column[n]) * 4u : kNowhere, 0, 0);
                    }
        }
    } else {
        // a chunk ahead what depends on dO alone, and behind it what the gradients need: dS behind the chunk, Z, and dV
        ChunkRows<T> dy((const T*)a.dy + b * p.y_batch + head * p.value_dim, p.y_row, p.value_dim, top, last);
        ChunkRows<T> dv((const T*)a.dv + (long long)b * p.length * dv_row + head * p.value_dim, dv_row, p.value_dim, top, p.length);
        unsigned dy_at[NT][4], dv_at[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                dy_at[n][e] = there[n] ? dy.offset(my_row + e, column[n]) : kNowhere;
                dv_at[n][e] = there[n] ? dv.offset(my_row + e, column[n]) : kNowhere;
            }
        b8 qta[TW][2][NX], pa[2][3];
        unsigned next_dy[NT][4];
        f4 next_gamma, next_strength;
        auto fetch_outs = [&](int c) {
            const __amdgpu_buffer_rsrc_t rows = dy.buffer();
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) next_dy[n][e] = buffer_load<T>(rows, my_row + e < dy.exist ? dy_at[n][e] : kNowhere);
            const float* from = w.scalars + (vc + c) * kScalars * kChunk;
            next_gamma = *(const f4*)(from + kGamma * kChunk + my_row);
            next_strength = *(const f4*)(from + kStrength * kChunk + my_row);
        };
        auto fetch_mixed = [&](int c) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (i >= first_step) {
#pragma unroll
                    for (int n = 0; n < 3; ++n) pa[i][n] = operand(w.pt + ((vc + c) * 3 + n) * kSquare, 2, wave, i, lane);
                }
        };
        auto fetch_queries = [&](int c) {
#pragma unroll
            for (int i = 0; i < TW; ++i)
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int n = 0; n < NX; ++n) qta[i][m][n] = operand(w.qt + ((kc + c) * NX + n) * kChunk * KD, 2, TW * wave + i, m, lane);
        };
        auto put_outs = [&] {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                f4 own;
#pragma unroll
                for (int e = 0; e < 4; ++e) own[e] = loaded<T>(next_dy[n][e]);
                outs.put_half(wave, n, lane, own);
                weighted.put_half(wave, n, lane, next_gamma * p.scale * own);
            }
        };
        auto mixed = [&] {                         // P^T dO
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                f4 u[3] = {};
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (i >= first_step) {
                        b8 parts[NX];
                        outs.take(i, n, lane, parts);
                        multiply_apart<2>(pa[i], parts, u);
                    }
                of_outs[wave][n][lane] = joined(u);
            }
        };
        auto queries = [&] {                       // Q^T (e^G dO)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                f4 more[TW][3] = {};
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    b8 parts[3];
                    weighted.take(m, n, lane, parts);
#pragma unroll
                    for (int i = 0; i < TW; ++i) multiply_apart<2>(qta[i][m], parts, more[i]);
                }
#pragma unroll
                for (int i = 0; i < TW; ++i) of_queries[TW * wave + i][n][lane] = joined(more[i]);
            }
        };
        auto store_values = [&](int c, f4 strength) {
            const __amdgpu_buffer_rsrc_t rows = dv.buffer();
            const int left = last - c * kChunk - my_row;               // (behind the sequence 0, also where a gradient is not finite)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const f4 z = zs[wave][n][lane], values = strength * z;
                *(f4*)(w.z + block_place(vc + c, kChunk, shape.columns, my_row + (r & 3), (tile * NT + n) * 16 + (r & ~3))) = turn_quad(z);
#pragma unroll
                for (int e = 0; e < 4; ++e) buffer_store<T>(rows, dv_at[n][e], (T)(e < left ? values[e] : 0.0f));
            }
            dv.move(-1);
        };
        if (chunks > 0) {
            fetch_outs(top), fetch_mixed(top), fetch_queries(top);
            f4 behind_strength = {}, strength = next_strength;
            put_outs();
            lds_barrier();
            mixed();
            for (int c = top; c >= 0; --c) {
                const int next = c > 0 ? c - 1 : 0;
                dy.move(next - c);                 // (a buffer has no lower end: rows before the first chunk must not be asked for, it is read twice instead)
                fetch_outs(next), fetch_mixed(next);
                // (dS stays as it is to the third barrier, Z to the second of the next chunk: the work is spread so that the other four wait for little of it)
                lds_barrier();
                queries();
                if (c < top) store_values(c + 1, behind_strength);
                fetch_queries(next);
                lds_barrier();
#pragma unroll
                for (int i = 0; i < TW; ++i)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        *(f4*)(w.ds + block_place(vc + c, KD, shape.columns, tile_row(TW * wave + i, 4 * g) + (r & 3), (tile * NT + n) * 16 + (r & ~3))) =
                            turn_quad(signed_rows(states.numbers(TW * wave + i, n, lane), TW * wave + i));
                behind_strength = strength, strength = next_strength;
                put_outs();
                lds_barrier();
                mixed();
            }
            store_values(0, behind_strength);
        }
        T* behind = (T*)a.dv + (long long)b * p.length * dv_row + head * p.value_dim;
        for (int t = chunks * kChunk + (int)((threadIdx.x & 255) >> 4); t < p.length; t += kSweepThreads / 32)
#pragma unroll
            for (int n = 0; n < NT; ++n)
                if (there[n]) behind[t * dv_row + column[n]] = (T)0.0f;
    }
}

// Sums over rows of 16 lanes of four values a lane: lane j of a quad gets that of v[j].
template <int CONTROL>
__device__ __forceinline__ double dpp(double v)
{
    const unsigned long long bits = __builtin_bit_cast(unsigned long long, v);
    const unsigned low = __builtin_amdgcn_mov_dpp((int)(unsigned)bits, CONTROL, 0xF, 0xF, true), high = __builtin_amdgcn_mov_dpp((int)(unsigned)(bits >> 32), CONTROL, 0xF, 0xF, true);
    return __builtin_bit_cast(double, (unsigned long long)high << 32 | low);
}
template <typename V>
__device__ __forceinline__ V row_sums(V v0, V v1, V v2, V v3)
{
    const bool odd = threadIdx.x & 1, high = threadIdx.x & 2;
    const V a = (odd ? v1 : v0) + dpp<0xB1>(odd ? v0 : v1), b = (odd ? v3 : v2) + dpp<0xB1>(odd ? v2 : v3);
    V sum = (high ? b : a) + dpp<0x4E>(high ? a : b);
    sum += dpp<0x124>(sum);                        // the quad four lanes away, and then the pair of quads eight lanes away
    return sum + dpp<0x128>(sum);
}

// The first or the last four numbers of an operand.
template <int N>
__device__ __forceinline__ f4 four_of(const b8 (&parts)[N], bool last)
{
    f4 sum = {};
#pragma unroll
    for (int n = N - 1; n >= 0; --n) {
        const u4 all = __builtin_bit_cast(u4, parts[n]);
        const unsigned a = last ? all[2] : all[0], b = last ? all[3] : all[1];
        sum += f4{__builtin_bit_cast(float, a << 16), __builtin_bit_cast(float, a & 0xffff0000u), __builtin_bit_cast(float, b << 16), __builtin_bit_cast(float, b & 0xffff0000u)};
    }
    return sum;
}

// Eight neighbouring fp32 numbers.
struct EightFloats {
    float v[8];
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t plane, unsigned offset, int block)
    {
        const f4 a = __builtin_bit_cast(f4, __builtin_amdgcn_raw_buffer_load_b128(plane, offset, block, 0));
        const f4 b = __builtin_bit_cast(f4, __builtin_amdgcn_raw_buffer_load_b128(plane, offset + 16, block, 0));
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
    }
};

// A workgroup a chunk of a key head, through the value heads that share it.  Eight wavefronts: wavefront w the positions of tile w % 4 and half w / 4 of the keys' entries; of the
// squares the first half has B and the second C.  S, dS' and U of 32 value columns at a time are split on their way into LDS, as the operands
// that all wavefronts need, and <S, dS'> is taken there.
// A head of 128 x 128 in bf16 is some 50 thousand clocks: 17 in products (70 % of them matrix instructions), 17 in splitting what comes from memory and waiting for it, 6 for the
// squares, 7 for what they give, the rest barriers and sums.  With two parts instead of three in the products it took 10 % less, but the gradients of the rates were off by
// 2.4e-6 of themselves instead of 3e-7.  One workgroup of eight wavefronts a CU: its operands and K, Q and their transposes fill LDS, and the squares take turns with their own
// transposes (with two parts there was room for both, and the launch of 4 x 2048 positions took 200 us instead of 211, but see delta_tile.h).
constexpr int kGradThreads = 512;

template <typename T, int KD>
__global__ __launch_bounds__(kGradThreads) void delta_grad_kernel(sys_gated_delta_t p, DeltaArgs a, DeltaShape shape, DeltaPlanes w)
{
    constexpr int NX = kInputParts<T>, KS = KD / 32, KT = KD / 16, KH = KT / 2, kPitch = kChunk + 8;
    const int shared = shape.apart ? 1 : p.value_heads / p.key_heads, groups = p.value_heads / shared;     // value heads of this workgroup, and groups of them
    const int chunk = blockIdx.x % shape.chunks, rest = blockIdx.x / shape.chunks, first_head = rest % groups * shared, b = rest / groups;
    const int key_head = first_head / (p.value_heads / p.key_heads);
    const int t0 = chunk * kChunk, last = sequence_length(a.lengths, b, p.length), rows = last - t0;
    const int tid = threadIdx.x, half = __builtin_amdgcn_readfirstlane(tid >> 8);
    // (the tiles of the second half the other way round: those of later positions have more below the diagonal, and wavefronts four apart share a SIMD)
    const int quarter = __builtin_amdgcn_readfirstlane(tid >> 6) & 3, wave = half ? 3 - quarter : quarter;
    const int here = p.length - t0 < kChunk ? p.length - t0 : kChunk;  // rows of the results
    const long long at0 = (long long)b * p.length + t0;
    if (rows <= 0) {
        for (int i = tid; !shape.apart && i < here * p.key_dim; i += kGradThreads) {
            const long long at = ((at0 + i / p.key_dim) * p.key_heads + key_head) * p.key_dim + i % p.key_dim;
            ((T*)a.dq)[at] = (T)0.0f;
            ((T*)a.dk)[at] = (T)0.0f;
        }
        return;
    }
    const size_t kc = ((size_t)b * p.key_heads + key_head) * shape.chunks + chunk;
    const int middle = wave >> 1;

    constexpr int kBlock = 64 + 4;                 // an operand's pieces, 17 for 16: lanes that write the four pieces of a row meet other banks
    struct Columns { b8 s[KT][3][kBlock], ds[KT][3][kBlock], u[4][3][kBlock], z[4][3][kBlock], dy[4][NX][kBlock]; };
    // B and b C, as they are and transposed: side by side, or one after the other where K and Q take the room
    constexpr bool kKeep = NX < 3, kKeepTransposed = NX == 1, kAtOnce = !kKeep;
    struct Squares {
        bf16_t v[kAtOnce ? 2 : 1][2][3][kChunk][kPitch];
        f4 numbers[kAtOnce ? 1 : 24][64];          // a tile's lanes: those that the transposed ones are made of
    };
    __shared__ union Pool {
        Columns columns;
        Squares squares;
        __device__ Pool() {}
    } pool;
    __shared__ float rows_db[2][kChunk], rows_end[2][kChunk], rows_zv[kChunk];
    __shared__ double rows_dg[2][kChunk], columns_dg[8][kChunk], waves_end[8][4];
    __shared__ __attribute__((aligned(16))) float scalars[kScalars * kChunk];

    // K and Q, which all value heads use, as operands and transposed: as many as LDS has room for
    __shared__ b8 kept[2][kKeep ? NX : 1][kKeep ? 4 * KS : 1][64], kept_transposed[2][kKeepTransposed ? 4 * KS : 1][64];
    if (kKeep) {
        for (int i = tid; i < NX * 4 * KS * 64; i += kGradThreads) {
            const int n = i / (4 * KS * 64), at = i % (4 * KS * 64);
            (&kept[0][n][0][0])[at] = *(const b8*)(w.k + (kc * NX + n) * kChunk * KD + at * 8);
            (&kept[1][n][0][0])[at] = *(const b8*)(w.q + (kc * NX + n) * kChunk * KD + at * 8);
            if (kKeepTransposed) {
                (&kept_transposed[0][0][0])[at] = *(const b8*)(w.kt + kc * kChunk * KD + at * 8);
                (&kept_transposed[1][0][0])[at] = *(const b8*)(w.qt + kc * kChunk * KD + at * 8);
            }
        }
    }
    f4 dq_all[KH] = {}, dk_all[KH] = {};
    const int steps = shape.columns / 32, items = steps * shared;      // of 32 columns, of one head after the other
    // What is on its way from memory, an item ahead; beyond the end of a head too where there are registers for it
    constexpr bool kBeyond = NX == 1;
    struct Ahead {
        EightFloats s, ds, rows;
        Eight<T> values;                           // V or dO
    } ahead;
    int fetch_head = first_head, fetch_step = 0;
    auto fetch = [&](Ahead& to, int tid) {
        // pieces of eight: four a row and step; S and dS' by all lanes, Z and V by the first half of them, U and dO by the second
        const size_t vc = ((size_t)b * p.value_heads + fetch_head) * shape.chunks + chunk;
        auto plane = [&](float* of, int rows) {
            return __builtin_amdgcn_make_buffer_rsrc((void*)(of + vc * rows * shape.columns), 0, (unsigned)(rows * shape.columns) * 4u, 0x00027000);
        };
        const int row = (tid & 255) >> 2, at = 8 * (tid & 3);
        if (tid < KD * 4) {
            const unsigned state_at = ((tid >> 2) * 32 + at) * 4u;
            to.s.load(plane(w.s, KD), state_at, fetch_step * KD * 128);
            to.ds.load(plane(w.ds, KD), state_at, fetch_step * KD * 128);
        }
        to.rows.load(plane(half ? w.u : w.z, kChunk), (row * 32 + at) * 4u, fetch_step * kChunk * 128);
        const T* base = half ? (const T*)a.dy + b * p.y_batch : (const T*)a.v + b * p.v_batch;
        const ChunkRows<T> values(base + fetch_head * p.value_dim, half ? p.y_row : p.v_row, p.value_dim, chunk, last);
        const int left = row < rows ? p.value_dim - 32 * fetch_step - at : 0;
        const unsigned offset = values.offset(row, 32 * fetch_step + at);
        if (shape.whole_values) to.values.load(values.buffer(), left > 0 ? offset : kNowhere);
        else to.values.load_each(values.buffer(), offset, left);
        if (++fetch_step == steps) fetch_step = 0, ++fetch_head;
    };
    if (kBeyond) fetch(ahead, threadIdx.x);
    for (int h = 0, item = 0; h < shared; ++h) {
        const int head = first_head + h;
        const size_t vc = ((size_t)b * p.value_heads + head) * shape.chunks + chunk;
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));              // (see below)
        const int lane = tid & 63, place = lane + (lane >> 4);
        const int piece_row = (tid & 255) >> 2, piece = 17 * (tid & 3) + row_in_tile(piece_row);
        auto scalar = [&] { return tid < kScalars * kChunk ? w.scalars[vc * kScalars * kChunk + tid] : 0.0f; };
        const float early_scalar = NX == 2 ? scalar() : 0.0f;
        f4 dq[KH] = {}, zs[KH] = {}, us[KH] = {}, square[4] = {};
        float both = 0.0f;                         // (8 products a lane and step; <S, dS'> is the sum of key_dim x value_dim terms of either sign, and all positions of the chunk get it)
        float zv = 0.0f;
        if (!kBeyond) fetch(ahead, tid);
        auto stage = [&](Ahead& next) {
            lds_barrier();
            b8 parts[3];
            if (tid < KD * 4) {
                const int tile = tile_of(tid >> 2), to = 17 * (tid & 3) + row_in_tile(tid >> 2);
#pragma unroll
                for (int i = 0; i < 8; ++i) both = __builtin_fmaf(next.s.v[i], next.ds.v[i], both);
                split8(next.s.v, parts);
#pragma unroll
                for (int m = 0; m < 3; ++m) pool.columns.s[tile][m][to] = parts[m];
                split8(next.ds.v, parts);
#pragma unroll
                for (int m = 0; m < 3; ++m) pool.columns.ds[tile][m][to] = parts[m];
            }
            const int tile = tile_of(piece_row);
            if (half) {
                b8 values[NX];
                next.values.split(values);
                split8(next.rows.v, parts);
#pragma unroll
                for (int m = 0; m < 3; ++m) pool.columns.u[tile][m][piece] = parts[m];
#pragma unroll
                for (int m = 0; m < NX; ++m) pool.columns.dy[tile][m][piece] = values[m];
            } else {
                float values[8];
                next.values.values(values);
#pragma unroll
                for (int i = 0; i < 8; ++i) zv = __builtin_fmaf(next.rows.v[i], values[i], zv);
                split8(next.rows.v, parts);
#pragma unroll
                for (int m = 0; m < 3; ++m) pool.columns.z[tile][m][piece] = parts[m];
            }
            ++item;
            if (NX < 3 && (kBeyond ? item < items : item % steps != 0)) fetch(next, tid);
            lds_barrier();
        };
        for (int step = 0; step < steps; ++step) {
            stage(ahead);
            b8 oa[NX], za[3], ua[3];
#pragma unroll
            for (int m = 0; m < NX; ++m) oa[m] = pool.columns.dy[wave][m][place];
#pragma unroll
            for (int m = 0; m < 3; ++m) za[m] = pool.columns.z[wave][m][place];
            auto squares = [&](const auto& of, auto which) {
#pragma unroll
                for (int n = 2 * decltype(which)::value; n < 2 * decltype(which)::value + 2; ++n) {
                    b8 ub[3];
#pragma unroll
                    for (int m = 0; m < 3; ++m) ub[m] = pool.columns.u[n][m][place];
                    square[n] = multiply<2>(of, ub, square[n]);
                }
            };
            if (half) {
                squares(za, std::integral_constant<int, 0>());
                if (middle) squares(za, std::integral_constant<int, 1>());
            } else {
                squares(oa, std::integral_constant<int, 0>());
                if (middle) squares(oa, std::integral_constant<int, 1>());
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int m = 0; m < 3; ++m) ua[m] = pool.columns.u[wave][m][place];
#pragma unroll
            for (int i = 0; i < KH; ++i) {
                __builtin_amdgcn_sched_barrier(0);                     // (operands of one tile at a time: 256 registers do)
                const int t = half * KH + i;
                b8 part[3];
#pragma unroll
                for (int m = 0; m < 3; ++m) part[m] = pool.columns.s[t][m][place];
                dq[i] = multiply<2>(oa, part, dq[i]);
                zs[i] = multiply<2>(za, part, zs[i]);
                if (NX > 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int m = 0; m < 3; ++m) part[m] = pool.columns.ds[t][m][place];
                us[i] = multiply<2>(ua, part, us[i]);
            }
            // (fp32 has the registers behind the products only)
            __builtin_amdgcn_sched_barrier(0);
            if (NX == 3 && item % steps != 0) fetch(ahead, tid);
        }
        asm volatile("" : "+v"(tid));
        if (tid < kScalars * kChunk) scalars[tid] = NX == 2 ? early_scalar : scalar();
        lds_barrier();
        int again = lane;
        asm volatile("" : "+v"(again));
        const int row = tile_row(wave, again & 15), mine = tile_row(wave, 4 * (again >> 4));       // of A operands; the first of four of D
        const double* sums = (const double*)(scalars + kSums * kChunk);
        const f4 strength = *(const f4*)(scalars + kStrength * kChunk + mine);
        // (new addresses for every head, as far as the compiler knows: worked out or loaded ahead of the loop they would take all registers)
        size_t keys_at = kc * NX * kChunk * KD;
        asm volatile("" : "+s"(keys_at));
        const bf16_t *kt = w.kt + keys_at, *qt = w.qt + keys_at, *kp = w.k + keys_at, *qp = w.q + keys_at;
        const bf16_t* own = half ? kp : qp;        // rows of C belong to keys, those of B to queries
        f4 of_strength = {};
        double of_h[4] = {};
        const int my_tiles = 12 * half + (middle ? 4 * (wave - 1) : 2 * wave);     // (two or four a wavefront)
        // the squares, as they are and transposed: two tiles of columns at a time
        auto squares = [&](auto which, auto second) {
            constexpr int N0 = 2 * decltype(which)::value;
            constexpr bool C = decltype(second)::value;
            constexpr int kSide = NX == 1 && KD == 64 ? 2 : 1;                     // tiles whose inner products are worked out side by side
            f4 inner[2] = {};
            auto products = [&](int n0) {
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    if (NX > 1) __builtin_amdgcn_sched_barrier(0);
                    b8 xa[NX], kb[kSide][NX];
#pragma unroll
                    for (int m = 0; m < NX; ++m) {
                        if constexpr (kKeep) xa[m] = kept[C ? 0 : 1][m][wave * KS + s][again];
                        else xa[m] = operand(own + m * kChunk * KD, KS, wave, s, again);
#pragma unroll
                        for (int n = 0; n < kSide; ++n) {
                            if constexpr (kKeep) kb[n][m] = kept[0][m][(N0 + n0 + n) * KS + s][again];
                            else kb[n][m] = operand(kp + m * kChunk * KD, KS, N0 + n0 + n, s, again);
                        }
                    }
#pragma unroll
                    for (int n = 0; n < kSide; ++n) inner[n0 + n] = multiply<2>(xa, kb[n], inner[n0 + n]);
                }
            };
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                if (n % kSide == 0) products(n);
                __builtin_amdgcn_sched_barrier(0);
                const int column = tile_row(N0 + n, again & 15);
                const double column_sum = sums[column];
                const f4 own_square = n & 1 ? -square[N0 + n] : square[N0 + n];
                f4 f;
                double of_column = 0.0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float ratio = fast_exp2((float)(sums[mine + e] - column_sum));
                    const bool below = column < mine + e;
                    if (C) {
                        const float c = below ? -(ratio * own_square[e]) : 0.0f;
                        of_strength[e] = below ? __builtin_fmaf(c, inner[n][e], of_strength[e]) : of_strength[e];
                        f[e] = strength[e] * c;
                    } else {
                        f[e] = column <= mine + e ? p.scale * (ratio * own_square[e]) : 0.0f;
                    }
                    const double product = below ? (double)(f[e] * inner[n][e]) : 0.0;
                    of_h[e] += product;
                    of_column += product;
                }
                of_column += __shfl_xor(of_column, 16);
                of_column += __shfl_xor(of_column, 32);
                if (again < 16) columns_dg[4 * half + wave][column] = of_column;
                u2 parts[3];
                split4(f, parts);
#pragma unroll
                for (int m = 0; m < 3; ++m) {
                    if constexpr (kAtOnce) *(u2*)&pool.squares.v[1][C][m][column][mine] = parts[m];
#pragma unroll
                    for (int e = 0; e < 4; ++e) pool.squares.v[0][C][m][mine + e][column] = as_bf16(parts[m][e / 2] >> 16 * (e & 1));
                }
                if constexpr (!kAtOnce) pool.squares.numbers[my_tiles + N0 + n][again] = f;
            }
        };
        auto put_transposed = [&] {
#pragma unroll
            for (int n = 0; n < 4; ++n)
                if (n < 2 || middle) {
                    const int column = tile_row(n, again & 15);
                    u2 parts[3];
                    split4(pool.squares.numbers[my_tiles + n][again], parts);
#pragma unroll
                    for (int m = 0; m < 3; ++m) *(u2*)&pool.squares.v[0][half][m][column][mine] = parts[m];
                }
        };
        auto both_squares = [&](auto second) {
            squares(std::integral_constant<int, 0>(), second);
            if (middle) {
                squares(std::integral_constant<int, 1>(), second);
            } else if (again < 16) {
                columns_dg[4 * half + wave][tile_row(2, again)] = 0.0;
                columns_dg[4 * half + wave][tile_row(3, again)] = 0.0;
            }
        };
        if (half) both_squares(std::true_type());
        else both_squares(std::false_type());
        lds_barrier();
        // what they and the products with the states give the queries and keys
        f4 of_g = {}, of_end = {};
        const f4 gamma = *(const f4*)(scalars + kGamma * kChunk + mine), left = *(const f4*)(scalars + kLeft * kChunk + mine);
        int at = again;
        auto finish = [&](auto which, bool turned) {
            constexpr int M = decltype(which)::value;
            auto operands = [&](int t, int s, b8 (&kb)[NX], b8 (&qb)[NX]) {
#pragma unroll
                for (int n = 0; n < NX; ++n) {
                    if constexpr (kKeepTransposed) {
                        kb[n] = kept_transposed[0][2 * t + s][at];
                        qb[n] = kept_transposed[1][2 * t + s][at];
                    } else {
                        kb[n] = operand(kt + n * kChunk * KD, 2, t, s, at);
                        qb[n] = operand(qt + n * kChunk * KD, 2, t, s, at);
                    }
                }
            };
            // the rows' steps, then the columns'
            auto pass = [&](bool turned, int s) {
                __builtin_amdgcn_sched_barrier(0);
                asm volatile("" : "+v"(at));       // (operands are loaded again rather than kept)
                b8 of_b[3], of_c[3];
                const auto& of = pool.squares.v[turned && kAtOnce];
#pragma unroll
                for (int m = 0; m < 3; ++m) {
                    of_b[m] = *(const b8*)&of[0][m][row][32 * s + 8 * (again >> 4)];
                    of_c[m] = *(const b8*)&of[1][m][row][32 * s + 8 * (again >> 4)];
                }
#pragma unroll
                for (int i = 0; i < KH; ++i) {
                    if (NX > 1) __builtin_amdgcn_sched_barrier(0);
                    b8 kb[NX], qb[NX];
                    operands(half * KH + i, s, kb, qb);
                    if (!turned && s == M) {
                        // (U's tile of these positions is a negative where the wavefront's number is odd)
                        const f4 of_dy = gamma * p.scale * (i & 1 ? -dq[i] : dq[i]), of_z = gamma * (i & 1 ? -zs[i] : zs[i]);
                        const f4 of_u = left * ((i ^ wave) & 1 ? -us[i] : us[i]);
                        // the entries of these positions' own keys and queries are a half of an operand
                        const f4 k = four_of(kb, wave & 1), q = four_of(qb, wave & 1);
                        of_g += q * of_dy - strength * (k * of_z);
                        of_strength -= k * of_z;
                        of_end += k * of_u;
                        dq_all[i] += of_dy;
                        dk_all[i] += of_u - strength * of_z;
                    }
                    if (turned) {
                        f4 more = {};
                        more = multiply<2>(of_b, qb, more);
                        dk_all[i] = multiply<2>(of_c, kb, dk_all[i]) + more;
                    } else {
                        dq_all[i] = multiply<2>(of_b, kb, dq_all[i]);
                        dk_all[i] = multiply<2>(of_c, kb, dk_all[i]);
                    }
                }
            };
            pass(turned, M);
            if (turned ? !M : M) pass(turned, 1 - M);
        };
        if (middle) finish(std::integral_constant<int, 1>(), false);
        else finish(std::integral_constant<int, 0>(), false);
        if constexpr (!kAtOnce) {
            lds_barrier();
            put_transposed();
            lds_barrier();
        }
        if (middle) finish(std::integral_constant<int, 1>(), true);
        else finish(std::integral_constant<int, 0>(), true);
        const double dg_sum = row_sums(of_h[0] + (double)of_g[0], of_h[1] + (double)of_g[1], of_h[2] + (double)of_g[2], of_h[3] + (double)of_g[3]);
        const float db_sum = row_sums(of_strength[0], of_strength[1], of_strength[2], of_strength[3]), end_sum = row_sums(of_end[0], of_end[1], of_end[2], of_end[3]);
        if ((again & 15) < 4) {
            rows_dg[half][mine + (again & 3)] = dg_sum;
            rows_db[half][mine + (again & 3)] = db_sum;
            rows_end[half][mine + (again & 3)] = end_sum;
        }
        zv = quad_sum(zv);
        if (!half && (again & 3) == 0) rows_zv[16 * wave + (again >> 2)] = zv;
        const double of_row = row_sums((double)both, 0.0, 0.0, 0.0);
        if ((again & 15) == 0) waves_end[4 * half + wave][again >> 4] = of_row;
        lds_barrier();
        if (!half && wave == 0) {
            // for the next kernel, which sums over positions: the share of a position, of what is left behind it, and of the whole chunk
            double dg = rows_dg[0][again] + rows_dg[1][again], end = 0.0;
#pragma unroll
            for (int m = 0; m < 8; ++m) {
                dg -= columns_dg[m][again];
#pragma unroll
                for (int i = 0; i < 4; ++i) end += waves_end[m][i];
            }
            double* out = w.gates + vc * kGates * kChunk;
            out[kGateRows * kChunk + again] = dg;
            out[kGateEnds * kChunk + again] = (double)rows_end[0][again] + (double)rows_end[1][again];
            out[kGateStrengths * kChunk + again] = (double)(rows_zv[again] + (rows_db[0][again] + rows_db[1][again]));
            out[kGateWhole * kChunk + again] = (double)scalars[kGamma * kChunk + kChunk - 1] * end;
        }
        // (the next head's operands are put where the squares lie behind a barrier of its own)
    }
    int out_lane = threadIdx.x & 63;
    asm volatile("" : "+v"(out_lane));
    float* parts = w.parts + (((size_t)b * p.value_heads + first_head) * shape.chunks + chunk) * 2 * kChunk * KD;
#pragma unroll
    for (int i = 0; i < KH; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int column = tile_row(half * KH + i, out_lane & 15), mine = tile_row(wave, 4 * (out_lane >> 4));
            if (shape.apart) {
                parts[(mine + e) * KD + column] = dq_all[i][e];
                parts[(kChunk + mine + e) * KD + column] = dk_all[i][e];
            } else if (mine + e < here && column < p.key_dim) {
                const long long at = ((at0 + mine + e) * p.key_heads + key_head) * p.key_dim + column;
                ((T*)a.dq)[at] = (T)(mine + e < rows ? dq_all[i][e] : 0.0f);
                ((T*)a.dk)[at] = (T)(mine + e < rows ? dk_all[i][e] : 0.0f);
            }
        }
}

// Where value heads are apart: dq and dk of a position, the sums over the value heads of a key head, in their order.
template <typename T>
__device__ __forceinline__ void sum_heads(const sys_gated_delta_t& p, const DeltaArgs& a, const DeltaShape& shape, const DeltaPlanes& w, int position)
{
    const int shared = p.value_heads / p.key_heads, b = position / p.length, t = position - b * p.length;
    const bool there = t < sequence_length(a.lengths, b, p.length);
    for (int i = threadIdx.x; i < p.key_heads * p.key_dim; i += kDeltaThreads) {
        const int key_head = i / p.key_dim, column = i - key_head * p.key_dim;
        float dq = 0.0f, dk = 0.0f;
        for (int h = 0; there && h < shared; ++h) {
            const size_t vc = ((size_t)b * p.value_heads + key_head * shared + h) * shape.chunks + t / kChunk;
            const float* from = w.parts + (vc * 2 * kChunk + t % kChunk) * shape.padded + column;
            dq += from[0];
            dk += from[kChunk * shape.padded];
        }
        const long long at = (long long)position * p.key_heads * p.key_dim + i;
        ((T*)a.dq)[at] = (T)dq;
        ((T*)a.dk)[at] = (T)dk;
    }
}

// Gradients of delta, beta and, a chunk each, of A and the bias: a wavefront a chunk of a value head, a lane a position.  The logarithm of a decay gets the gradients
// of the sums G that end in its position and behind it, what is left behind the positions before it, and what the whole chunk shares, in 64 bits.
template <typename T>
__global__ __launch_bounds__(kDeltaThreads) void delta_gates_kernel(sys_gated_delta_t p, DeltaArgs a, DeltaShape shape, DeltaPlanes w, long long all, int blocks)
{
    if ((int)blockIdx.x >= blocks) {               // (in the same launch: a workgroup a position)
        sum_heads<T>(p, a, shape, w, blockIdx.x - blocks);
        return;
    }
    const long long vc = (long long)blockIdx.x * (kDeltaThreads / 64) + (threadIdx.x >> 6);
    if (vc >= all) return;
    const int lane = threadIdx.x & 63, chunk = (int)(vc % shape.chunks), head = (int)(vc / shape.chunks % p.value_heads), b = (int)(vc / shape.chunks / p.value_heads);
    const int t0 = chunk * kChunk, rows = sequence_length(a.lengths, b, p.length) - t0;
    float of_a = 0.0f, of_bias = 0.0f, db = 0.0f;
    if (rows > 0) {
        const double* from = w.gates + vc * kGates * kChunk;
        const float* scalars = w.scalars + vc * kScalars * kChunk;
        const double own_end = from[kGateEnds * kChunk + lane];
        double dg = from[kGateRows * kChunk + lane], de = own_end;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const double behind = __shfl_down(dg, m), before = __shfl_up(de, m);
            if (lane + m < 64) dg += behind;
            if (lane >= m) de += before;
        }
        const float log_decay = (float)(dg + (de - own_end) + from[kGateWhole * kChunk + lane]);
        if (lane < rows) {
            of_a = scalars[kStep * kChunk + lane] * log_decay;
            of_bias = a.a[head] * log_decay * scalars[kSlope * kChunk + lane];
            db = (float)from[kGateStrengths * kChunk + lane];
            if (p.sigmoid) {
                // (1 - b is the sigmoid of -beta, and keeps its digits there)
                const float raw = (float)((const T*)a.beta)[b * p.beta_batch + (t0 + lane) * p.beta_row + head];
                db *= sigmoid(raw) * sigmoid(-raw);
            }
        }
    }
    if (t0 + lane < p.length) {
        const long long at = ((long long)b * p.length + t0 + lane) * p.value_heads + head;
        ((T*)a.ddelta)[at] = (T)of_bias;
        ((T*)a.dbeta)[at] = (T)db;
    }
    double sum_a = (double)of_a, sum_bias = (double)of_bias;
#pragma unroll
    for (int m = 32; m; m >>= 1) sum_a += __shfl_xor(sum_a, m), sum_bias += __shfl_xor(sum_bias, m);
    if (lane == 0) {
        w.shares[vc * 2] = sum_a;
        w.shares[vc * 2 + 1] = sum_bias;
    }
}

// The chunks' sums of a head, a workgroup a head, in 64 bits.
__global__ __launch_bounds__(kDeltaThreads) void delta_rates_kernel(sys_gated_delta_t p, DeltaArgs a, DeltaShape shape, DeltaPlanes w)
{
    const int head = blockIdx.x;
    const long long all = (long long)p.batch * shape.chunks;
    double of_a = 0.0, of_bias = 0.0;
    for (long long i = threadIdx.x; i < all; i += kDeltaThreads) {
        const long long b = i / shape.chunks;
        const double* from = w.shares + ((b * p.value_heads + head) * shape.chunks + (i - b * shape.chunks)) * 2;
        of_a += from[0];
        of_bias += from[1];
    }
#pragma unroll
    for (int m = 32; m; m >>= 1) of_a += __shfl_xor(of_a, m), of_bias += __shfl_xor(of_bias, m);
    __shared__ double waves[2][kDeltaThreads / 64];
    if ((threadIdx.x & 63) == 0) waves[0][threadIdx.x >> 6] = of_a, waves[1][threadIdx.x >> 6] = of_bias;
    __syncthreads();
    if (threadIdx.x) return;
    of_a = of_bias = 0.0;
#pragma unroll
    for (int i = 0; i < kDeltaThreads / 64; ++i) of_a += waves[0][i], of_bias += waves[1][i];
    a.da[head] = (float)of_a;
    if (a.ddelta_bias) a.ddelta_bias[head] = (float)of_bias;
}

template <typename T, int KD>
hipError_t run(const sys_gated_delta_t& p, const DeltaArgs& a, const DeltaShape& shape, const DeltaPlanes& w, hipStream_t s)
{
    DeltaShape of = shape;
    const bool wide = delta_wide(p);
    of.tiles = shape.columns / (wide ? 32 : 16);
    const long long sweeps = (long long)of.tiles * p.value_heads * p.batch, chunks = (long long)shape.chunks * (shape.apart ? p.value_heads : p.key_heads) * p.batch;
    if (sweeps > 0x7fffffffLL || chunks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    constexpr int kMost = sizeof(T) == 4 && KD > 64 ? 1 : 2;
    if (wide) hipLaunchKernelGGL((delta_back_kernel<T, KD, kMost>), dim3((unsigned)sweeps), dim3(kSweepThreads), 0, s, p, a, of, w);
    else hipLaunchKernelGGL((delta_back_kernel<T, KD, 1>), dim3((unsigned)sweeps), dim3(kSweepThreads), 0, s, p, a, of, w);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !chunks) return e;
    hipLaunchKernelGGL((delta_grad_kernel<T, KD>), dim3((unsigned)chunks), dim3(kGradThreads), 0, s, p, a, shape, w);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const long long all = (long long)shape.chunks * p.value_heads * p.batch, blocks = (all + kDeltaThreads / 64 - 1) / (kDeltaThreads / 64);
    const long long positions = shape.apart ? (long long)p.batch * p.length : 0;   // (of fewer chunks than CUs)
    hipLaunchKernelGGL(delta_gates_kernel<T>, dim3((unsigned)(blocks + positions)), dim3(kDeltaThreads), 0, s, p, a, shape, w, all, (int)blocks);
    return hipGetLastError();
}

template <typename T>
hipError_t run_type(const sys_gated_delta_t& p, const DeltaArgs& a, const DeltaShape& shape, const DeltaPlanes& w, hipStream_t s)
{
    return shape.padded == 64 ? run<T, 64>(p, a, shape, w, s) : run<T, 128>(p, a, shape, w, s);
}

}  // namespace

size_t delta_grad_workspace(const sys_gated_delta_t& p) { return p.length && p.batch ? delta_planes(p, delta_shape(p), true, nullptr, nullptr) : 0; }

hipError_t launch_delta_grad(const sys_gated_delta_t& p, const DeltaArgs& a, hipStream_t s)
{
    const DeltaShape shape = delta_shape(p, &a);
    DeltaPlanes w = {};
    if (p.batch) {
        if (p.length) delta_planes(p, shape, true, a.workspace, &w);
        hipError_t e = p.length ? launch_delta_matrices(p, a, shape, w, true, s) : hipSuccess;
        if (e == hipSuccess && p.length) e = launch_delta_sweep(p, a, shape, w, true, s);
        if (e != hipSuccess) return e;
        switch (p.dtype) {
        case SYS_F32: e = run_type<float>(p, a, shape, w, s); break;
        case SYS_F16: e = run_type<f16_t>(p, a, shape, w, s); break;
        default: e = run_type<bf16_t>(p, a, shape, w, s); break;
        }
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(delta_rates_kernel, dim3((unsigned)p.value_heads), dim3(kDeltaThreads), 0, s, p, a, shape, w);
    return hipGetLastError();
}

}  // namespace sysconv
