// Gated delta rule in chunks of 64 positions on the matrix cores (delta_tile.h has the formulas, the precision and the layout).
//
// Two launches.  The first makes X, P and K^T of all chunks side by side, a workgroup a chunk of a value head.  The second goes through the chunks: a workgroup
// a tile of value columns, the state in the registers of four wavefronts (wavefront w the rows of step w of the keys), S, R and U handed round as bf16
// parts through LDS with three barriers a chunk; operands that do not depend on the state are loaded a chunk ahead.  Four more wavefronts take S and U from LDS
// and make the outputs of them (or store them for the gradients) in what time the barriers leave.
//
// 4096 positions of 16 key heads and 32 value heads of 128 in bf16, 8400 us as torch operators: 132 us (43 + 98 by the profiler).  The first launch moves 162 MB at 3.8 TB/s, three workgroups
// a CU that load, work and store in turn; each operand that is not stored (the quarter of X and P that is 0) is time.  The second is a chain: 64 chunks of 2900 clocks, 870 + 960 + 820 for the three
// products and 300 at their barriers, with 590 of matrix instructions in each of the four wavefronts of the chain and 450 beside them.  What is left in a
// phase is reading and writing LDS and the latency of an instruction after the other; U from U and S of the chunk before, one exchange a chunk, would need
// two more matrices a chunk of the first launch.  With one group of wavefronts for everything the sweep took 107 us for 16 columns (the outputs in the chain's way).
#include "delta_tile.h"
#include "launch.h"

#include <initializer_list>

namespace sysconv {
namespace {

// ---------------------------------------------------------------- the chunks' matrices

template <typename T, int KD, bool GRAD>
__global__ __launch_bounds__(kDeltaThreads) void delta_matrices_kernel(sys_gated_delta_t p, DeltaArgs a, DeltaShape shape, DeltaPlanes w)
{
    constexpr int NX = kInputParts<T>, KS = KD / 32, kPitch = KD + 8, kSide = kChunk + 4;
    const int chunk = blockIdx.x % shape.chunks, rest = blockIdx.x / shape.chunks, head = rest % p.value_heads, b = rest / p.value_heads;
    const int shared = p.value_heads / p.key_heads, key_head = head / shared;
    const bool first = head % shared == 0;         // of the value heads of a key head: it writes what they have in common
    const int t0 = chunk * kChunk, last = sequence_length(a.lengths, b, p.length), rows = last - t0;
    if (rows <= 0) return;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 15, g = lane >> 4;
    const size_t vc = ((size_t)b * p.value_heads + head) * shape.chunks + chunk, kc = ((size_t)b * p.key_heads + key_head) * shape.chunks + chunk;

    // X is put where the keys lay
    __shared__ __attribute__((aligned(16))) union Pool {
        bf16_t keys[NX][kChunk][kPitch];
        float x[kChunk][kSide];
        __device__ Pool() {}
    } pool;
    auto& keys = pool.keys;
    auto& xm = pool.x;
    __shared__ __attribute__((aligned(16))) float am[kChunk][kSide];
    __shared__ double sums[kChunk];                // of the logarithms of the decays, to base 2
    __shared__ float strengths[kChunk];

    // what the first wavefront makes the decays of, K into LDS, and the rows of Q that this wavefront works on, as operands have them
    constexpr int kPieces = kChunk * KD / 8 / kDeltaThreads;
    b8 qa[KS][NX];
    float raw_delta = 0.0f, raw_beta = 0.0f, bias = 0.0f, rate = 0.0f;
    {
        if (wave == 0 && lane < rows) {
            raw_delta = (float)((const T*)a.delta)[b * p.delta_batch + (t0 + lane) * p.delta_row + head];
            raw_beta = (float)((const T*)a.beta)[b * p.beta_batch + (t0 + lane) * p.beta_row + head];
        }
        if (wave == 0) rate = a.a[head], bias = a.delta_bias ? a.delta_bias[head] : 0.0f;
        Eight<T> from_k[kPieces], from_q[KS];
        const ChunkRows<T> k_rows((const T*)a.k + b * p.k_batch + key_head * p.key_dim, p.k_row, p.key_dim, chunk, last);
        const ChunkRows<T> q_rows((const T*)a.q + b * p.q_batch + key_head * p.key_dim, p.q_row, p.key_dim, chunk, last);
        const __amdgpu_buffer_rsrc_t k_buffer = k_rows.buffer(), q_buffer = q_rows.buffer();
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int row = (tid + i * kDeltaThreads) / (KD / 8), at = (tid + i * kDeltaThreads) % (KD / 8) * 8;
            if (shape.whole) from_k[i].load(k_buffer, at < p.key_dim ? k_rows.place(row, at) : kNowhere);
            else from_k[i].load_each(k_buffer, k_rows.offset(row, at), row < rows ? p.key_dim - at : 0);
        }
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int row = tile_row(wave, r), at = 32 * s + 8 * g;
            if (shape.whole) from_q[s].load(q_buffer, at < p.key_dim ? q_rows.place(row, at) : kNowhere);
            else from_q[s].load_each(q_buffer, q_rows.offset(row, at), row < rows ? p.key_dim - at : 0);
        }
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int row = (tid + i * kDeltaThreads) / (KD / 8), at = (tid + i * kDeltaThreads) % (KD / 8) * 8;
            b8 parts[NX];
            from_k[i].split(parts);
#pragma unroll
            for (int n = 0; n < NX; ++n) *(b8*)&keys[n][row][at] = parts[n];
        }
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            from_q[s].split(qa[s]);
            if (first) {
#pragma unroll
                for (int n = 0; n < NX; ++n) *(b8*)(w.q + (kc * NX + n) * kChunk * KD + ((wave * KS + s) * 64 + lane) * 8) = qa[s][n];
            }
        }
    }
    lds_barrier();
    // (beside the other wavefronts' products, of which the first has the fewest)
    if (wave == 0) {
        // in 64 bits: what a step size is off by adds up over all positions that a state lives through, and a ratio of decays is the exponential of a small
        // difference of what may be large sums (with the step sizes of sequence.h, off by up to 8 2^-24, the gradients of A were off by 2e-6 of themselves
        // after 2048 positions, now 5e-7)
        double step = 0.0, strength = 0.0, slope = 0.0;
        if (lane < rows) {
            step = (double)raw_delta + (double)bias;
            strength = (double)raw_beta;
            slope = 1.0;
            if (p.softplus) {
                const double small = exp(-fabs(step)), large = step < 0.0 ? small : 1.0;
                slope = large / (1.0 + small);
                step = (step < 0.0 ? 0.0 : step) + log1p(small);       // (a NaN comes back with `small`)
            }
            if (p.sigmoid) strength = 1.0 / (1.0 + exp(-strength));
        }
        // a decay of 2^-10000 is 0 as any smaller one, and leaves the differences behind it their digits (NaN passes)
        double sum = step * (double)rate * 1.4426950408889634;
        sum = sum < -10000.0 ? -10000.0 : sum > 10000.0 ? 10000.0 : sum;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const double other = __shfl_up(sum, m);
            if (lane >= m) sum += other;
        }
        const double end = __shfl(sum, 63);
        sums[lane] = sum;
        strengths[lane] = (float)strength;
        float* out = w.scalars + vc * kScalars * kChunk;
        out[kGamma * kChunk + lane] = fast_exp2((float)sum);
        out[kLeft * kChunk + lane] = fast_exp2((float)(end - sum));
        out[kStrength * kChunk + lane] = (float)strength;
        if (GRAD) {
            out[kStep * kChunk + lane] = (float)step;
            out[kSlope * kChunk + lane] = (float)slope;
            ((double*)(out + kSums * kChunk))[lane] = sum;
        }
    }

    // A plane's pieces from LDS: K^T (Q^T), eight positions of a column; a square, or its transpose, without the quarter above (below) the diagonal
    auto transposed = [&](bf16_t* to) {
        for (int i = wave; i < KD / 16 * 2; i += kDeltaThreads / 64) {
            const int d = tile_row(i / 2, r), at = 32 * (i % 2) + 8 * g;
#pragma unroll
            for (int n = 0; n < NX; ++n) {
                b8 v;
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = keys[n][at + j][d];
                *(b8*)(to + (kc * NX + n) * kChunk * KD + (i * 64 + lane) * 8) = v;
            }
        }
    };
    auto square = [&](bf16_t* to, bool turned) {
        for (int i = wave; i < 8; i += kDeltaThreads / 64) {
            const int tile = i / 2, step = i % 2;
            if (turned ? step < tile / 2 : step > tile / 2) continue;
            const int row = tile_row(tile, r), at = 32 * step + 8 * g;
            float v[8];
            b8 parts[3];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = turned ? xm[at + j][row] : xm[row][at + j];
            split8(v, parts);
#pragma unroll
            for (int n = 0; n < 3; ++n) *(b8*)(to + n * kSquare + (i * 64 + lane) * 8) = parts[n];
        }
    };

    // K K^T, rows of this wavefront (as they lie), columns up to its own; and K Q^T, whose columns are the wavefront's queries (for gradients Q K^T, whose rows are)
    f4 kk[4] = {}, qk[4] = {};
    {
        b8 ka[KS][NX];
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int n = 0; n < NX; ++n) ka[s][n] = *(const b8*)&keys[n][16 * wave + r][32 * s + 8 * g];
#pragma unroll
        for (int n = 0; n < 4; ++n)
            if (n <= (wave | 1)) {
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    b8 kb[NX];
                    if (n <= wave) {
#pragma unroll
                        for (int m = 0; m < NX; ++m) kb[m] = *(const b8*)&keys[m][16 * n + r][32 * s + 8 * g];
                        kk[n] = multiply<2>(ka[s], kb, kk[n]);
                    }
#pragma unroll
                    for (int m = 0; m < NX; ++m) kb[m] = *(const b8*)&keys[m][tile_row(n, r)][32 * s + 8 * g];
                    qk[n] = GRAD ? multiply<2>(qa[s], kb, qk[n]) : multiply<2>(kb, qa[s], qk[n]);
                }
            }
    }
    lds_barrier();
    // A
    double row_sum[4];
    float row_strength[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) row_sum[e] = sums[16 * wave + 4 * g + e], row_strength[e] = strengths[16 * wave + 4 * g + e];
#pragma unroll
    for (int n = 0; n < 4; ++n)
        if (n <= wave) {
            const int column = 16 * n + r;
            const double column_sum = sums[column];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int row = 16 * wave + 4 * g + e;
                am[row][column] = column < row ? row_strength[e] * (fast_exp2((float)(row_sum[e] - column_sum)) * kk[n][e]) : 0.0f;
            }
        }
    // P, without the quarter above the diagonal, in the order of its operands as the products leave it: K Q^T, whose columns are queries, gives a lane eight keys of a
    // row of P in two tiles; for gradients Q K^T gives it four queries of a row of P^T, half an operand
    if constexpr (GRAD) {
        const int query = tile_row(wave, 4 * g);
        double query_sum[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) query_sum[e] = sums[query + e];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            if (n > (wave | 1)) break;
            const int key = tile_row(n, r);
            const double key_sum = sums[key];
            f4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = key <= query + e ? p.scale * (fast_exp2((float)(query_sum[e] - key_sum)) * qk[n][e]) : 0.0f;
            u2 parts[3];
            split4(v, parts);
#pragma unroll
            for (int m = 0; m < 3; ++m) *(u2*)(w.pt + (vc * 3 + m) * kSquare + ((2 * n + (wave >> 1)) * 64 + lane) * 8 + 4 * (wave & 1)) = parts[m];
        }
    } else {
        const int query = tile_row(wave, r);
        const double query_sum = sums[query];
#pragma unroll
        for (int step = 0; step < 2; ++step) {
            if (step > wave >> 1) break;
            float v[8];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = 32 * step + 8 * g + 4 * n + e;
                    v[4 * n + e] = key <= query ? p.scale * (fast_exp2((float)(query_sum - sums[key])) * qk[2 * step + n][e]) : 0.0f;
                }
            }
            b8 parts[3];
            split8(v, parts);
#pragma unroll
            for (int m = 0; m < 3; ++m) *(b8*)(w.p + (vc * 3 + m) * kSquare + ((2 * wave + step) * 64 + lane) * 8) = parts[m];
        }
    }
    if (first) {
        // K as it is and transposed, 1 KB a wavefront
        for (int i = wave; i < 4 * KS; i += kDeltaThreads / 64)
#pragma unroll
            for (int n = 0; n < NX; ++n)
                *(b8*)(w.k + (kc * NX + n) * kChunk * KD + (i * 64 + lane) * 8) = *(const b8*)&keys[n][tile_row(i / KS, r)][32 * (i % KS) + 8 * g];
        transposed(w.kt);
    }
    if (GRAD && first) {
        // Q^T the same way as K^T, through its place
        lds_barrier();
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int n = 0; n < NX; ++n) *(b8*)&keys[n][tile_row(wave, r)][32 * s + 8 * g] = qa[s][n];
        lds_barrier();
        transposed(w.qt);
    }

    // X: the 16 x 16 blocks on the diagonal by substitution, a column a lane (four times over) ...
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        x[i] = i == r ? 1.0f : 0.0f;
#pragma unroll
        for (int j = 0; j < i; ++j) x[i] = __builtin_fmaf(-am[16 * wave + i][16 * wave + j], x[j], x[i]);
    }
    lds_barrier();                               // (all are done with the keys)
    if (g == 0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) xm[16 * wave + i][16 * wave + r] = x[i];
    }
    lds_barrier();
    // ... and those below, X_ij = -X_ii (sum_k A_ik X_kj), a column of blocks a wavefront, in fp32
    f4 column[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) column[0][e] = xm[16 * wave + 4 * g + e][16 * wave + r];
#pragma unroll
    for (int d = 1; d < 4; ++d) {
        const int i = wave + d;
        if (i < 4) {
            f4 sum = {}, block = {};
#pragma unroll
            for (int m = 0; m < d; ++m) {
                const f4 v = *(const f4*)&am[16 * i + r][16 * (wave + m) + 4 * g];
#pragma unroll
                for (int e = 0; e < 4; ++e) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e], column[m][e], sum, 0, 0, 0);
            }
            const f4 v = *(const f4*)&xm[16 * i + r][16 * i + 4 * g];
#pragma unroll
            for (int e = 0; e < 4; ++e) block = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e], sum[e], block, 0, 0, 0);
            column[d] = -block;
        }
    }
#pragma unroll
    for (int d = 1; d < 4; ++d)
        if (wave + d < 4) {
#pragma unroll
            for (int e = 0; e < 4; ++e) xm[16 * (wave + d) + 4 * g + e][16 * wave + r] = column[d][e];
        }
    for (int i = 0; i < wave; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) xm[16 * i + 4 * g + e][16 * wave + r] = 0.0f;
    lds_barrier();
    square(w.x + vc * 3 * kSquare, false);
    if (GRAD) square(w.xt + vc * 3 * kSquare, true);
}

// ---------------------------------------------------------------- the sweep

template <typename T, int KD, int NT, bool GRAD>
__global__ __launch_bounds__(kSweepThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void delta_sweep_kernel(sys_gated_delta_t p, DeltaArgs a, DeltaShape shape, DeltaPlanes w)
{
    constexpr int NX = kInputParts<T>, KS = KD / 32, TW = KD / 64;
    constexpr bool kAtOnce = NX * NT <= 2;         // there are registers for all operands of a product
    const unsigned place = xcd_place(blockIdx.x, gridDim.x);
    const int tile = place % shape.tiles, rest = place / shape.tiles, head = rest % p.value_heads, b = rest / p.value_heads;
    const int key_head = head / (p.value_heads / p.key_heads);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) & 3, lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const bool chain = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8) == 0;
    const int last = sequence_length(a.lengths, b, p.length), chunks = (last + kChunk - 1) / kChunk;
    const int steps = (wave >> 1) + 1;             // of X and P: what lies above their diagonals is zero
    const int my_row = tile_row(wave, 4 * g);      // the first of this lane's four positions
    int column[NT];
    bool there[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) column[n] = (tile * NT + n) * 16 + r, there[n] = column[n] < p.value_dim;

    __shared__ Operands<KS, 3, NT> states;
    __shared__ Operands<2, 3, NT> misses, writes, values;

    const size_t vc = ((size_t)b * p.value_heads + head) * shape.chunks, kc = ((size_t)b * p.key_heads + key_head) * shape.chunks;
    // (loads come back in their order: they are made in the order of their use, a chunk ahead, each kind when the one before it has been used up)
    if (chain) {
        const size_t state_base = ((size_t)b * p.value_heads + head) * p.key_dim * p.value_dim;
        const unsigned state_bytes = (unsigned)(p.key_dim * p.value_dim) * 4u;
        f4 s[TW][NT];
        {
            const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc((void*)(a.state + state_base), 0, a.state ? state_bytes : 0u, 0x00027000);
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
        ChunkRows<T> v((const T*)a.v + b * p.v_batch + head * p.value_dim, p.v_row, p.value_dim, 0, last);
        unsigned v_at[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) v_at[n][e] = there[n] ? v.offset(my_row + e, column[n]) : kNowhere;
        b8 ka[KS][NX], kta[TW][2][NX], xa[2][3];
        unsigned next_v[NT][4];
        f4 next_gamma, next_left, next_strength;
        float next_end;
        auto fetch_keys = [&](int c) {
#pragma unroll
            for (int i = 0; i < KS; ++i)
#pragma unroll
                for (int n = 0; n < NX; ++n) ka[i][n] = operand(w.k + ((kc + c) * NX + n) * kChunk * KD, KS, wave, i, lane);
        };
        auto fetch_values = [&](int c) {
            const __amdgpu_buffer_rsrc_t rows = v.buffer();
            if (v.exist < kChunk) {                // (the last chunk: what does not exist there does not behind it)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v_at[n][e] = my_row + e < v.exist ? v_at[n][e] : kNowhere;
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) next_v[n][e] = buffer_load<T>(rows, v_at[n][e]);
            v.move(1);
            const float* from = w.scalars + (vc + c) * kScalars * kChunk;
            next_gamma = *(const f4*)(from + kGamma * kChunk + my_row);
            next_left = *(const f4*)(from + kLeft * kChunk + my_row);
            next_strength = *(const f4*)(from + kStrength * kChunk + my_row);
            next_end = from[kGamma * kChunk + kChunk - 1];
        };
        auto fetch_inverse = [&](int c) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (i < steps) {
#pragma unroll
                    for (int n = 0; n < 3; ++n) xa[i][n] = operand(w.x + ((vc + c) * 3 + n) * kSquare, 2, wave, i, lane);
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
            fetch_keys(0), fetch_values(0), fetch_inverse(0), fetch_transposed(0);
            put_state();
        }
        for (int c = 0; c < chunks; ++c) {
            const int next = c + 1 < chunks ? c + 1 : c;
            lds_barrier();
            // K S, and of it b (V - e^G (K S))
            f4 ks[NT][3] = {};
            {
                b8 parts[KS][NT][3];
#pragma unroll
                for (int i = 0; i < KS; ++i)
#pragma unroll
                    for (int n = 0; n < NT; ++n) states.take(i, n, lane, parts[i][n]);
                if (kAtOnce) __builtin_amdgcn_sched_barrier(0);        // (or they are read one by one, and each is waited for)
#pragma unroll
                for (int i = 0; i < KS; ++i)
#pragma unroll
                    for (int n = 0; n < NT; ++n) multiply_apart<2>(ka[i], parts[i][n], ks[n]);
            }
            fetch_keys(next);
            const f4 gamma = next_gamma, left = next_left, strength = next_strength;
            const float end = next_end;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const f4 sum = joined(ks[n]);
                f4 miss;
#pragma unroll
                for (int e = 0; e < 4; ++e) miss[e] = strength[e] * __builtin_fmaf(-gamma[e], sum[e], loaded<T>(next_v[n][e]));
                misses.put_half(wave, n, lane, miss);
            }
            fetch_values(next);                    // (past the last chunk: zeros that nobody takes)
            lds_barrier();
            // U
            f4 u[NT][3] = {};
            {
                b8 parts[2][NT][3];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int n = 0; n < NT; ++n) misses.take(i, n, lane, parts[i][n]);
                if (kAtOnce) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (i < steps) {
#pragma unroll
                        for (int n = 0; n < NT; ++n) multiply_apart<2>(xa[i], parts[i][n], u[n]);
                    }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const f4 sum = joined(u[n]);
                writes.put_half(wave, n, lane, left * sum);
                values.put_half(wave, n, lane, sum);
            }
            fetch_inverse(next);
            lds_barrier();
            // the state behind the chunk
            {
                b8 parts[2][NT][3];
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int n = 0; n < NT; ++n) writes.take(m, n, lane, parts[m][n]);
                if (kAtOnce) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    f4 more[TW][3] = {};
#pragma unroll
                    for (int i = 0; i < TW; ++i) more[i][0] = s[i][n] * end;
#pragma unroll
                    for (int m = 0; m < 2; ++m)
#pragma unroll
                        for (int i = 0; i < TW; ++i) multiply_apart<2>(kta[i][m], parts[m][n], more[i]);
#pragma unroll
                    for (int i = 0; i < TW; ++i) s[i][n] = joined(more[i]);
                }
            }
            put_state();
            fetch_transposed(next);
        }
        if (!GRAD && a.state_out) {
            const __amdgpu_buffer_rsrc_t to = __builtin_amdgcn_make_buffer_rsrc((void*)(a.state_out + state_base), 0, state_bytes, 0x00027000);
#pragma unroll
            for (int i = 0; i < TW; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const unsigned row = tile_row(TW * wave + i, 4 * g) + e;
                        const float value = s[i][n][e];    // (an element of a vector is not a place that bits can be taken from)
                        __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, value), to, there[n] ? (row * p.value_dim + column[n]) * 4u : kNowhere, 0, 0);
                    }
        }
    } else if (GRAD) {
        // what the gradients need of it: S before the chunk, and U.  (From wavefronts of their own: loads that were made behind stores wait for them.)
        auto store_state = [&](int c, int i) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const f4 of_s = turn_quad(signed_rows(states.numbers(TW * wave + i, n, lane), TW * wave + i));
                *(f4*)(w.s + block_place(vc + c, KD, shape.columns, tile_row(TW * wave + i, 4 * g) + (r & 3), (tile * NT + n) * 16 + (r & ~3))) = of_s;
            }
        };
        auto store_u = [&](int c) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const f4 u = turn_quad(signed_rows(values.numbers(wave, n, lane), wave));
                *(f4*)(w.u + block_place(vc + c, kChunk, shape.columns, my_row + (r & 3), (tile * NT + n) * 16 + (r & ~3))) = u;
            }
        };
        for (int c = 0; c < chunks; ++c) {
            // (the state stays as it is to the third barrier, U to the second of the next chunk: nobody waits for this)
            lds_barrier();
            if (c) store_u(c - 1);
            if (TW == 1) store_state(c, 0);
            lds_barrier();
            if (TW == 2) store_state(c, 0), store_state(c, 1);
            lds_barrier();
        }
        if (chunks > 0) store_u(chunks - 1);
    } else {
        // the outputs
        ChunkRows<T> y((const T*)a.y + b * p.y_batch + head * p.value_dim, p.y_row, p.value_dim, 0, p.length);
        unsigned y_at[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) y_at[n][e] = there[n] ? y.offset(my_row + e, column[n]) : kNowhere;
        b8 qa[KS][NX], pa[2][3];
        f4 next_gamma;
        auto fetch_queries = [&](int c) {
#pragma unroll
            for (int i = 0; i < KS; ++i)
#pragma unroll
                for (int n = 0; n < NX; ++n) qa[i][n] = operand(w.q + ((kc + c) * NX + n) * kChunk * KD, KS, wave, i, lane);
            next_gamma = *(const f4*)(w.scalars + (vc + c) * kScalars * kChunk + kGamma * kChunk + my_row);
        };
        auto fetch_mixed = [&](int c) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (i < steps) {
#pragma unroll
                    for (int n = 0; n < 3; ++n) pa[i][n] = operand(w.p + ((vc + c) * 3 + n) * kSquare, 2, wave, i, lane);
                }
        };
        if (chunks > 0) fetch_queries(0), fetch_mixed(0);
        f4 out[NT] = {}, done[NT];
        auto of_state = [&](int i) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                b8 parts[3];
                states.take(i, n, lane, parts);
                out[n] = multiply<2>(qa[i], parts, out[n]);
            }
        };
        auto store = [&](int c) {
            const __amdgpu_buffer_rsrc_t rows = y.buffer();
            const int left = last - c * kChunk - my_row;               // (behind the sequence 0, also where the state is not finite)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) buffer_store<T>(rows, y_at[n][e], (T)(e < left ? done[n][e] : 0.0f));
            y.move(1);
        };
        for (int c = 0; c < chunks; ++c) {
            const int next = c + 1 < chunks ? c + 1 : c;
            // (the state stays as it is to the third barrier, U to the second of the next chunk: the work is spread so that the other four never wait for it)
            lds_barrier();
            if (c) store(c - 1);
#pragma unroll
            for (int i = 0; i < KS / 2; ++i) of_state(i);
            lds_barrier();
#pragma unroll
            for (int i = KS / 2; i < KS; ++i) of_state(i);
            const f4 gamma = next_gamma * p.scale;
            fetch_queries(next);
            lds_barrier();
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                f4 o = out[n] * gamma;
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (i < steps) {
                        b8 parts[3];
                        values.take(i, n, lane, parts);
                        o = multiply<2>(pa[i], parts, o);
                    }
                done[n] = o;
                out[n] = f4{};
            }
            fetch_mixed(next);
        }
        if (chunks > 0) store(chunks - 1);
        T* behind = (T*)a.y + b * p.y_batch + head * p.value_dim;
        for (int t = chunks * kChunk + (int)((threadIdx.x & 255) >> 4); t < p.length; t += kSweepThreads / 32)
#pragma unroll
            for (int n = 0; n < NT; ++n)
                if (there[n]) behind[t * p.y_row + column[n]] = (T)0.0f;
    }
}

template <typename T, int KD, bool GRAD>
hipError_t matrices(const sys_gated_delta_t& p, const DeltaArgs& a, const DeltaShape& shape, const DeltaPlanes& w, hipStream_t s)
{
    const long long blocks = (long long)shape.chunks * p.value_heads * p.batch;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    if (blocks) hipLaunchKernelGGL((delta_matrices_kernel<T, KD, GRAD>), dim3((unsigned)blocks), dim3(kDeltaThreads), 0, s, p, a, shape, w);
    return hipGetLastError();
}

template <typename T, int KD, bool GRAD>
hipError_t sweep(const sys_gated_delta_t& p, const DeltaArgs& a, const DeltaShape& shape, const DeltaPlanes& w, hipStream_t s)
{
    DeltaShape of = shape;
    const bool wide = delta_wide(p);
    of.tiles = wide ? shape.columns / 32 : GRAD ? shape.columns / 16 : (p.value_dim + 15) / 16;
    const long long blocks = (long long)of.tiles * p.value_heads * p.batch;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    constexpr int kMost = sizeof(T) == 4 && KD > 64 ? 1 : 2;
    if (wide) hipLaunchKernelGGL((delta_sweep_kernel<T, KD, kMost, GRAD>), dim3((unsigned)blocks), dim3(kSweepThreads), 0, s, p, a, of, w);
    else hipLaunchKernelGGL((delta_sweep_kernel<T, KD, 1, GRAD>), dim3((unsigned)blocks), dim3(kSweepThreads), 0, s, p, a, of, w);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_type(bool is_sweep, const sys_gated_delta_t& p, const DeltaArgs& a, const DeltaShape& shape, const DeltaPlanes& w, bool grad, hipStream_t s)
{
    auto run = [&](auto kd, auto g) {
        constexpr int KD = decltype(kd)::value;
        constexpr bool GRAD = decltype(g)::value;
        return is_sweep ? sweep<T, KD, GRAD>(p, a, shape, w, s) : matrices<T, KD, GRAD>(p, a, shape, w, s);
    };
    auto wide = [&](auto g) { return shape.padded == 64 ? run(std::integral_constant<int, 64>(), g) : run(std::integral_constant<int, 128>(), g); };
    return grad ? wide(std::true_type()) : wide(std::false_type());
}

hipError_t launch(bool is_sweep, const sys_gated_delta_t& p, const DeltaArgs& a, const DeltaShape& shape, const DeltaPlanes& w, bool grad, hipStream_t s)
{
    switch (p.dtype) {
    case SYS_F32: return launch_type<float>(is_sweep, p, a, shape, w, grad, s);
    case SYS_F16: return launch_type<f16_t>(is_sweep, p, a, shape, w, grad, s);
    default: return launch_type<bf16_t>(is_sweep, p, a, shape, w, grad, s);
    }
}

// Whether sequences are so short that they go a position at a time, which takes 2 us a position and hardly goes by the state's size, while a chunk's two launches take
// longer where inputs have more parts.  Us a position at a time and in chunks: one sequence of 32 heads of 128 x 128 in bf16 10 positions 14.9 and 14.2 (8: 12.5 and 14.1, 12:
// 17.2 and 14.3), in fp16 12 positions 17.1 and 16.5 (14: 19.4 and 16.8), in fp32 16.3 and 19.1 (14: 18.4 and 19.1); of eight heads of 64 x 64 in bf16 10 positions 12.3 and
// 12.2, in fp16 12 positions 14.2 and 13.0, in fp32 13.8 and 14.1.  Where there are more heads than CUs the chunks' matrices take longer: 20 positions of 8 sequences of 32 heads of
// 128 x 128 in bf16 32.7 and 35.2 (24: 37.8 and 35.2), of 32 sequences of eight heads of 64 x 64 22.9 and 24.4 (24: 26.7 and 24.5), of 64 sequences of 32 heads 170 and 202 (24: 200 and 203).
bool delta_short(const sys_gated_delta_t& p)
{
    return p.length <= ((long long)p.batch * p.value_heads >= kCus ? 20 : p.dtype == SYS_BF16 ? 10 : 12);
}

}  // namespace

hipError_t launch_delta_matrices(const sys_gated_delta_t& p, const DeltaArgs& a, const DeltaShape& shape, const DeltaPlanes& w, bool grad, hipStream_t s)
{
    return launch(false, p, a, shape, w, grad, s);
}
hipError_t launch_delta_sweep(const sys_gated_delta_t& p, const DeltaArgs& a, const DeltaShape& shape, const DeltaPlanes& w, bool grad, hipStream_t s)
{
    return launch(true, p, a, shape, w, grad, s);
}

bool delta_wide(const sys_gated_delta_t& p)
{
    // 32 columns a workgroup where 16 would be more workgroups than CUs: half the operands' loads.  1024 positions in bf16, 16 columns and 32: 32 heads of 128 x 128 43 us and
    // 57, 34 heads 63 and 57, 64 heads 66 and 61 (gradients 273 and 251); eight heads of 64 x 128 of five sequences in fp16 57 and 50
    // (keys of more than 64 entries in fp32, three parts each, take all registers with 16 columns)
    return !(p.dtype == SYS_F32 && p.key_dim > 64) && (long long)((p.value_dim + 15) / 16) * p.value_heads * p.batch > kCus;
}

DeltaShape delta_shape(const sys_gated_delta_t& p, const DeltaArgs* a)
{
    DeltaShape s = {};
    // whole pieces of eight entries, at addresses that are multiples of four
    const size_t element = p.dtype == SYS_F32 ? 4 : 2;
    s.whole = a && p.key_dim % 8 == 0 && (uintptr_t)a->q % 4 == 0 && (uintptr_t)a->k % 4 == 0;
    for (long long stride : {p.q_batch, p.q_row, p.k_batch, p.k_row})
        if (stride * element % 4) s.whole = 0;
    s.whole_values = a && p.value_dim % 8 == 0 && (uintptr_t)a->v % 4 == 0 && (uintptr_t)a->dy % 4 == 0;
    for (long long stride : {p.v_batch, p.v_row, p.y_batch, p.y_row})
        if (stride * element % 4) s.whole_values = 0;
    s.chunks = delta_chunks(p);
    s.padded = delta_padded(p);
    s.columns = (p.value_dim + 31) / 32 * 32;
    // where that leaves half of the CUs or more without a workgroup: 24 chunks of key heads with two value heads of 64 x 100 each in fp32 take 24 us apart, and 4 for
    // the join of their sums, against 41 one after the other; from half of the CUs on there are no fewer rounds of workgroups to win
    s.apart = p.value_heads > p.key_heads && 2 * (long long)s.chunks * p.key_heads * p.batch <= kCus;
    return s;
}

size_t delta_planes(const sys_gated_delta_t& p, const DeltaShape& shape, bool grad, void* base, DeltaPlanes* w)
{
    const size_t value_chunks = (size_t)p.batch * p.value_heads * shape.chunks, key_chunks = (size_t)p.batch * p.key_heads * shape.chunks;
    const size_t input = p.dtype == SYS_F32 ? 3 : p.dtype == SYS_F16 ? 2 : 1;
    const size_t keys = key_chunks * input * kChunk * shape.padded * sizeof(bf16_t), square = value_chunks * kSquare * sizeof(bf16_t);
    const size_t begin = ((uintptr_t)base + 255) / 256 * 256;
    size_t at = begin;
    auto take = [&](auto*& to, size_t bytes) {
        to = (std::remove_reference_t<decltype(to)>)at;
        at += (bytes + 255) / 256 * 256;
    };
    DeltaPlanes of = {};
    take(of.x, 3 * square);
    take(of.k, keys);
    take(of.q, keys);
    take(of.kt, keys);
    take(of.scalars, value_chunks * kScalars * kChunk * sizeof(float));
    if (!grad) {
        take(of.p, 3 * square);
    } else {
        take(of.xt, 3 * square);
        take(of.pt, 3 * square);
        take(of.qt, keys);
        const size_t state = value_chunks * shape.padded * shape.columns * sizeof(float), rows = value_chunks * kChunk * shape.columns * sizeof(float);
        take(of.s, state);
        take(of.ds, state);
        take(of.u, rows);
        take(of.z, rows);
        if (shape.apart) take(of.parts, 2 * value_chunks * kChunk * shape.padded * sizeof(float));
        take(of.gates, value_chunks * kGates * kChunk * sizeof(double));
        take(of.shares, 2 * value_chunks * sizeof(double));
    }
    if (w) *w = of;
    return at - begin + 256;                       // (the base may lie anywhere)
}

size_t delta_workspace(const sys_gated_delta_t& p)
{
    return !delta_short(p) && p.batch ? delta_planes(p, delta_shape(p), false, nullptr, nullptr) : 0;
}

hipError_t launch_delta(const sys_gated_delta_t& p, const DeltaArgs& a, hipStream_t s)
{
    if (delta_short(p)) return launch_delta_positions(p, a, s);
    const DeltaShape shape = delta_shape(p, &a);
    DeltaPlanes w;
    delta_planes(p, shape, false, a.workspace, &w);
    const hipError_t e = launch_delta_matrices(p, a, shape, w, false, s);
    return e != hipSuccess ? e : launch_delta_sweep(p, a, shape, w, false, s);
}

}  // namespace sysconv
