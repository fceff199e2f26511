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
//   H_ij = B_ij q_i . k_j + b_i C_ij k_i . k_j  (j < i)  they are the row's sum less the column's, of the same numbers,
// and what else there is comes from the products with the states: q_i . (e^G S dO)_i + b_i k_i . (-e^G S Z)_i from the position on, E_i k_i . (dS' U_i) up
// to it, e^(G_end) <S, dS'> for all; sums over the positions of a chunk are in 64 bits.
#include "delta_tile.h"
#include "launch.h"

namespace sysconv {
namespace {

template <typename T, int KD>
__global__ __launch_bounds__(kDeltaThreads) void delta_back_kernel(sys_gated_delta_t p, DeltaArgs a, DeltaShape shape, DeltaPlanes w)
{
    constexpr int NX = kInputParts<T>, KS = KD / 32, TW = KD / 64, RP = kResultParts<T>;
    const unsigned place = xcd_place(blockIdx.x, gridDim.x);
    const int tile = place % shape.tiles, rest = place / shape.tiles, head = rest % p.value_heads, b = rest / p.value_heads;
    const int key_head = head / (p.value_heads / p.key_heads);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int last = sequence_length(a.lengths, b, p.length), chunks = (last + kChunk - 1) / kChunk;
    const int first_step = wave >> 1;              // of X^T and P^T: what lies below their diagonals is zero
    const int my_row = tile_row(wave, 4 * g);
    const int column = tile * 16 + r;
    const bool there = column < p.value_dim;

    __shared__ Operands<KS, 3, 1> states;
    __shared__ Operands<2, 3, 1> misses, writes, weighted;
    __shared__ Operands<2, NX, 1> outs;

    const size_t state_base = ((size_t)b * p.value_heads + head) * p.key_dim * p.value_dim;
    const unsigned state_bytes = (unsigned)(p.key_dim * p.value_dim) * 4u;
    f4 s[TW];
    {
        const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc((void*)(a.dstate_out + state_base), 0, a.dstate_out ? state_bytes : 0u, 0x00027000);
#pragma unroll
        for (int i = 0; i < TW; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned row = tile_row(TW * wave + i, 4 * g) + e;
                s[i][e] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(from, there ? (row * p.value_dim + column) * 4u : kNowhere, 0, 0));
            }
    }
    auto put_state = [&] {
        if constexpr (TW == 2) states.put(wave, 0, lane, s[0], s[1]);
        else states.put_half(wave, 0, lane, s[0]);
    };
    const int top = chunks > 0 ? chunks - 1 : 0;
    const long long dv_row = (long long)p.value_heads * p.value_dim;
    ChunkRows<T> dy((const T*)a.dy + b * p.y_batch + head * p.value_dim, p.y_row, p.value_dim, top, last);
    ChunkRows<T> dv((const T*)a.dv + (long long)b * p.length * dv_row + head * p.value_dim, dv_row, p.value_dim, top, p.length);
    unsigned dy_at[4], dv_at[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        dy_at[e] = there ? dy.offset(my_row + e, column) : kNowhere;
        dv_at[e] = there ? dv.offset(my_row + e, column) : kNowhere;
    }
    const size_t vc = ((size_t)b * p.value_heads + head) * shape.chunks, kc = ((size_t)b * p.key_heads + key_head) * shape.chunks;

    b8 ka[KS][NX], kta[TW][2][NX], qta[TW][2][NX], xa[2][3], pa[2][3];
    unsigned next_dy[4];
    f4 gamma, left, strength, own_dy;
    float end;
    auto fetch_keys = [&](int c) {
#pragma unroll
        for (int i = 0; i < KS; ++i)
#pragma unroll
            for (int n = 0; n < NX; ++n) ka[i][n] = operand(w.k + ((kc + c) * NX + n) * kChunk * KD, KS, wave, i, lane);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (i >= first_step) {
#pragma unroll
                for (int n = 0; n < 3; ++n) pa[i][n] = operand(w.pt + ((vc + c) * 3 + n) * kSquare, 2, wave, i, lane);
            }
    };
    auto fetch_outs = [&] {
        const __amdgpu_buffer_rsrc_t rows = dy.buffer();
#pragma unroll
        for (int e = 0; e < 4; ++e) next_dy[e] = buffer_load<T>(rows, dy_at[e]);
        dy.move(-1);
    };
    auto put_outs = [&] {
#pragma unroll
        for (int e = 0; e < 4; ++e) own_dy[e] = loaded<T>(next_dy[e]);
        outs.put_half(wave, 0, lane, own_dy);
    };
    auto fetch_inverse = [&](int c) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (i >= first_step) {
#pragma unroll
                for (int n = 0; n < 3; ++n) xa[i][n] = operand(w.xt + ((vc + c) * 3 + n) * kSquare, 2, wave, i, lane);
            }
    };
    auto fetch_rest = [&](int c) {
#pragma unroll
        for (int i = 0; i < TW; ++i)
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int n = 0; n < NX; ++n) {
                    kta[i][m][n] = operand(w.kt + ((kc + c) * NX + n) * kChunk * KD, 2, TW * wave + i, m, lane);
                    qta[i][m][n] = operand(w.qt + ((kc + c) * NX + n) * kChunk * KD, 2, TW * wave + i, m, lane);
                }
        const float* from = w.scalars + (vc + c) * kScalars * kChunk;
        gamma = *(const f4*)(from + kGamma * kChunk + my_row);
        left = *(const f4*)(from + kLeft * kChunk + my_row);
        strength = *(const f4*)(from + kStrength * kChunk + my_row);
        end = from[kGamma * kChunk + kChunk - 1];
    };
    if (chunks > 0) {
        fetch_outs(), fetch_keys(top), fetch_inverse(top), fetch_rest(top);
        put_state();
        put_outs();
    }
    for (int c = top; c >= 0 && chunks > 0; --c) {
        const int next = c > 0 ? c - 1 : 0;
        lds_barrier();
        if (c > 0) fetch_outs();
        {
            // dS behind the chunk
#pragma unroll
            for (int i = 0; i < TW; ++i) {
                u2 parts[RP];
                split4(s[i], parts);
#pragma unroll
                for (int m = 0; m < RP; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        w.ds[(((vc + c) * RP + m) * KD + tile_row(TW * wave + i, 4 * g) + e) * shape.columns + column] = as_bf16(parts[m][e / 2] >> 16 * (e & 1));
            }
        }
        // dU
        f4 ks = {}, u = {};
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            b8 parts[3];
            states.take(i, 0, lane, parts);
            ks = multiply<2>(ka[i], parts, ks);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (i >= first_step) {
                b8 parts[NX];
                outs.take(i, 0, lane, parts);
                u = multiply<2>(pa[i], parts, u);
            }
        fetch_keys(next);
        misses.put_half(wave, 0, lane, u + left * ks);
        lds_barrier();
        // Z
        f4 z = {};
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (i >= first_step) {
                b8 parts[3];
                misses.take(i, 0, lane, parts);
                z = multiply<2>(xa[i], parts, z);
            }
        const f4 values = strength * z;
        writes.put_half(wave, 0, lane, -(gamma * values));
        weighted.put_half(wave, 0, lane, gamma * p.scale * own_dy);
        {
            const __amdgpu_buffer_rsrc_t rows = dv.buffer();
            u2 parts[RP];
            split4(z, parts);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                buffer_store<T>(rows, dv_at[e], (T)values[e]);
#pragma unroll
                for (int m = 0; m < RP; ++m)
                    w.z[(((vc + c) * RP + m) * kChunk + my_row + e) * shape.columns + column] = as_bf16(parts[m][e / 2] >> 16 * (e & 1));
            }
            dv.move(-1);
        }
        fetch_inverse(next);
        lds_barrier();
#pragma unroll
        for (int i = 0; i < TW; ++i) s[i] *= end;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            b8 of_z[3], of_dy[3];
            writes.take(m, 0, lane, of_z);
            weighted.take(m, 0, lane, of_dy);
#pragma unroll
            for (int i = 0; i < TW; ++i) {
                s[i] = multiply<2>(kta[i][m], of_z, s[i]);
                s[i] = multiply<2>(qta[i][m], of_dy, s[i]);
            }
        }
        put_state();
        if (c > 0) put_outs();
        fetch_rest(next);
    }
    T* behind = (T*)a.dv + (long long)b * p.length * dv_row + head * p.value_dim;
    for (int t = chunks * kChunk + (threadIdx.x >> 4); t < p.length; t += kDeltaThreads / 16)
        if (there) behind[t * dv_row + column] = (T)0.0f;
    if (a.dstate) {
        const __amdgpu_buffer_rsrc_t to = __builtin_amdgcn_make_buffer_rsrc((void*)(a.dstate + state_base), 0, state_bytes, 0x00027000);
#pragma unroll
        for (int i = 0; i < TW; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned row = tile_row(TW * wave + i, 4 * g) + e;
                const float value = s[i][e];
                __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, value), to, there ? (row * p.value_dim + column) * 4u : kNowhere, 0, 0);
            }
    }
}

// Sum over the 16 lanes that hold a row of D.
__device__ __forceinline__ float row_sum(float v)
{
    v += dpp<0xB1>(v);
    v += dpp<0x4E>(v);
    v += dpp<0x141>(v);
    v += dpp<0x140>(v);
    return v;
}

template <int N>
__device__ __forceinline__ float together(const b8 (&parts)[N], int i)
{
    float v = (float)parts[N - 1][i];
#pragma unroll
    for (int n = N - 2; n >= 0; --n) v += (float)parts[n][i];
    return v;
}

// A workgroup a chunk of a key head, through the value heads that share it; wavefront w the positions of tile w.  S, dS' and U of 32 value columns at a time
// go through LDS, as the operands that all four wavefronts need.
template <typename T, int KD>
__global__ __launch_bounds__(kDeltaThreads) void delta_grad_kernel(sys_gated_delta_t p, DeltaArgs a, DeltaShape shape, DeltaPlanes w)
{
    constexpr int NX = kInputParts<T>, RP = kResultParts<T>, KS = KD / 32, KT = KD / 16, TW = KD / 64, kPitch = kChunk + 8;
    const int chunk = blockIdx.x % shape.chunks, rest = blockIdx.x / shape.chunks, key_head = rest % p.key_heads, b = rest / p.key_heads;
    const int shared = p.value_heads / p.key_heads;
    const int t0 = chunk * kChunk, last = sequence_length(a.lengths, b, p.length), rows = last - t0;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, r = lane & 15, g = lane >> 4;
    const int here = p.length - t0 < kChunk ? p.length - t0 : kChunk;  // rows of the results
    const long long at0 = (long long)b * p.length + t0;
    T* ddelta = (T*)a.ddelta + at0 * p.value_heads;
    T* dbeta = (T*)a.dbeta + at0 * p.value_heads;
    if (rows <= 0) {
        for (int i = tid; i < here * p.key_dim; i += kDeltaThreads) {
            const long long at = ((at0 + i / p.key_dim) * p.key_heads + key_head) * p.key_dim + i % p.key_dim;
            ((T*)a.dq)[at] = (T)0.0f;
            ((T*)a.dk)[at] = (T)0.0f;
        }
        for (int i = tid; i < here * shared; i += kDeltaThreads) {
            const int at = i / shared * p.value_heads + key_head * shared + i % shared;
            ddelta[at] = (T)0.0f;
            dbeta[at] = (T)0.0f;
        }
        for (int i = tid; i < 2 * shared; i += kDeltaThreads)
            w.dg[(((size_t)b * p.value_heads + key_head * shared + i / 2) * shape.chunks + chunk) * 2 + i % 2] = 0.0f;
        return;
    }
    const size_t kc = ((size_t)b * p.key_heads + key_head) * shape.chunks + chunk;

    struct Columns { b8 s[KT][RP][64], ds[KT][RP][64], u[4][RP][64]; };
    struct Squares { bf16_t b[RP][kChunk][kPitch], c[RP][kChunk][kPitch], bt[RP][kChunk][kPitch], ct[RP][kChunk][kPitch]; };
    __shared__ union Pool {
        Columns columns;
        Squares squares;
        __device__ Pool() {}
    } pool;
    __shared__ float rows_dg[kChunk], rows_db[kChunk], rows_end[kChunk], columns_dg[4][kChunk], waves_end[4];

    f4 dq_all[KT] = {}, dk_all[KT] = {};
    for (int h = 0; h < shared; ++h) {
        const int head = key_head * shared + h;
        const size_t vc = ((size_t)b * p.value_heads + head) * shape.chunks + chunk;
        const T* dy = (const T*)a.dy + b * p.y_batch + t0 * p.y_row + head * p.value_dim;
        const T* v = (const T*)a.v + b * p.v_batch + t0 * p.v_row + head * p.value_dim;
        const bf16_t* from_s = w.s + vc * RP * KD * shape.columns;
        const bf16_t* from_ds = w.ds + vc * RP * KD * shape.columns;
        const bf16_t* from_u = w.u + vc * RP * kChunk * shape.columns;
        const bf16_t* from_z = w.z + vc * RP * kChunk * shape.columns;

        // pieces of 16 bytes: a row's four, then the rows
        b8 next_s[TW * RP], next_ds[TW * RP], next_u[RP], next_z[RP];
        float next_dy[8], next_v[8];
        auto fetch = [&](int step) {
            const int at = 32 * step + 8 * (tid & 3), row = tid >> 2;
#pragma unroll
            for (int m = 0; m < RP; ++m) {
#pragma unroll
                for (int i = 0; i < TW; ++i) {
                    next_s[i * RP + m] = *(const b8*)(from_s + ((size_t)m * KD + 64 * i + row) * shape.columns + at);
                    next_ds[i * RP + m] = *(const b8*)(from_ds + ((size_t)m * KD + 64 * i + row) * shape.columns + at);
                }
                next_u[m] = *(const b8*)(from_u + ((size_t)m * kChunk + row) * shape.columns + at);
                next_z[m] = *(const b8*)(from_z + ((size_t)m * kChunk + tile_row(wave, r)) * shape.columns + 32 * step + 8 * g);
            }
            const int mine = tile_row(wave, r);
            load_eight(dy + mine * p.y_row, 32 * step + 8 * g, p.value_dim, mine < rows, next_dy);
            load_eight(v + mine * p.v_row, 32 * step + 8 * g, p.value_dim, mine < rows, next_v);
        };
        f4 dq[KT] = {}, zs[KT] = {}, us[KT] = {}, dp[4] = {}, da[4] = {}, zv = {};
        float both = 0.0f;
        fetch(0);
        const int steps = shape.columns / 32;
        for (int step = 0; step < steps; ++step) {
            lds_barrier();
            {
                const int tile = tile_of(tid >> 2), to = (tid & 3) * 16 + row_in_tile(tid >> 2);
#pragma unroll
                for (int m = 0; m < RP; ++m) {
#pragma unroll
                    for (int i = 0; i < TW; ++i) {
                        pool.columns.s[4 * i + tile][m][to] = next_s[i * RP + m];
                        pool.columns.ds[4 * i + tile][m][to] = next_ds[i * RP + m];
                    }
                    pool.columns.u[tile][m][to] = next_u[m];
                }
            }
            b8 oa[NX], va[NX], za[RP], ua[RP];
            split8(next_dy, oa);
            split8(next_v, va);
#pragma unroll
            for (int m = 0; m < RP; ++m) za[m] = next_z[m];
            lds_barrier();
            if (step + 1 < steps) fetch(step + 1);
#pragma unroll
            for (int m = 0; m < RP; ++m) ua[m] = pool.columns.u[wave][m][lane];
            zv = multiply<RP - 1>(za, va, zv);
#pragma unroll
            for (int n = 0; n < 4; ++n)
                if (n / 2 <= wave / 2) {
                    b8 ub[RP];
#pragma unroll
                    for (int m = 0; m < RP; ++m) ub[m] = pool.columns.u[n][m][lane];
                    dp[n] = multiply<RP - 1>(oa, ub, dp[n]);
                    da[n] = multiply<RP - 1>(za, ub, da[n]);
                }
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                __builtin_amdgcn_sched_barrier(0);                     // (operands of one tile at a time, or the registers do not do)
                b8 sb[RP], db[RP];
#pragma unroll
                for (int m = 0; m < RP; ++m) sb[m] = pool.columns.s[t][m][lane], db[m] = pool.columns.ds[t][m][lane];
                dq[t] = multiply<RP - 1>(oa, sb, dq[t]);
                zs[t] = multiply<RP - 1>(za, sb, zs[t]);
                us[t] = multiply<RP - 1>(ua, db, us[t]);
                if (t / TW == wave) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) both = __builtin_fmaf(together(sb, i), together(db, i), both);
                }
            }
        }
        lds_barrier();
        // the squares B and C, as they are and transposed
        const float* scalars = w.scalars + vc * kScalars * kChunk;
        const double* sums = (const double*)(scalars + kSums * kChunk);
        const int mine = tile_row(wave, 4 * g), middle = wave >> 1;
        const f4 gamma = *(const f4*)(scalars + kGamma * kChunk + mine), left = *(const f4*)(scalars + kLeft * kChunk + mine);
        const f4 strength = *(const f4*)(scalars + kStrength * kChunk + mine);
        double mine_sum[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) mine_sum[e] = sums[mine + e];
        // (new addresses for every head, as far as the compiler knows: loaded ahead of the loop these operands would take all registers)
        const bf16_t *kt = w.kt + kc * NX * kChunk * KD, *qt = w.qt + kc * NX * kChunk * KD, *kp = w.k + kc * NX * kChunk * KD, *qp = w.q + kc * NX * kChunk * KD;
        asm volatile("" : "+s"(kt), "+s"(qt), "+s"(kp), "+s"(qp));
        f4 of_g = {}, of_b = {}, of_end = {};
#pragma unroll
        for (int n = 0; n < 4; ++n)
            if (n / 2 <= middle) {
                f4 kk = {}, qk = {};
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    b8 ka[NX], qa[NX], kb[NX];
#pragma unroll
                    for (int m = 0; m < NX; ++m) {
                        ka[m] = operand(kp + m * kChunk * KD, KS, wave, s, lane);
                        qa[m] = operand(qp + m * kChunk * KD, KS, wave, s, lane);
                        kb[m] = operand(kp + m * kChunk * KD, KS, n, s, lane);
                    }
                    kk = multiply<2>(ka, kb, kk);
                    qk = multiply<2>(qa, kb, qk);
                }
                const int column = tile_row(n, r);
                const double column_sum = sums[column];
                f4 fb, fc;
                float of_column = 0.0f;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float ratio = fast_exp2((float)(mine_sum[e] - column_sum));
                    fb[e] = column <= mine + e ? p.scale * (ratio * dp[n][e]) : 0.0f;
                    fc[e] = column < mine + e ? -(ratio * da[n][e]) : 0.0f;
                    const float both_of = column < mine + e ? __builtin_fmaf(fb[e], qk[e], strength[e] * (fc[e] * kk[e])) : 0.0f;
                    of_g[e] += both_of;
                    of_column += both_of;
                    of_b[e] = __builtin_fmaf(fc[e], kk[e], of_b[e]);
                }
                of_column += __shfl_xor(of_column, 16);
                of_column += __shfl_xor(of_column, 32);
                if (g == 0) columns_dg[wave][column] = of_column;
                u2 pb[RP], pc[RP], pct[RP];
                split4(fb, pb);
                split4(fc, pc);
                split4(strength * fc, pct);
#pragma unroll
                for (int m = 0; m < RP; ++m) {
                    *(u2*)&pool.squares.bt[m][column][mine] = pb[m];
                    *(u2*)&pool.squares.ct[m][column][mine] = pct[m];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        pool.squares.b[m][mine + e][column] = as_bf16(pb[m][e / 2] >> 16 * (e & 1));
                        pool.squares.c[m][mine + e][column] = as_bf16(pc[m][e / 2] >> 16 * (e & 1));
                    }
                }
            } else if (g == 0) {
                columns_dg[wave][tile_row(n, r)] = 0.0f;
            }
        lds_barrier();
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            __builtin_amdgcn_sched_barrier(0);
            f4 kr = -(gamma * zs[t]), kcol = left * us[t], qrow = gamma * p.scale * dq[t];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                b8 kb[NX], qb[NX], m1[RP], m2[RP];
#pragma unroll
                for (int n = 0; n < NX; ++n) {
                    kb[n] = operand(kt + n * kChunk * KD, 2, t, s, lane);
                    qb[n] = operand(qt + n * kChunk * KD, 2, t, s, lane);
                }
                if (s == middle) {
                    // the entries of these positions' own keys and queries are a half of this operand
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float k = wave & 1 ? together(kb, 4 + e) : together(kb, e), q = wave & 1 ? together(qb, 4 + e) : together(qb, e);
                        of_g[e] += __builtin_fmaf(q, gamma[e] * p.scale * dq[t][e], -(strength[e] * gamma[e]) * (k * zs[t][e]));
                        of_b[e] = __builtin_fmaf(-k, gamma[e] * zs[t][e], of_b[e]);
                        of_end[e] = __builtin_fmaf(k, left[e] * us[t][e], of_end[e]);
                    }
                }
                if (s <= middle) {
#pragma unroll
                    for (int m = 0; m < RP; ++m) {
                        m1[m] = *(const b8*)&pool.squares.b[m][tile_row(wave, r)][32 * s + 8 * g];
                        m2[m] = *(const b8*)&pool.squares.c[m][tile_row(wave, r)][32 * s + 8 * g];
                    }
                    qrow = multiply<RP - 1>(m1, kb, qrow);
                    kr = multiply<RP - 1>(m2, kb, kr);
                }
                if (s >= middle) {
#pragma unroll
                    for (int m = 0; m < RP; ++m) {
                        m1[m] = *(const b8*)&pool.squares.bt[m][tile_row(wave, r)][32 * s + 8 * g];
                        m2[m] = *(const b8*)&pool.squares.ct[m][tile_row(wave, r)][32 * s + 8 * g];
                    }
                    kcol = multiply<RP - 1>(m1, qb, kcol);
                    kcol = multiply<RP - 1>(m2, kb, kcol);
                }
            }
            dq_all[t] += qrow;
            dk_all[t] += strength * kr + kcol;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float dg = row_sum(of_g[e]), db = row_sum(of_b[e]), de = row_sum(of_end[e]);
            if (r == 0) {
                rows_dg[mine + e] = dg;
                rows_db[mine + e] = db;
                rows_end[mine + e] = de;
            }
        }
        // Z_i . V_i lies on the diagonal of this wavefront's tile
        lds_barrier();
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (r == 4 * g + e) rows_db[mine + e] += zv[e];
        for (int m = 32; m; m >>= 1) both += __shfl_xor(both, m);
        if (lane == 0) waves_end[wave] = both;
        lds_barrier();
        if (wave == 0) {
            // gradients of the sums G that end in a position and behind it, and of what is left behind the positions before it
            const double own = (double)rows_end[lane];
            double dg = (double)rows_dg[lane] - ((double)columns_dg[0][lane] + (double)columns_dg[1][lane] + (double)columns_dg[2][lane] + (double)columns_dg[3][lane]), de = own;
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) {
                const double behind = __shfl_down(dg, m), before = __shfl_up(de, m);
                if (lane + m < 64) dg += behind;
                if (lane >= m) de += before;
            }
            const double end = (double)scalars[kGamma * kChunk + kChunk - 1];
            const float log_decay =
                (float)(dg + (de - own) + end * ((double)waves_end[0] + (double)waves_end[1] + (double)waves_end[2] + (double)waves_end[3]));
            float of_a = 0.0f, of_bias = 0.0f, db = 0.0f;
            if (lane < rows) {
                const float pre = (float)((const T*)a.delta)[b * p.delta_batch + (t0 + lane) * p.delta_row + head] + (a.delta_bias ? a.delta_bias[head] : 0.0f);
                const float step = p.softplus ? softplus(pre) : pre;
                const float raw = (float)((const T*)a.beta)[b * p.beta_batch + (t0 + lane) * p.beta_row + head];
                of_a = step * log_decay;
                of_bias = a.a[head] * log_decay * (p.softplus ? sigmoid(pre) : 1.0f);
                db = rows_db[lane];
                if (p.sigmoid) {
                    const float x = sigmoid(raw);
                    db *= x * (1.0f - x);
                }
            }
            if (lane < here) {
                ddelta[lane * p.value_heads + head] = (T)of_bias;
                dbeta[lane * p.value_heads + head] = (T)db;
            }
#pragma unroll
            for (int m = 32; m; m >>= 1) of_a += __shfl_xor(of_a, m), of_bias += __shfl_xor(of_bias, m);
            if (lane == 0) {
                w.dg[vc * 2] = of_a;
                w.dg[vc * 2 + 1] = of_bias;
            }
        }
        // (the next head's operands are put where the squares lie behind a barrier of its own)
    }
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int row = tile_row(wave, 4 * g) + e, column = tile_row(t, r);
            if (row < here && column < p.key_dim) {
                const long long at = ((at0 + row) * p.key_heads + key_head) * p.key_dim + column;
                ((T*)a.dq)[at] = (T)dq_all[t][e];
                ((T*)a.dk)[at] = (T)dk_all[t][e];
            }
        }
}

// dA and the bias's gradient: the chunks' sums of a head, a wavefront a head, in 64 bits.
__global__ __launch_bounds__(64) void delta_gates_kernel(sys_gated_delta_t p, DeltaArgs a, DeltaShape shape, DeltaPlanes w)
{
    const int head = blockIdx.x, lane = threadIdx.x;
    double of_a = 0.0, of_bias = 0.0;
    for (int b = 0; b < p.batch; ++b)
        for (int c = lane; c < shape.chunks; c += 64) {
            const float* from = w.dg + (((size_t)b * p.value_heads + head) * shape.chunks + c) * 2;
            of_a += (double)from[0];
            of_bias += (double)from[1];
        }
#pragma unroll
    for (int m = 32; m; m >>= 1) of_a += __shfl_xor(of_a, m), of_bias += __shfl_xor(of_bias, m);
    if (lane == 0) {
        a.da[head] = (float)of_a;
        if (a.ddelta_bias) a.ddelta_bias[head] = (float)of_bias;
    }
}

template <typename T, int KD>
hipError_t run(const sys_gated_delta_t& p, const DeltaArgs& a, const DeltaShape& shape, const DeltaPlanes& w, hipStream_t s)
{
    DeltaShape of = shape;
    of.tiles = shape.columns / 16;
    const long long sweeps = (long long)of.tiles * p.value_heads * p.batch, chunks = (long long)shape.chunks * p.key_heads * p.batch;
    if (sweeps > 0x7fffffffLL || chunks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((delta_back_kernel<T, KD>), dim3((unsigned)sweeps), dim3(kDeltaThreads), 0, s, p, a, of, w);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !chunks) return e;
    hipLaunchKernelGGL((delta_grad_kernel<T, KD>), dim3((unsigned)chunks), dim3(kDeltaThreads), 0, s, p, a, shape, w);
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
    hipLaunchKernelGGL(delta_gates_kernel, dim3((unsigned)p.value_heads), dim3(64), 0, s, p, a, shape, w);
    return hipGetLastError();
}

}  // namespace sysconv
