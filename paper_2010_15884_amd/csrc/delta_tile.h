// How the gated delta rule in chunks is laid on the matrix cores (delta_chunk.hip, delta_grad.hip).
//
// Over a chunk of 64 positions with the state S before it, G_i the sum of the logarithms of the decays up to position i,
//   X = (I + A)^-1,  A_ij = b_i e^(G_i - G_j) k_i . k_j (j < i)
//   U = X (b (V - e^G (K S))),  Y = scale e^G (Q S) + P U,  P_ij = scale e^(G_i - G_j) q_i . k_j (j <= i)
//   S' = e^(G_end) S + K^T (e^(G_end - G) U)
// A, X and P belong to the keys and queries alone and are made for all chunks side by side; what is left to do one chunk after
// the other are products with S, U and the like, whose columns (of the values) do not meet.
//
// Precision: v_mfma_f32_16x16x32_bf16 on numbers that are split into bf16 parts, accumulated in fp32.  Inputs in bf16 are one part, in fp16
// two, in fp32 three, exactly; states, U and what leads to them are three (24 bits), and products of parts i and j are taken up to
// i + j = 2, so that what is left out is below 2^-24 of the term, as in split_bf16.h.  What only leads to 16-bit results is no exception: what a position reads of the state
// before its chunk and what the chunk writes cancel where values are written over larger ones, and with two parts outputs and the gradients of q and k came out off by 2^-17 of the
// old values (three cost 3 % of the forward call in bf16, 8 in fp16, and 2 of the gradients' in bf16).
// The split keeps fp32's range; infinities in it become NaN, and a NaN reaches all positions of its chunk (0 times NaN).
//
// Layout: D of an instruction holds rows 4 (lane / 16) + i of column lane % 16, B takes rows 8 (lane / 16) + j of column lane % 16.
// With the rows of A permuted (row m of tile 2s + h is row 32 s + 8 (m / 4) + 4 h + m % 4 of the matrix) two tiles of D are a B operand as they
// lie: products follow each other without an exchange between lanes, and every A operand is 16 bytes of a row of a matrix.
#pragma once

#include "scan_tile.h"
#include "sequence.h"
#include "split_bf16.h"

#include <type_traits>

namespace sysconv {

typedef float f4 __attribute__((ext_vector_type(4)));

constexpr int kChunk = 64;
constexpr int kDeltaThreads = 256;
constexpr int kSweepThreads = 512;                 // four wavefronts that go through the state, four that do the rest
constexpr int kSquare = kChunk * kChunk;           // elements of X, P

// Parts of an input.
template <typename T> constexpr int kInputParts = sizeof(T) == 4 ? 3 : std::is_same<T, f16_t>::value ? 2 : 1;
__device__ __forceinline__ f4 mfma(b8 a, b8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// c += a b, parts whose order is at most MOST, the small ones first.
template <int MOST, int NA, int NB>
__device__ __forceinline__ f4 multiply(const b8 (&a)[NA], const b8 (&b)[NB], f4 c)
{
#pragma unroll
    for (int order = MOST; order >= 0; --order)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (order - i >= 0 && order - i < NB) c = mfma(a[i], b[order - i], c);
    return c;
}

// The same with a sum of its own for each order, so that instructions do not wait for each other; and the sum of these.
template <int MOST, int NA, int NB>
__device__ __forceinline__ void multiply_apart(const b8 (&a)[NA], const b8 (&b)[NB], f4 (&c)[MOST + 1])
{
#pragma unroll
    for (int order = MOST; order >= 0; --order)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (order - i >= 0 && order - i < NB) c[order] = mfma(a[i], b[order - i], c[order]);
}
template <int N>
__device__ __forceinline__ f4 joined(const f4 (&c)[N])
{
    f4 sum = c[N - 1];
#pragma unroll
    for (int i = N - 2; i >= 0; --i) sum += c[i];
    return sum;
}

// Eight numbers as N parts each.
template <int N>
__device__ __forceinline__ void split8(const float (&v)[8], b8 (&out)[N])
{
    float rest[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = v[i];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        u4 packed;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            packed[i] = __builtin_bit_cast(unsigned, __builtin_convertvector(f2{rest[2 * i], rest[2 * i + 1]}, b2));
            if (n + 1 < N) {
                rest[2 * i] -= __builtin_bit_cast(float, packed[i] << 16);
                rest[2 * i + 1] -= __builtin_bit_cast(float, packed[i] & 0xffff0000u);
            }
        }
        out[n] = __builtin_bit_cast(b8, packed);
    }
}

// Four numbers as N parts each, 8 bytes a part.
template <int N>
__device__ __forceinline__ void split4(f4 rest, u2 (&out)[N])
{
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const unsigned packed = __builtin_bit_cast(unsigned, __builtin_convertvector(f2{rest[2 * i], rest[2 * i + 1]}, b2));
            out[n][i] = packed;
            if (n + 1 < N) {
                rest[2 * i] -= __builtin_bit_cast(float, packed << 16);
                rest[2 * i + 1] -= __builtin_bit_cast(float, packed & 0xffff0000u);
            }
        }
}

// The row of a matrix that is row m of tile `tile` of an A operand, and of D; and the other way round.
__device__ __forceinline__ constexpr int tile_row(int tile, int m) { return 32 * (tile >> 1) + 8 * (m >> 2) + 4 * (tile & 1) + (m & 3); }
__device__ __forceinline__ constexpr int tile_of(int row) { return 2 * (row >> 5) + (row >> 2 & 1); }
__device__ __forceinline__ constexpr int row_in_tile(int row) { return 4 * (row >> 3 & 3) + (row & 3); }

// Matrices lie in the workspace as the operands that are taken of them: 1 KB a tile of rows and step of 32 columns, where lane l has the eight entries from
// column 8 (l / 16) on of row l % 16 of the tile.  (Row-major, a load's neighbouring lanes would be in rows of their own: 45 cache accesses an
// instruction instead of 16, and the addresses' unit was what the sweep waited for: it took half again as long for 4096 positions of 32 heads of 128 x 128.)
__device__ __forceinline__ b8 operand(const bf16_t* matrix, int steps, int tile, int step, int lane)
{
    return *(const b8*)(matrix + ((tile * steps + step) * 64 + lane) * 8);
}

// Four rows of a column a lane, as D has them, to four columns of a row: lane q of a quad gets row q of the quad's columns.
__device__ __forceinline__ f4 turn_quad(f4 v)
{
    const bool odd = threadIdx.x & 1, high = threadIdx.x & 2;
    const float a = dpp<0xB1>(odd ? v[0] : v[1]), b = dpp<0xB1>(odd ? v[2] : v[3]);
    const float p0 = odd ? a : v[0], p1 = odd ? v[1] : a, p2 = odd ? b : v[2], p3 = odd ? v[3] : b;
    const float c = dpp<0x4E>(high ? p0 : p2), d = dpp<0x4E>(high ? p1 : p3);
    return high ? f4{c, d, p2, p3} : f4{p0, p1, c, d};
}

// The matrix cores cut the sums of an instruction off towards minus infinity; with operands whose entries are mostly of one sign, as keys behind an
// activation are, that adds up over a row and over the positions, and the gradients of A were off by 2e-6 of themselves.  So S, dS and U lie in the workspace
// with every other tile of rows negated, which are columns of the products that are taken of them; their sums are taken back where they are used, and it cancels.
__device__ __forceinline__ f4 signed_rows(f4 v, int tile) { return tile & 1 ? -v : v; }

// Where an element of S, dS, U or Z lies: blocks of 32 columns, row-major.
__device__ __forceinline__ size_t block_place(size_t chunk, int rows, int columns, int row, int column)
{
    return (chunk * columns + (column & ~31)) * rows + row * 32 + (column & 31);
}

// The barrier of a workgroup whose wavefronts exchange through LDS alone: loads from memory stay in flight.
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    // lgkmcnt(0): the wait that the fence stands for is dropped by the compiler where a loop begins with the barrier and nothing is outstanding when it is entered, also
    // if its last writes are on the way back
    __builtin_amdgcn_s_waitcnt(0xc07f);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Where a workgroup keeps B operands: [step][part][column tile], 1 KB each, 16 bytes a lane.
template <int STEPS, int PARTS, int NT>
struct Operands {
    b8 v[STEPS][PARTS][NT][64];
    // all of step `step` from two tiles of D that lie above each other, or half of it from one
    __device__ __forceinline__ void put(int step, int n, int lane, f4 upper, f4 lower)
    {
        float both[8];
        b8 parts[PARTS];
#pragma unroll
        for (int e = 0; e < 4; ++e) both[e] = upper[e], both[4 + e] = lower[e];
        split8(both, parts);
#pragma unroll
        for (int m = 0; m < PARTS; ++m) v[step][m][n][lane] = parts[m];
    }
    __device__ __forceinline__ void put_half(int tile, int n, int lane, f4 d)
    {
        u2 parts[PARTS];
        split4(d, parts);
#pragma unroll
        for (int m = 0; m < PARTS; ++m) ((u2*)&v[tile >> 1][m][n][lane])[tile & 1] = parts[m];
    }
    // as many parts of it as are wanted
    template <int N>
    __device__ __forceinline__ void take(int step, int n, int lane, b8 (&out)[N]) const
    {
#pragma unroll
        for (int m = 0; m < N; ++m) out[m] = v[step][m][n][lane];
    }
    // the numbers that put_half was given
    __device__ __forceinline__ f4 numbers(int tile, int n, int lane) const
    {
        f4 sum = {};
#pragma unroll
        for (int m = PARTS - 1; m >= 0; --m) {
            const u2 part = ((const u2*)&v[tile >> 1][m][n][lane])[tile & 1];
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += __builtin_bit_cast(float, e & 1 ? part[e / 2] & 0xffff0000u : part[e / 2] << 16);
        }
        return sum;
    }
};

// What the kernel that makes the chunks' matrices leaves in the workspace for those that go through them: planes of parts, as operands.  Per value head and
// chunk X and P [64][64] (gradients: transposes of both; three parts), and for every position the Scalars; per key head and chunk
// K, Q [64][padded] and their transposes (parts of inputs).  Gradients: S, U of the sweep forwards and dS, Z of the one backwards as well, in fp32.
struct DeltaPlanes {
    bf16_t *x, *p, *xt, *pt, *k, *q, *kt, *qt;
    float *s, *ds, *u, *z;             // [columns / 32][padded][32], [columns / 32][64][32]
    float* scalars;                    // [kScalars][64]
    float* parts;                      // where heads are apart, their shares of dq and dk: [2][64][padded]
    double *gates, *shares;            // of a chunk of a value head: [kGates][64]; its share of the gradients of A and the bias
};

struct DeltaShape {
    int chunks;                        // of a sequence
    int padded;                        // the key dimension as the kernels have it, 64 or 128
    int columns;                       // the value dimension rounded up to 32
    int tiles;                         // of columns
    int whole, whole_values;           // rows of q and k, of v and dy may be loaded 16 bytes at a time
    int apart;                         // gradients of a chunk: a workgroup for each of the value heads of a key head
};

// e^G, e^(G_end - G), b; for gradients the step size and its derivative by delta, and G in 64 bits, to base 2
enum Scalars { kGamma, kLeft, kStrength, kStep, kSums, kSlope = 6, kScalars };

// Of a position: the gradient of the sum G that ends there, of what is left behind it, of its strength; of all alike
enum Gates { kGateRows, kGateEnds, kGateStrengths, kGateWhole, kGates };

inline int delta_padded(const sys_gated_delta_t& p) { return p.key_dim <= 64 ? 64 : 128; }
inline int delta_chunks(const sys_gated_delta_t& p) { return (p.length + kChunk - 1) / kChunk; }

__device__ __forceinline__ bf16_t as_bf16(unsigned bits) { return __builtin_bit_cast(bf16_t, (unsigned short)bits); }

// Entries of neighbouring positions of a chunk, one column a lane, addressed as a buffer that ends with the last row that exists.  Rows behind it lie past that end
// only where rows are no less apart than they are long: inputs may use a row again, or one row's end as another's beginning, and where there is one row the
// distance to the next may be anything.  So what is read goes by the row's number.
template <typename T>
struct ChunkRows {
    T* at;                             // row 0 of the present chunk
    long long left, row;               // bytes to the end of the last row
    int exist;                         // rows from the present chunk's first one on
    __device__ __forceinline__ ChunkRows(const void* base, long long row_stride, int columns, int chunk, int end)
        : at((T*)base + chunk * kChunk * row_stride), left(bytes_left(chunk * kChunk, end, row_stride, columns, sizeof(T))), row(row_stride), exist(end - chunk * kChunk)
    {
    }
    __device__ __forceinline__ void move(int chunks)
    {
        at += chunks * kChunk * row, left -= chunks * kChunk * row * (long long)sizeof(T), exist -= chunks * kChunk;
    }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer() const { return __builtin_amdgcn_make_buffer_rsrc((void*)at, 0, buffer_size(left), 0x00027000); }
    __device__ __forceinline__ unsigned offset(int r, int column) const { return (unsigned)((r * row + column) * (long long)sizeof(T)); }
    // of an entry that is read: nowhere, which gives 0, if its row does not exist
    __device__ __forceinline__ unsigned place(int r, int column) const { return r < exist ? offset(r, column) : kNowhere; }
};

// Eight neighbouring entries of a row on their way into parts.
template <typename T>
struct Eight {
    u4 v[sizeof(T) / 2];
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rows, unsigned offset)
    {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = __builtin_bit_cast(u4, __builtin_amdgcn_raw_buffer_load_b128(rows, offset, 16 * i, 0));
    }
    // one by one; those behind the `left` that belong to the row (none of a row that does not exist) are dropped when they are there (they lie in the buffer or past its end)
    __device__ __forceinline__ void load_each(__amdgpu_buffer_rsrc_t rows, unsigned offset, int left)
    {
        constexpr int kEach = 4 / (int)sizeof(T);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                unsigned word = 0;
#pragma unroll
                for (int e = 0; e < kEach; ++e) {
                    const int at = (4 * i + j) * kEach + e;
                    unsigned got;
                    if constexpr (sizeof(T) == 4) got = __builtin_amdgcn_raw_buffer_load_b32(rows, offset + at * 4, 0, 0);
                    else got = __builtin_amdgcn_raw_buffer_load_b16(rows, offset + at * 2, 0, 0);
                    word |= (at < left ? got : 0u) << 16 * e;
                }
                v[i][j] = word;
            }
    }
    __device__ __forceinline__ void values(float (&f)[8]) const
    {
        typedef T Piece __attribute__((ext_vector_type(16 / sizeof(T))));
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            const Piece piece = __builtin_bit_cast(Piece, v[i]);
#pragma unroll
            for (int j = 0; j < 16 / (int)sizeof(T); ++j) f[16 / sizeof(T) * i + j] = (float)piece[j];
        }
    }
    template <int N>
    __device__ __forceinline__ void split(b8 (&out)[N]) const
    {
        if constexpr (N == 1) {
            out[0] = __builtin_bit_cast(b8, v[0]);
        } else {
            float f[8];
            values(f);
            split8(f, out);
        }
    }
};

// The two kernels in front of all others (delta_chunk.hip): the chunks' matrices, and the sweep forwards, which gives the outputs or, for gradients, S and U.
hipError_t launch_delta_matrices(const sys_gated_delta_t& p, const DeltaArgs& a, const DeltaShape& shape, const DeltaPlanes& w, bool grad, hipStream_t s);
hipError_t launch_delta_sweep(const sys_gated_delta_t& p, const DeltaArgs& a, const DeltaShape& shape, const DeltaPlanes& w, bool grad, hipStream_t s);
DeltaShape delta_shape(const sys_gated_delta_t& p, const DeltaArgs* a = nullptr);
// Whether the sweeps take 32 columns a workgroup, not 16: where there are more workgroups of 16 than CUs, of which each holds one.
constexpr int kCus = 256;
bool delta_wide(const sys_gated_delta_t& p);
// The planes of a call, from `base` on (a null pointer: for their size), and the bytes that they take.
size_t delta_planes(const sys_gated_delta_t& p, const DeltaShape& shape, bool grad, void* base, DeltaPlanes* w);
// A position at a time (delta_rule.hip).
hipError_t launch_delta_positions(const sys_gated_delta_t& p, const DeltaArgs& a, hipStream_t s);

}  // namespace sysconv
