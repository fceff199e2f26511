// How the selective scan's kernels lay a problem on the chip (selective_scan.hip, selective_scan_grad.hip).
//
// A channel's states lie with the four lanes of a quad, NS = ceil(states / 4) (rounded up to a power of two) to a lane, so a
// wavefront runs 16 channels and sums over states take two DPP additions.  What belongs to a (position, channel) alone -- the
// step size with its softplus, the gate -- would be computed four times over; instead lane j of a quad owns the positions
// 4k + j and hands its values to the others by DPP, which costs nothing where the multiply takes the operand.
// A workgroup runs 64 neighbouring channels of one group of B and C.  B and C of a tile of positions are converted once and
// lie in LDS as fp32 (the 16 channels of a wavefront read the same 16 bytes: no bank conflicts).
#pragma once

#include "sequence.h"

namespace sysconv {

constexpr int kScanThreads = 256;
constexpr int kScanChannels = kScanThreads / 4;     // a workgroup
constexpr int kScanTile = 16;                       // positions a tile

// An offset within a tile that is never read or written: no tile's buffer reaches it, and every element of a tile lies below it.
constexpr unsigned kNowhere = 0xfffffff0u;
static_assert(4 * ((kScanTile - 1) * SYS_MAX_SCAN_ROW + (1LL << 24)) <= kNowhere, "a tile's rows lie below kNowhere (up to 2^24 channels)");

// Bytes from row t0 to the end of the last row that exists, row end - 1; none or less where no row does, whatever the stride (rows that are
// used again, or of an empty sequence, which has no memory at all).
__host__ __device__ __forceinline__ long long bytes_left(int t0, int end, long long row, int columns, size_t element)
{
    return ((long long)(end - 1 - t0) * row + (t0 < end ? columns : 0)) * (long long)element;
}

// The size of a tile's buffer: the bytes from its first element to the end of the last row that exists, where they are that many.
__host__ __device__ __forceinline__ unsigned buffer_size(long long bytes)
{
    const int high = (int)(bytes >> 32);
    const unsigned low = (unsigned)bytes;
    return high < 0 ? 0u : high || low > kNowhere ? kNowhere : low;
}

struct ScanShape {
    int channels_a_group, blocks_a_group, channel_blocks;   // of 64 channels
    int chunks, chunk_rows;                                 // the positions in parts that run side by side
};

inline int scan_states_a_lane(int states)
{
    int ns = 1;
    while (4 * ns < states) ns *= 2;
    return ns;
}

// Index arithmetic of one workgroup.
struct ScanPlace {
    int batch, chunk, group, channel;   // channel: of this lane
    bool there;                         // it exists (lanes past the last channel repeat it and store nothing)
    int length, begin, end;             // positions of the sequence that exist; those of the chunk
};

__device__ __forceinline__ ScanPlace scan_place(const sys_selective_scan_t& p, const ScanShape& shape, const int* lengths, int block)
{
    ScanPlace at;
    const int channel_block = block % shape.channel_blocks;
    const int rest = block / shape.channel_blocks;
    at.chunk = rest % shape.chunks;
    at.batch = rest / shape.chunks;
    at.group = channel_block / shape.blocks_a_group;
    const int within = (channel_block - at.group * shape.blocks_a_group) * kScanChannels + (int)(threadIdx.x >> 2);
    at.there = within < shape.channels_a_group;
    at.channel = at.group * shape.channels_a_group + (at.there ? within : shape.channels_a_group - 1);
    at.length = sequence_length(lengths, at.batch, p.length);
    at.begin = at.chunk * shape.chunk_rows;
    at.end = at.begin + shape.chunk_rows < p.length ? at.begin + shape.chunk_rows : p.length;
    return at;
}

// A tile of rows of a strided tensor, addressed as a buffer that ends with the last row that exists: a lane's offset within a tile is worked
// out once, the tile's place is uniform, and rows past the end give zeros (or are not written) without a branch, which would make
// every load wait for the one before it.  Rows are at most SYS_MAX_SCAN_ROW elements apart, so that a tile's offsets fit 32 bits.
template <typename T>
struct RowBuffer {
    T* at;                             // row 0 of the present tile, column 0
    long long left;                    // bytes from there to the end of the last row that exists; none left: every load gives 0
    long long row;
    __device__ __forceinline__ RowBuffer(const void* base, long long row_stride, int columns, int t0, int end)
        : at((T*)base + t0 * row_stride), left(bytes_left(t0, end, row_stride, columns, sizeof(T))), row(row_stride)
    {
    }
    // the rows from `down` rows below the present tile's first one on
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t tile(int down = 0) const
    {
        const long long bytes = left - down * row * (long long)sizeof(T);
        return __builtin_amdgcn_make_buffer_rsrc((void*)(at + down * row), 0, buffer_size(bytes), 0x00027000);
    }
    __device__ __forceinline__ void next() { at += kScanTile * row, left -= kScanTile * row * (long long)sizeof(T); }
    __device__ __forceinline__ unsigned offset(int r, int column) const { return (unsigned)((r * row + column) * (long long)sizeof(T)); }
};

// An element as it was loaded, 32 bits a value: 16-bit values in a register each, or the compiler packs pairs and waits for the loads to do so.
template <typename T>
__device__ __forceinline__ unsigned buffer_load(__amdgpu_buffer_rsrc_t b, unsigned offset)
{
    if constexpr (sizeof(T) == 4) return __builtin_amdgcn_raw_buffer_load_b32(b, offset, 0, 0);
    else return __builtin_amdgcn_raw_buffer_load_b16(b, offset, 0, 0);
}

template <typename T>
__device__ __forceinline__ float loaded(unsigned v)
{
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, v);
    else return (float)__builtin_bit_cast(T, (unsigned short)v);
}

template <typename T>
__device__ __forceinline__ void buffer_store(__amdgpu_buffer_rsrc_t b, unsigned offset, T v)
{
    if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, v), b, offset, 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, v), b, offset, 0, 0);
}

// B or C of kScanTile positions for LDS, [position][4 * NS], zeros past the last state and the sequence's end: first into registers ...
template <typename T, int NS>
struct StateTile {
    static constexpr int kWidth = 4 * NS;
    static constexpr int kEach = (kScanTile * kWidth + kScanThreads - 1) / kScanThreads;
    static constexpr int kRowStep = kScanThreads / kWidth;             // rows from one of a lane's elements to the next
    static_assert(kScanThreads % kWidth == 0, "a lane keeps its state");
    RowBuffer<T> rows;
    unsigned v[kEach], offset[kEach];
    int end;
    bool is;
    __device__ __forceinline__ StateTile(const T* base, long long row, int states, int t0, int end_row)
        : rows(base, row, states, t0, end_row), end(end_row), is((int)threadIdx.x % kWidth < states)
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) offset[i] = rows.offset((int)threadIdx.x / kWidth + i * kRowStep, (int)threadIdx.x % kWidth);
    }
    __device__ __forceinline__ void load()
    {
        const __amdgpu_buffer_rsrc_t b = rows.tile();
#pragma unroll
        for (int i = 0; i < kEach; ++i) v[i] = buffer_load<T>(b, offset[i]);
        rows.next();
    }
    // ... and from there into LDS
    __device__ __forceinline__ void store(float* lds, int t0) const
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int r = (int)threadIdx.x / kWidth + i * kRowStep;
            if (kEach * kRowStep <= kScanTile || r < kScanTile)
                lds[r * kWidth + (int)threadIdx.x % kWidth] = is && t0 + r < end ? loaded<T>(v[i]) : 0.0f;
        }
    }
};

// NS floats of LDS, 16 bytes at a time where there are as many.
template <int NS>
__device__ __forceinline__ void take(const float* lds, float (&out)[NS])
{
    typedef float F4 __attribute__((ext_vector_type(4)));
    typedef float F2 __attribute__((ext_vector_type(2)));
    if constexpr (NS >= 4) {
#pragma unroll
        for (int i = 0; i < NS / 4; ++i) {
            const F4 v = *(const F4*)(lds + 4 * i);
#pragma unroll
            for (int k = 0; k < 4; ++k) out[4 * i + k] = v[k];
        }
    } else if constexpr (NS == 2) {
        const F2 v = *(const F2*)lds;
        out[0] = v[0];
        out[1] = v[1];
    } else {
        out[0] = *lds;
    }
}

}  // namespace sysconv
