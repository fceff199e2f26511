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

// B or C of kScanTile positions for LDS, [position][4 * NS], zeros past the last state and the sequence's end: first into registers ...
template <typename T, int NS>
struct StateTile {
    static constexpr int kWidth = 4 * NS;
    static constexpr int kEach = (kScanTile * kWidth + kScanThreads - 1) / kScanThreads;
    float v[kEach];
    __device__ __forceinline__ void load(const T* rows, long long row, int states, int t0, int length)
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int k = i * kScanThreads + (int)threadIdx.x;
            const int t = t0 + k / kWidth, n = k % kWidth;
            v[i] = k < kScanTile * kWidth && t < length && n < states ? (float)rows[t * row + n] : 0.0f;
        }
    }
    // ... and from there into LDS
    __device__ __forceinline__ void store(float* lds) const
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int k = i * kScanThreads + (int)threadIdx.x;
            if (k < kScanTile * kWidth) lds[k] = v[i];
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
