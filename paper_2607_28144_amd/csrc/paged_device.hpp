// Device helpers of the kernels of a cache in pages: which sequence a piece of
// a call belongs to, and sums over a wave.
#pragma once
#include "paged_kernels.hpp"

namespace regenvc {
namespace paged {

__device__ __forceinline__ int first_of(const Batch &n, int b)
{
    return max(0, min(n.first[b], n.T));
}
__device__ __forceinline__ int places_of(const Batch &n, int b, int shift)
{
    return max(0, min(n.lens[b], n.columns << shift));
}

// The last sequence whose first piece is at most j, or -1; from(b) ascends.
// Every lane of the wave takes part and gets the answer: 64 sequences are
// looked at together, so up to 64 cost one load.
template <typename F>
__device__ __forceinline__ int last_from(int B, int64_t j, F from)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, n = B;
    while (n > 0) {
        const int step = (n + 63) >> 6, b = lo + lane * step;
        const bool le = b < lo + n && from(min(b, B - 1)) <= j;
        const int c = __popcll(__builtin_amdgcn_ballot_w64(le));
        if (c == 0) return -1;
        const int at = lo + (c - 1) * step;
        if (step == 1) return at;
        n = min(step, lo + n - at);
        lo = at;
    }
    return -1;
}

// The queries of block j: rows row .. row + rows - 1, of which the first stands
// at place `pos` of sequence b, which has `len` places.  rows 0: no such block.
// A sequence's blocks begin at first[b] / size + b, so that T / size + B numbers
// are enough for any division of T rows into B sequences.
struct Block {
    int b, row, rows, pos, len;
};
__device__ __forceinline__ Block block_of(const Batch &n, int shift, int size, int64_t j)
{
    Block k{0, 0, 0, 0, 0};
    // the same for all lanes, which the compiler does not see in what was loaded: scalars
    const int b = __builtin_amdgcn_readfirstlane(last_from(n.B, j, [&](int i) { return (int64_t)(first_of(n, i) / size) + i; }));
    if (b < 0) return k;
    const int f0 = __builtin_amdgcn_readfirstlane(first_of(n, b)), f1 = __builtin_amdgcn_readfirstlane(first_of(n, b + 1));
    const int64_t at = (j - f0 / size - b) * size;
    if (at >= f1 - f0) return k;
    k.b = b;
    k.row = f0 + (int)at;
    k.rows = min(size, f1 - k.row);
    k.len = __builtin_amdgcn_readfirstlane(places_of(n, b, shift));
    k.pos = k.len - (f1 - k.row);
    return k;
}

// Exchanges within 16 lanes, by a lane's number: its neighbour 1 and 2 off, its
// mirror image in 8, the lane 8 off.
constexpr int kXor1 = 0xb1, kXor2 = 0x4e, kMirror8 = 0x141, kRotate8 = 0x128;
// The larger of a wave's numbers, in every lane.
__device__ __forceinline__ uint32_t wave_max(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, kXor1, 0xf, 0xf, true));
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, kXor2, 0xf, 0xf, true));
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, kMirror8, 0xf, 0xf, true));
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, kRotate8, 0xf, 0xf, true));
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max(r[0], r[1]);
    const auto u = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return max(u[0], u[1]);
}
// The sum of the numbers of the lanes up to this one.
__device__ __forceinline__ uint32_t wave_upto(uint32_t x)
{
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false);  // from 1, 2, 4, 8 lanes below, within 16
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false);  // lane 15 to the next 16, 31 to the last 32
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false);
    return x;
}
// The sum of a wave's numbers, the same in every lane: each exchange adds the same two numbers on both sides.
__device__ __forceinline__ float wave_sum(float x)
{
    x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), kXor1, 0xf, 0xf, true));
    x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), kXor2, 0xf, 0xf, true));
    x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), kMirror8, 0xf, 0xf, true));
    x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), kRotate8, 0xf, 0xf, true));
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    const auto u = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(u[0]) + __uint_as_float(u[1]);
}

}  // namespace paged
}  // namespace regenvc
