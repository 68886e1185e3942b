// Device code shared by the products with experts' weights in 4-bit floating point.
#pragma once

#include "block_device.h"
#include "mx_ops.h"

namespace fluxmoe {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

struct Tile {
    uint32_t expert, first, rows;            // rows 0: no such tile
};

// Rows of expert e that lie within the matrix, whatever offsets and counts hold.
__device__ __forceinline__ uint32_t rows_of(const MxProductArgs& a, uint32_t e) {
    const int32_t c = a.counts[e], o = a.offsets[e];
    if (c <= 0 || o < 0 || uint32_t(o) >= a.cap) return 0;
    return min(uint32_t(c), a.cap - uint32_t(o));
}

// Tile number `wanted` of the experts' groups in their order, `size` rows to a tile.  All threads of the workgroup; a thread
// adds up neighbouring experts.  s: kTileWords of LDS.
constexpr uint32_t kTileWords = 16;
template <uint32_t THREADS>
__device__ __forceinline__ Tile find_tile(const MxProductArgs& a, uint32_t size, uint32_t wanted, uint32_t* s) {
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t per = (a.E + THREADS - 1) / THREADS, from = min(tid * per, a.E), to = min(from + per, a.E);
    static_assert(THREADS / 64 + 3 <= kTileWords, "wavefronts' sums and the tile");
    uint32_t mine = 0;
    for (uint32_t e = from; e < to; ++e) mine += (rows_of(a, e) + size - 1) / size;
    uint32_t upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t below = __shfl_up(upto, d);
        if (lane >= uint32_t(d)) upto += below;
    }
    __syncthreads();                                     // the last tile's readers are done with s
    if (lane == 63) s[wave] = upto;
    if (tid == 0) s[THREADS / 64 + 2] = 0;
    __syncthreads();
    for (uint32_t w = 0; w < wave; ++w) upto += s[w];
    uint32_t before = upto - mine;
    if (wanted >= before && wanted < upto) {
        for (uint32_t e = from; e < to; ++e) {
            const uint32_t rows = rows_of(a, e), tiles = (rows + size - 1) / size;
            if (wanted < before + tiles) {
                const uint32_t at = (wanted - before) * size;
                s[THREADS / 64] = e;
                s[THREADS / 64 + 1] = uint32_t(a.offsets[e]) + at;
                s[THREADS / 64 + 2] = min(size, rows - at);
                break;
            }
            before += tiles;
        }
    }
    __syncthreads();
    Tile t;
    t.expert = __builtin_amdgcn_readfirstlane(s[THREADS / 64]);
    t.first = __builtin_amdgcn_readfirstlane(s[THREADS / 64 + 1]);
    t.rows = __builtin_amdgcn_readfirstlane(s[THREADS / 64 + 2]);
    return t;
}

// `records` bytes from `base` on, by offset: reads past them give 0
__device__ __forceinline__ row_t bytes_at(const void* base, uint64_t offset, uint32_t records) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(base) + offset), 0, int(records), 0x00020000);
}
constexpr uint32_t kNowhere = 0x7FFFFFF0u;               // an offset past any resource's records

__device__ __forceinline__ float scale_operand(uint32_t s) { return __uint_as_float(s << 23); }

// Eight codes as BF16
__device__ __forceinline__ bf16x8 codes_bf16(uint32_t codes, float scale) {
    const u32x4 v = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
    return __builtin_bit_cast(bf16x8, v);
}

}  // namespace fluxmoe
