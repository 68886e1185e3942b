// Device code shared by the products with experts' weights in 4-bit floating point.
#pragma once

#include <type_traits>

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

// The four scales of blocks `at` .. `at` + 3 of a row of `blocks` that lies `row` bytes into m, 0 past its end.  WHOLE: they are whole words.
template <bool WHOLE>
__device__ __forceinline__ uint32_t four_scales(row_t m, uint32_t row, uint32_t at, uint32_t blocks) {
    if constexpr (WHOLE) return __builtin_amdgcn_raw_buffer_load_b32(m, at < blocks ? row + at : kNowhere, 0, kCached);
    uint32_t v[4];
#pragma unroll
    for (uint32_t b = 0; b < 4; ++b) v[b] = __builtin_amdgcn_raw_buffer_load_b8(m, at + b < blocks ? row + at + b : kNowhere, 0, kCached);
    return v[0] | v[1] << 8 | v[2] << 16 | v[3] << 24;
}

// The scales of blocks block, block + 4, block + 8, block + 12 of such a row, block being q (0 .. 3) past a multiple of 16.
template <bool WHOLE>
__device__ __forceinline__ uint32_t spread_scales(row_t m, uint32_t row, uint32_t block, uint32_t q, uint32_t blocks) {
    uint32_t v[4];
    if constexpr (WHOLE) {
        const u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(m, row + (block - q), 0, kCached);
        const uint32_t two = 0x0C0C0400u + q * 0x0101u;  // byte q of either word
        uint32_t s = __builtin_amdgcn_perm(w[1], w[0], two) | __builtin_amdgcn_perm(w[3], w[2], two) << 16;
        // the words past a row's end are the next row's
        const uint32_t left = blocks - min(blocks, block), here = min((left + 3) / 4, 4u);
        return here == 4 ? s : s & ((1u << (8 * here)) - 1);
    }
#pragma unroll
    for (uint32_t b = 0; b < 4; ++b) v[b] = __builtin_amdgcn_raw_buffer_load_b8(m, block + 4 * b < blocks ? row + block + 4 * b : kNowhere, 0, kCached);
    return v[0] | v[1] << 8 | v[2] << 16 | v[3] << 24;
}

// The scales of blocks block and block + 4, block being q (0 .. 3) past a multiple of 8.
template <bool WHOLE>
__device__ __forceinline__ uint32_t pair_scales(row_t m, uint32_t row, uint32_t block, uint32_t q, uint32_t blocks) {
    if constexpr (WHOLE) {
        const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(m, row + (block - q), 0, kCached);
        const uint32_t s = __builtin_amdgcn_perm(w[1], w[0], 0x0C0C0400u + q * 0x0101u);
        return block + 4 < blocks ? s : block < blocks ? s & 255 : 0;            // the words past a row's end are the next row's
    }
    uint32_t v[2];
#pragma unroll
    for (uint32_t b = 0; b < 2; ++b) v[b] = __builtin_amdgcn_raw_buffer_load_b8(m, block + 4 * b < blocks ? row + block + 4 * b : kNowhere, 0, kCached);
    return v[0] | v[1] << 8;
}

template <int N>
using Int = std::integral_constant<int, N>;

}  // namespace fluxmoe
