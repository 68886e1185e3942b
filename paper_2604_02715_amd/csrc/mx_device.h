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

// Rows of expert e that lie within the matrix, whatever offsets and counts hold, and the first of them.
__device__ __forceinline__ uint32_t rows_of(const MxProductArgs& a, uint32_t e, uint32_t& first) {
    const int32_t c = a.counts[e], o = a.offsets[e];
    first = uint32_t(o);
    return c <= 0 || o < 0 || uint32_t(o) >= a.cap ? 0 : min(uint32_t(c), a.cap - uint32_t(o));
}

// Tile number `wanted` of the experts' groups in their order, `size` rows to a tile; rows 0 where there are no more.  All threads of the
// workgroup; a thread adds up neighbouring experts and keeps what it read of up to four.  s: kTileWords of LDS.
constexpr uint32_t kTileWords = 16;
template <uint32_t THREADS>
__device__ __forceinline__ Tile find_tile(const MxProductArgs& a, uint32_t size, uint32_t wanted, uint32_t* s) {
    constexpr uint32_t kFound = THREADS / 64, kKept = 4;
    static_assert(kFound + 3 <= kTileWords, "wavefronts' sums and the tile");
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t per = (a.E + THREADS - 1) / THREADS, from = min(tid * per, a.E), to = min(from + per, a.E);
    uint32_t rows[kKept], first[kKept], mine = 0;
#pragma unroll
    for (uint32_t i = 0; i < kKept; ++i) {
        rows[i] = first[i] = 0;
        if (from + i < to) rows[i] = rows_of(a, from + i, first[i]);
    }
#pragma unroll
    for (uint32_t i = 0; i < kKept; ++i) mine += (rows[i] + size - 1) / size;
    for (uint32_t e = from + kKept; e < to; ++e) {
        uint32_t at;
        mine += (rows_of(a, e, at) + size - 1) / size;
    }
    uint32_t upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t below = __shfl_up(upto, d);
        if (lane >= uint32_t(d)) upto += below;
    }
    __syncthreads();                                     // the last tile's readers are done with s
    if (lane == 63) s[wave] = upto;
    if (tid == 0) s[kFound + 2] = 0;
    __syncthreads();
    for (uint32_t w = 0; w < wave; ++w) upto += s[w];
    uint32_t before = upto - mine;
    if (wanted >= before && wanted < upto) {
        auto found = [&](uint32_t e, uint32_t n, uint32_t at) __attribute__((always_inline)) {
            const uint32_t tiles = (n + size - 1) / size, skip = (wanted - before) * size;
            const bool here = wanted >= before && wanted < before + tiles;
            if (here) {
                s[kFound] = e;
                s[kFound + 1] = at + skip;
                s[kFound + 2] = min(size, n - skip);
            }
            before += tiles;
            return here;
        };
#pragma unroll
        for (uint32_t i = 0; i < kKept; ++i) found(from + i, rows[i], first[i]);
        for (uint32_t e = from + kKept; e < to; ++e) {
            uint32_t at;
            const uint32_t n = rows_of(a, e, at);
            if (found(e, n, at)) break;
        }
    }
    __syncthreads();
    Tile t;
    t.expert = __builtin_amdgcn_readfirstlane(s[kFound]);
    t.first = __builtin_amdgcn_readfirstlane(s[kFound + 1]);
    t.rows = __builtin_amdgcn_readfirstlane(s[kFound + 2]);
    return t;
}

// Item number `item` of a launch over tiles of `strips` strips each: (tile, strip).  Nearly always within 32 bits, where a division is a
// tenth as long.
struct Item {
    uint32_t tile, strip;
};
__device__ __forceinline__ Item item_at(uint64_t item, uint32_t strips) {
    Item i;
    i.tile = item >> 32 ? uint32_t(item / strips) : uint32_t(item) / strips;
    i.strip = uint32_t(item - uint64_t(i.tile) * strips);
    return i;
}

// `records` bytes from `base` on, by offset: reads past them give 0
__device__ __forceinline__ row_t bytes_at(const void* base, uint64_t offset, uint32_t records) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(base) + offset), 0, int(records), 0x00020000);
}
constexpr uint32_t kNowhere = 0x7FFFFFF0u;               // an offset past any resource's records
// 16 bytes, or 0 where there are none
__device__ __forceinline__ u32x4 piece_at(row_t m, bool there, uint32_t offset) {
    return __builtin_amdgcn_raw_buffer_load_b128(m, there ? offset : kNowhere, 0, kCached);
}

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
