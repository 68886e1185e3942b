// Which kernel a product with experts in 4 bits, or its gradient, runs: host arithmetic on sizes, strides and alignment, apart from HIP
// so that the tests can ask it, too, which kernel a call of theirs gets.
#pragma once

#include <algorithm>
#include <cstdint>

namespace fluxmoe {

struct MxCall {
    uint64_t cap;                            // rows of the matrix
    uint32_t E, N, K;
    uint64_t row_stride, row_scales_stride;  // bytes; for the gradient those of d_out, and none
    bool mx_rows;
    bool rows_vec;                           // rows at 16-byte addresses
    bool w_words, row_words;                 // scales of each weight row, and of each row in 4 bits, begin at 4-byte addresses
};

enum MxKernel : uint32_t { kMxStream, kMxStrip, kMxWide };
struct MxChoice {
    MxKernel kernel;
    uint32_t rows, outs;                     // a workgroup's tile (strips: of each wavefront's outputs); columns for the gradient
    uint32_t waves;
    bool vec, whole;                         // rows by 16-byte pieces at their addresses; scales by words
};

constexpr uint32_t kMxWideOuts = 256;

// Tiles of `size` rows that the groups can have: full ones and one unfinished one for each expert that has rows.
inline uint64_t mx_most_tiles(const MxCall& c, uint32_t size) { return c.cap / size + std::min<uint64_t>(c.cap, c.E); }
// 64 rows' places, counted from the first one's, within 31 bits
inline bool mx_near_rows(const MxCall& c) { return c.row_stride < (1u << 24) && (!c.mx_rows || c.row_scales_stride < (1u << 24)); }
// The wide tiles' places within 31 bits, and a launch of less than 2^31 threads
inline bool mx_wide_takes(const MxCall& c, uint32_t outs) {
    return c.row_stride < (1u << 23) && mx_most_tiles(c, 128) * ((uint64_t(outs) + kMxWideOuts - 1) / kMxWideOuts + 8) < (1u << 21) &&
           (!c.mx_rows || (c.rows_vec && c.row_scales_stride < (1u << 22)));
}
// Workgroups of the wide tiles of `rows` rows that a call is expected to have: an expert's last tile is half full
inline uint64_t mx_wide_workgroups(const MxCall& c, uint32_t rows, uint32_t outs) {
    return (c.cap / rows + std::min<uint64_t>(c.cap, c.E) / 2) * ((uint64_t(outs) + kMxWideOuts - 1) / kMxWideOuts);
}

// Outputs to a wavefront of a strip
constexpr uint32_t mx_strip_outs(bool mx_rows, uint32_t rows) { return mx_rows || rows == 32 ? 64 : 32; }

// Few rows, at 16-byte addresses not too far apart: side by side in strips, or a quarter of the columns to each wavefront. Times in us, 16-bit
// outputs, even routing but for 512 experts:
//   rows in 4 bits, side by side / quarters: 512 columns (512 experts, 900 tokens) 88 / 203, 1536 (160, 256) 143 / 167,
//   2048 (512, 256) 100 / 106, 4096 (8, 64) 154 / 134, 5120 (160, 16) 151 / 116: long rows are better read a whole piece at a time, and
//   there are more workgroups;
//   BF16 rows, which quarters fetch for every 64 outputs: 1536 (160, 256) 153 / 253, 5120 (160, 16) 145 / 156;
//   BF16 rows, 32 / 64 outputs to a wavefront: one tile of rows 153 / 159 (1536), 145 / 155 (5120), two 176 / 171.
// Where the workgroups would be few, narrow ones with a quarter each (one token of 512 experts, 2048 columns, 1024 outputs 7.7); 64 rows have
// strips only.
inline MxChoice mx_choose_few(const MxCall& c, uint32_t rows) {
    const uint64_t tiles = std::max<uint64_t>(c.cap / rows, std::min<uint64_t>(c.cap, c.E));
    const uint32_t strip = mx_strip_outs(c.mx_rows, rows);
    const bool whole = c.w_words && (!c.mx_rows || c.row_words);
    if (rows == 64 || ((!c.mx_rows || c.K <= 2048) && tiles * (c.N / (4 * strip)) >= 448)) return {kMxStrip, rows, strip, 4, true, whole};
    return {kMxStream, rows, tiles * (c.N / 64) >= 512 ? 64u : 16u, 4, true, whole};
}

// Two 16-row tiles of rows to a workgroup from this many rows for each expert on, on average: some experts have more than 16 then, and
// their weights are read once (8 experts of 16 rows, 4096 columns, 28672 outputs: 156 -> 133 us, rows in 4 bits 134 -> 111; 12.8 rows level).
constexpr uint32_t kMxTwoTiles = 9;
// and for the gradient, where they cost a wavefront to a SIMD (one / two, us: 512 experts, 10 rows, 2048 columns 149 / 164, 160 experts, 13 rows, 5120
// columns 307 / 283, 512 experts, 17 rows 100 / 91, 20 rows 466 / 304)
constexpr uint32_t kMxTwoTilesGrad = 12;

// The wide tiles take over where the matrix cores bound the call, by the rows to an expert on average. Times in us, streamed / wide tiles
// of 128 rows / of 256, 160 experts of 1536 columns and 5120 outputs (and turned round for the gradient):
//   rows           26               40               60               120             200
//   4 bits         151 /  - / 207   159 /  - / 216   180 /  - / 224   279 /  - / 254  433 /  - / 311      (80: 246 / 234)
//   BF16           171 / 215 / 278  235 / 252 / 288  292 / 269 / 308    - / 409 / 408   - / 631 / 558
//   gradient       197 / 276 / 346  303 / 293 / 355  379 / 354 / 386    - / 504 / 447   - / 788 / 568  (35: 279 / 291)
// and where they are enough for the CUs: 8 experts, 96 rows, 4096 outputs of 14336 columns 152 / 186 / 207 with BF16 rows; of 256
// columns, 1024 outputs 256 rows in 4 bits 8.3 /  - / 12.1, the gradient of 1024 rows 24 /  - / 31, of 28672 outputs
// and 4096 columns 40 rows 256 / 305 /  - , 56 rows 303 / 334 /  - , 64 rows 453 / 392 /  - .  Tiles of 128 rows
// also where those of 256 would be two rounds with the last one far from full (BF16, 128 / 256; same layer: 512 rows 527 / 598, 700 rows
// 591 / 620, 1000 rows 877 / 869; 28672 outputs, 300 rows 595 / 551), for the gradient where they are one round (28672 outputs of 4096
// columns: 150 rows 447 / 478, 300 rows 877 / 630).
inline MxChoice mx_choose_product(const MxCall& c) {
    const uint64_t per_expert = c.cap / c.E;
    if (c.mx_rows) {
        if (per_expert > 64 && mx_wide_workgroups(c, 256, c.N) >= 96 && mx_wide_takes(c, c.N))
            return {kMxWide, 256, kMxWideOuts, 8, true, c.w_words && c.row_words};
    } else if (per_expert > 48 && mx_wide_workgroups(c, 128, c.N) >= 176 && mx_wide_takes(c, c.N)) {
        // (256 rows that come through registers are more than there are)
        const bool half = per_expert <= 112 || mx_wide_workgroups(c, 256, c.N) < 512 || !c.rows_vec;
        return {kMxWide, half ? 128u : 256u, kMxWideOuts, 8, c.rows_vec, c.rows_vec && c.w_words};
    }
    if (!c.rows_vec || !mx_near_rows(c)) return {kMxStream, 32, 64, 4, false, false};
    return mx_choose_few(c, per_expert > 32 ? 64 : per_expert >= kMxTwoTiles ? 32 : 16);
}

inline MxChoice mx_choose_grad(const MxCall& c) {
    const uint64_t per_expert = c.cap / c.E;
    const bool vec = c.rows_vec && c.N % 8 == 0;
    // Rows through registers make longer steps, streamed / wide: 160 experts of 5119 outputs and 1536 columns, 100 rows each 704 / 985, 260 rows
    // 1644 / 2390, 400 rows 2470 / 3108; 8 experts of 4095 outputs and 14336 columns, 100 rows 301 / 298, 200 rows 540 / 543, 260 rows 688 / 675,
    // 400 rows 1020 / 844.
    if (per_expert > (vec ? 32 : 256) && mx_wide_workgroups(c, 128, c.K) >= 128 && mx_wide_takes(c, c.K) && c.N >= 8) {
        const bool half = (vec && per_expert <= 80) || mx_wide_workgroups(c, 128, c.K) <= 256;
        return {kMxWide, half ? 128u : 256u, kMxWideOuts, 8, vec, vec && c.w_words};
    }
    const uint32_t rows = per_expert >= kMxTwoTilesGrad ? 32 : 16;
    // Eight wavefronts where there are fewer workgroups than CUs. Four / eight, us: 20 workgroups (one token of 512 experts, 512 columns)
    // 15.9 / 13.7, 128 (8 experts, 16 rows, 4096 columns of 28672 outputs) 290 / 221, 448 (8 experts, 14336 columns, 4 rows) 66 / 71,
    // 960 (160 experts, 1536 columns) 3 rows 140 / 137, 13 rows 149 / 165, 3200 (160 experts, 5120 columns, 13 rows) 283 / 329.
    const uint64_t workgroups = std::max<uint64_t>(c.cap / rows, std::min<uint64_t>(c.cap, c.E)) * ((uint64_t(c.K) + 255) / 256);
    return {kMxStream, rows, 256, workgroups < 256 ? 8u : 4u, vec, false};
}

}  // namespace fluxmoe
