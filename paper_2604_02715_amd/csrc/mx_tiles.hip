// The product with experts' weights in 4-bit floating point where an expert has many rows: bound by the matrix cores.
//
// A workgroup's tile is 256 rows by 256 outputs, eight wavefronts as 4 (rows) x 2 (outputs), two to a SIMD, 64 x 128 each as
// 2 x 4 tiles of the 32x32 matrix instructions.  (Rows in 4 bits, 8 experts, 2048 rows of 14336 columns each, 4096 outputs: 510 us, 3.8
// PFLOP/s, on zeros 451; four wavefronts of 128 x 128, which read a third less from LDS, 541.)  Both operands go from memory straight to
// LDS, as they are: rows of 128 bytes, which are 256 columns of codes (a superblock: eight blocks of 32, a 16-byte piece each) or 64
// columns of BF16.  A load fills 1 KiB of LDS without gaps, so instead of padding, the lane that fills position p of a row fetches piece
// p ^ ((row >> 1) & 7): 16 neighbouring rows' pieces of one number then lie in 64 different banks.
// Which columns a matrix instruction's k numbers stand for is free as long as both operands agree.  Lanes 0..31 take the first half
// of a superblock's blocks and lanes 32..63 the second, so that a lane's scales of a superblock are four neighbouring bytes.
#include "mx_device.h"

namespace fluxmoe {
namespace {

constexpr uint32_t kTile = kMxWideOuts;
constexpr int kStage = 32768;                            // 256 rows of 128 bytes
constexpr uint32_t kThreads = 512;
constexpr uint32_t kScaleRow = 260;                      // words between the gradient's scales of two blocks of columns: in different banks
constexpr int kScaleStage = 8 * kScaleRow * 4;

// Where a workgroup's tile lies.  Workgroups go to the eight XCDs in turn; up to 32 that run on one at a time take a super-tile of
// 1 << sm_log2 row tiles by 1 << sn_log2 strips, whose rows and weights they share in that XCD's L2.  Smaller ones where there would be fewer
// than 32, of which one XCD may have two and another one: 1500 rows of one expert, 4096 outputs of 5120 columns, gradient 132 -> 72 us, 3000
// rows in 4 bits of 2048 columns, 5120 outputs 42 -> 24, 8 experts, 512 rows in 4 bits 233 -> 220; up to 3 % slower at others.  With 16 for the
// limit the first two stay as they were.
constexpr uint32_t kFewSupers = 32, kLeastSuper = 2;     // (log2 of the smallest one's tiles)
struct WideGrid {
    uint32_t strips, sn_log2, sm_log2, row_tiles, total;
    __host__ WideGrid(const MxProductArgs& a, uint32_t rows, uint32_t outs) {
        const uint64_t row_tiles_most = a.cap / rows + (a.cap < a.E ? a.cap : a.E);
        strips = (outs + kTile - 1) / kTile;
        row_tiles = uint32_t(row_tiles_most);
        uint64_t supers = 0;
        for (uint32_t size_log2 = 5; size_log2 >= kLeastSuper; --size_log2) {
            sn_log2 = 0;
            while (sn_log2 < 3 && sn_log2 + 1 < size_log2 && (1u << sn_log2) < strips) ++sn_log2;
            sm_log2 = size_log2 - sn_log2;
            supers = ((row_tiles_most + (1u << sm_log2) - 1) >> sm_log2) * ((strips + (1u << sn_log2) - 1) >> sn_log2);
            if (supers >= kFewSupers) break;
        }
        total = uint32_t(((supers + 7) / 8 * 8) << (sn_log2 + sm_log2));
    }
    __device__ __forceinline__ bool locate(uint32_t L, uint32_t& row_tile, uint32_t& strip) const {
        const uint32_t sn = 1u << sn_log2, n_sn = (strips + sn - 1) >> sn_log2, size_log2 = sn_log2 + sm_log2;
        const uint32_t xcd = L % 8u, jj = L / 8u, st = (jj >> size_log2) * 8u + xcd, within = jj & ((1u << size_log2) - 1);
        row_tile = (st / n_sn << sm_log2) + (within >> sn_log2);
        strip = (st % n_sn << sn_log2) + (within & (sn - 1));
        return strip < strips && row_tile < row_tiles;
    }
};

// 16 (4) bytes to each lane's place of the KiB (256 bytes) at lds_addr, from its offset to the wavefront's base.  Assembly on purpose: with
// the compiler's builtin every later LDS read waits for all loads into LDS that are under way, as it cannot tell that they fill another
// stage.  The waits are those written below, ahead of the barriers.  M0 holds the destination; the compiler has reserved it, so its value
// is put back.
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t offset, uint32_t lds_addr) {
    uint32_t saved;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved) : "v"(offset), "s"(base), "s"(lds_addr) : "memory");
}
__device__ __forceinline__ void load_word_to_lds(const void* base, uint32_t offset, uint32_t lds_addr) {
    uint32_t saved;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved) : "v"(offset), "s"(base), "s"(lds_addr) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory"); }

// What is multiplied: rows in 4 bits or BF16 by weights, summed over their columns; or for the gradient BF16 rows of d_out by weights turned
// round, summed over the outputs.  "Columns" below are those of the result, n0 the tile's first.
enum Mode { kMxRows, kBf16Rows, kGradRows };

constexpr int kRawScales = kTile * 8;                    // bytes of a superblock's scales
constexpr int scale_bytes(Mode mode) { return mode == kMxRows ? 4 * kRawScales : 2 * kRawScales + (mode == kGradRows ? 2 * kScaleStage : 0); }

// RT: 32-row groups of a wavefront, 2 for tiles of 256 rows and 1 for 128, whose columns are fetched four steps ahead in as much LDS as two
// take there.  WHOLE: scales are read four at a time.  VEC: the rows are whole 16-byte pieces at 16-byte addresses; others come through
// registers.
template <Mode MODE, int RT, bool WHOLE, bool VEC, typename OUT>
__global__ __launch_bounds__(kThreads) void mx_wide_kernel(MxProductArgs a, WideGrid grid) {
    constexpr bool MX = MODE == kMxRows, GRAD = MODE == kGradRows;
    static_assert(VEC || (!MX && !WHOLE), "BF16 rows at any address, scales too");
    constexpr uint32_t kRows = 128 * RT;
    constexpr int kXStages = MX ? 2 : 4 / RT, kXLoads = 2 * RT;      // and a wavefront's loads of a stage
    constexpr uint32_t kXStage = kRows * 128;
    // rows' stages, weights' two stages, scales twice (for the gradient as the conversion takes them, then as they come; for rows in 4 bits the
    // weights', then the rows'), find_tile's words
    extern __shared__ __align__(16) uint8_t lds[];
    uint32_t row_tile, strip;
    if (!grid.locate(blockIdx.x, row_tile, strip)) return;
    const Tile t = find_tile<kThreads>(a, kRows, row_tile, reinterpret_cast<uint32_t*>(lds + 4 * kStage + scale_bytes(MODE)));
    if (t.rows == 0) return;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t wm = wave >> 1, wn = wave & 1, q = lane & 31, h = lane >> 5;
    const uint32_t n0 = strip * kTile, blocks = a.K / kMxBlock;
    const uint32_t outs = GRAD ? a.K : a.N, supers = GRAD ? (a.N + 255) / 256 : (blocks + 7) / 8;
    const uint32_t lds_base = uint32_t(uintptr_t((__attribute__((address_space(3))) void*)lds));

    // What the lane fetches: four KiB of weights to a wavefront and stage, rows 8 (4 wave + i) + lane / 8, and as many or half of rows.
    const uint8_t* const x_base = static_cast<const uint8_t*>(a.rows) + uint64_t(t.first) * a.row_stride;
    const uint8_t* const w_base = a.w + (uint64_t(t.expert) * a.N + (GRAD ? 0 : n0)) * (a.K / 2) + (GRAD ? n0 / 2 : 0);
    uint32_t x_off[kXLoads], w_off[4];                       // of the rows
#pragma unroll
    for (int i = 0; i < kXLoads; ++i) x_off[i] = min(8 * (wave * kXLoads + i) + (lane >> 3), t.rows - 1) * uint32_t(a.row_stride);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t row = 8 * (wave * 4 + i) + (lane >> 3);
        w_off[i] = GRAD ? row : min(row, a.N - 1 - n0) * (a.K / 2);
    }
    auto piece_of = [&](int i) __attribute__((always_inline)) { return (lane & 7) ^ ((4 * (i & 1) + (lane >> 4)) & 7); };
    // Past the end of a row its last block is fetched in place of those that are missing, whose weights become 0 ahead of their products.
    auto fetch_w = [&](int i, uint32_t super) __attribute__((always_inline)) {
        if constexpr (GRAD) {                                // 256 outputs of the strip's eight blocks of columns
            load_to_lds(w_base + uint64_t(super) * 256 * (a.K / 2),
                        min(w_off[i], a.N - 1 - super * 256) * (a.K / 2) + min((lane & 7) ^ (4 * (wave & 1)), (a.K - n0) / kMxBlock - 1) * 16,
                        lds_base + (2 + (super & 1)) * kStage + (wave * 4 + i) * 1024);
            return;
        }
        load_to_lds(w_base + uint64_t(super) * 128, w_off[i] + min(piece_of(i), blocks - 1 - super * 8) * 16,
                    lds_base + (2 + (super & 1)) * kStage + (wave * 4 + i) * 1024);
    };
    // the rows' codes of a superblock, or BF16 columns of its blocks s and 4 + s, into stage `to`
    auto fetch_x = [&](int i, uint32_t super, uint32_t s, uint32_t to) __attribute__((always_inline)) {
        if constexpr (GRAD) {                                // 64 outputs of a superblock's 256
            load_to_lds(x_base, x_off[i] + min(super * 32 + s * 8 + piece_of(i), a.N / 8 - 1) * 16, lds_base + to * kXStage + (wave * kXLoads + i) * 1024);
            return;
        }
        const uint32_t block = min(MX ? piece_of(i) : s + 4 * (piece_of(i) >> 2), blocks - 1 - super * 8);
        load_to_lds(x_base + uint64_t(super) * (MX ? 128 : 512), x_off[i] + block * (MX ? 16 : 64) + (MX ? 0 : (piece_of(i) & 3) * 16),
                    lds_base + to * kXStage + (wave * kXLoads + i) * 1024);
    };

    // (not VEC) The same pieces into registers, to be put where the loads into LDS would put them in the next step.  0 past a row's end: a piece
    // that reaches beyond it is the row's last eight numbers, moved.  No branches: between matrix instructions they would be moved behind them.
    u32x4 held[VEC ? 1 : kXLoads];
    auto hold_x = [&](int i, uint32_t super, uint32_t s) __attribute__((always_inline)) {
        const uint32_t sum = GRAD ? a.N : a.K;
        const uint32_t column =
            GRAD ? super * 256 + s * 64 + piece_of(i) * 8 : (super * 8 + s + 4 * (piece_of(i) >> 2)) * 32 + (piece_of(i) & 3) * 8;
        const uint32_t from = min(column, sum - 8), beyond = min(column - from, 8u);
        uint64_t v[2];
        __builtin_memcpy(v, x_base + x_off[i] + from * 2, 16);
        const uint64_t low = beyond >= 4 ? v[1] : v[0], high = beyond >= 4 ? 0 : v[1];
        const uint32_t by = 16 * (beyond & 3);
        const uint64_t a0 = beyond == 8 ? 0 : (low >> by) | ((high << 1) << (63 - by)), a1 = high >> by;
        held[i] = u32x4{uint32_t(a0), uint32_t(a0 >> 32), uint32_t(a1), uint32_t(a1 >> 32)};
    };
    auto put_x = [&](uint32_t to) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kXLoads; ++i) *reinterpret_cast<u32x4*>(lds + to * kXStage + (wave * kXLoads + i) * 1024 + lane * 16) = held[i];
    };

    const row_t ws_at = bytes_at(a.ws, (uint64_t(t.expert) * a.N + n0) * blocks, GRAD ? 0 : min(kTile, a.N - n0) * blocks);
    const row_t xs_at = bytes_at(a.row_scales, uint64_t(t.first) * a.row_scales_stride,
                                 MX ? (t.rows - 1) * uint32_t(a.row_scales_stride) + blocks : 0);
    auto w_scales = [&](int j, uint32_t super) __attribute__((always_inline)) {
        return four_scales<WHOLE>(ws_at, min(wn * 128 + j * 32 + q, a.N - 1 - n0) * blocks, super * 8 + 4 * h, blocks);
    };
    auto x_scales = [&](int i, uint32_t super) __attribute__((always_inline)) {
        return four_scales<WHOLE>(xs_at, min((wm + 4 * i) * 32 + q, t.rows - 1) * uint32_t(a.row_scales_stride), super * 8 + 4 * h, blocks);
    };

    f32x16 acc[RT][4];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

    // Piece 4 h + ks of the lane's rows: the rows of a wavefront's 32 x 32 tiles lie 32 apart, which leaves the place of a piece as it is.
    uint32_t at[4];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) at[ks] = q * 128 + 16 * ((4 * h + ks) ^ ((q >> 1) & 7));
    auto read = [&](uint32_t addr) __attribute__((always_inline)) { return *reinterpret_cast<const u32x4*>(lds + addr); };
    auto read_x = [&](int i, int ks, uint32_t stage) __attribute__((always_inline)) { return read(at[ks] + (stage * kXStage + wm * 4096) + i * 16384); };
    auto read_w = [&](int j, int ks, uint32_t stage) __attribute__((always_inline)) { return read(at[ks] + ((2 + stage) * kStage + wn * 16384) + j * 4096); };

    // The next superblock's scales as they come: two words of each row, one to a lane.  (Fetched by the lanes that multiply by them, a word from
    // each of 32 rows at a time, they were a third of a step: 16382 rows in 4 bits of 14336 columns, 4096 outputs 822 us, through LDS 572.)
    auto fetch_words = [&](uint32_t super) __attribute__((always_inline)) {
        const uint32_t row = tid >> 1, to = lds_base + 4 * kStage + (GRAD ? 2 * kScaleStage : 0) + (super & 1) * kRawScales + wave * 256;
        const uint32_t first = GRAD ? super * 256 : n0, block = min((GRAD ? n0 / kMxBlock : super * 8) + 4 * (tid & 1), blocks - 4);
        if constexpr (MX)
            load_word_to_lds(a.row_scales + uint64_t(t.first) * a.row_scales_stride, min(row, t.rows - 1) * uint32_t(a.row_scales_stride) + block,
                             to + 2 * kRawScales);
        load_word_to_lds(a.ws + (uint64_t(t.expert) * a.N + first) * blocks, min(row, a.N - 1 - first) * blocks + block, to);
    };
    // the columns of a tile's first steps
    auto first_rows = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < kXStages; ++s) {
#pragma unroll
            for (int i = 0; i < kXLoads; ++i) {
                if constexpr (VEC) fetch_x(i, 0, s, s);
                else hold_x(i, 0, s);
            }
            if constexpr (!VEC) put_x(s);
        }
        wait_loads<VEC ? (kXStages - 1) * kXLoads : 0>();
    };
    // Ahead of the barrier of step s the loads that may still be under way: those issued behind the next step's columns, and behind
    // the next superblock's weights where that is about to begin.  A step issues columns in its last sub-step; steps 0 and 1 issue two loads of
    // weights each in their first, step 0 a word of scales before those.
    auto wait_step = [&](auto S, auto MORE) __attribute__((always_inline)) {
        constexpr int s = decltype(S)::value, words = WHOLE ? 1 : 0;
        if constexpr (!VEC) wait_loads<0>();
        else if constexpr (decltype(MORE)::value == 0) wait_loads<RT == 2 ? 0 : s == 0 ? 4 : s == 1 ? 2 : 0>();
        else if constexpr (RT == 2) wait_loads<s == 0 ? 2 + words : s == 1 ? 2 : 0>();
        else wait_loads<s == 0 ? 6 + words : s == 3 ? 4 : 8 + words>();
    };

    // (not VEC) Behind step s's barrier its columns' stage is free: what is to lie there is fetched, and put there ahead of the next barrier.
    auto take_up = [&](auto S, auto MORE, uint32_t super) __attribute__((always_inline)) {
        constexpr int s = decltype(S)::value;
        if constexpr (!VEC && (decltype(MORE)::value != 0 || s + kXStages < 4)) {
#pragma unroll
            for (int i = 0; i < kXLoads; ++i) hold_x(i, super + (s + kXStages) / 4, (s + kXStages) % 4);
        }
    };
    auto hand_over = [&](auto S, auto MORE) __attribute__((always_inline)) {
        constexpr int s = decltype(S)::value;
        if constexpr (!VEC && s == 0) put_x(3 % kXStages);       // of the last superblock's step 3, or once more of the tile's first steps
        else if constexpr (!VEC && (decltype(MORE)::value != 0 || s - 1 + kXStages < 4)) put_x((s - 1) % kXStages);
    };

    // ACT: row groups wm, wm + 4 of the tile that have rows
    auto k_loop = [&](auto ACT) __attribute__((always_inline)) {
        constexpr int act = decltype(ACT)::value;
        if constexpr (MX) {
            // A step is a superblock, a sub-step 64 of its columns: blocks ks and 4 + ks.  Fragments of the next sub-step are read between
            // the matrix instructions; a step's one barrier lies ahead of its last sub-step, which covers the first reads from the other stage.
            uint32_t ws[4], xs[2], ws_next[4], xs_next[2];
            u32x4 fx[2][2], fw[2][4];
            auto fetch_scales = [&](uint32_t super) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < 4; ++j) ws_next[j] = w_scales(j, super);
#pragma unroll
                for (int i = 0; i < act; ++i) xs_next[i] = x_scales(i, super);
            };
            auto read_scales = [&](uint32_t super) __attribute__((always_inline)) {
                const uint8_t* from = lds + 4 * kStage + (super & 1) * kRawScales + 4 * h;
#pragma unroll
                for (int j = 0; j < 4; ++j) ws_next[j] = *reinterpret_cast<const uint32_t*>(from + (wn * 128 + j * 32 + q) * 8);
#pragma unroll
                for (int i = 0; i < act; ++i) xs_next[i] = *reinterpret_cast<const uint32_t*>(from + 2 * kRawScales + ((wm + 4 * i) * 32 + q) * 8);
            };
            auto scales_arrive = [&]() __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < 4; ++j) { asm volatile("" : "+v"(ws_next[j])); }
#pragma unroll
                for (int i = 0; i < act; ++i) { asm volatile("" : "+v"(xs_next[i])); }
            };
            auto take_scales = [&]() __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < 4; ++j) ws[j] = ws_next[j];
#pragma unroll
                for (int i = 0; i < act; ++i) xs[i] = xs_next[i];
            };
            auto read_item = [&](int n, uint32_t stage, int ks, int set) __attribute__((always_inline)) {
                if (act == 0) return;
                if (n < 4) fw[set][n] = read_w(n, ks, stage);
                else if (n - 4 < act) fx[set][n - 4] = read_x(n - 4, ks, stage);
            };
            auto sub = [&](auto KS, auto NEXT, auto LOAD, uint32_t stage, uint32_t super) __attribute__((always_inline)) {
                constexpr int ks = decltype(KS)::value, set = ks & 1;
                constexpr bool next = decltype(NEXT)::value != 0, load = decltype(LOAD)::value != 0;
                if constexpr (!next && act > 0) {           // 0 for blocks past the end; the rows' codes are finite whatever they are
                    if constexpr (WHOLE && ks == 0) {        // and so are scales
                        const bool in = super * 8 + 4 * h < blocks;
#pragma unroll
                        for (int j = 0; j < 4; ++j) ws[j] = in ? ws[j] : 0;
#pragma unroll
                        for (int i = 0; i < act; ++i) xs[i] = in ? xs[i] : 0;
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int c = 0; c < 4; ++c) fw[set][j][c] = super * 8 + 4 * h + ks < blocks ? fw[set][j][c] : 0;
                }
#pragma unroll
                for (int n = 0; n < 8; ++n) {
                    const int i = n / 4, j = n % 4;
                    if (i < act) {
                        const i32x8 xv = {int(fx[set][i][0]), int(fx[set][i][1]), int(fx[set][i][2]), int(fx[set][i][3]), 0, 0, 0, 0};
                        const i32x8 wv = {int(fw[set][j][0]), int(fw[set][j][1]), int(fw[set][j][2]), int(fw[set][j][3]), 0, 0, 0, 0};
                        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(xv, wv, acc[i][j], 4, 4, ks, int(xs[i]), ks, int(ws[j]));
                    }
                    if (ks < 3) {
                        if (n < 6) read_item(n, stage, ks + 1, set ^ 1);
                    } else {
                        if (next && n < 6) read_item(n, stage ^ 1, 0, set ^ 1);
                        if (WHOLE && next && n == 6) read_scales(super + 1);
                        if (WHOLE && load && n == 0) fetch_words(super + 2);
                        if (load) {
                            if (n & 1) fetch_w(n / 2, super + 2);
                            else fetch_x(n / 2, super + 2, 0, stage);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            auto step = [&](auto NEXT, auto LOAD, uint32_t super) __attribute__((always_inline)) {
                const uint32_t stage = super & 1;
                if constexpr (!WHOLE && decltype(NEXT)::value != 0) fetch_scales(super + 1);
                sub(Int<0>{}, NEXT, LOAD, stage, super);
                sub(Int<1>{}, NEXT, LOAD, stage, super);
                sub(Int<2>{}, NEXT, LOAD, stage, super);
                wait_loads<0>();
                if constexpr (!WHOLE) scales_arrive();
                __syncthreads();
                sub(Int<3>{}, NEXT, LOAD, stage, super);
                take_scales();
            };
            if constexpr (WHOLE) fetch_words(0);
            else fetch_scales(0);
#pragma unroll
            for (int i = 0; i < 4; ++i) { fetch_w(i, 0); fetch_x(i, 0, 0, 0); }
            if constexpr (!WHOLE) {
                wait_loads<0>();
                scales_arrive();
            }
            if (supers > 1) {
                if constexpr (WHOLE) fetch_words(1);
#pragma unroll
                for (int i = 0; i < 4; ++i) { fetch_w(i, 1); fetch_x(i, 1, 0, 1); }
                wait_loads<8 + (WHOLE ? 2 : 0)>();
            } else {
                wait_loads<0>();
            }
            __syncthreads();
            if constexpr (WHOLE) read_scales(0);
            take_scales();
#pragma unroll
            for (int n = 0; n < 6; ++n) read_item(n, 0, 0, 0);
            uint32_t super = 0;
            for (; super + 2 < supers; ++super) step(Int<1>{}, Int<1>{}, super);
            if (super + 1 < supers) step(Int<1>{}, Int<0>{}, super++);
            step(Int<0>{}, Int<0>{}, super);
        } else if constexpr (GRAD) {
            // A superblock is 256 outputs, a step 64 of them, a sub-step eight of either half of those.  Lane q has four neighbouring columns,
            // a 32 x 32 tile every fourth one: two bytes of codes of each of eight outputs become the tiles' fragments by a conversion and a
            // permutation to each two numbers.  The scales lie in LDS as the conversion takes them, a block's outputs one after the other.
            uint32_t scales_next = 0;
            u32x4 fx[2][RT], fw[2][4], sc[2];
            uint32_t raw[8], pair[8][2];
            const uint32_t raw_at = 2 * kStage + h * 4096 + 16 * ((wn * 4 + q / 8) ^ (4 * h)) + 2 * (q & 7);
            const uint32_t sc_at = 4 * kStage + ((wn * 4 + q / 8) * kScaleRow + 32 * h) * 4;
            auto fetch_scales = [&](uint32_t super) __attribute__((always_inline)) {
                const row_t m = bytes_at(a.ws, (uint64_t(t.expert) * a.N + super * 256) * blocks, min(a.N - super * 256, 256u) * blocks);
                scales_next = four_scales<WHOLE>(m, (tid >> 1) * blocks, n0 / kMxBlock + 4 * (tid & 1), blocks);
            };
            auto put_scales = [&](uint32_t super) __attribute__((always_inline)) {
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    *reinterpret_cast<float*>(lds + 4 * kStage + (super & 1) * kScaleStage + ((4 * (tid & 1) + b) * kScaleRow + (tid >> 1)) * 4) =
                        scale_operand((scales_next >> (8 * b)) & 255);
            };
            auto read_raw = [&](uint32_t super, int s, int ks) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    raw[j] = *reinterpret_cast<const uint16_t*>(lds + (raw_at + (super & 1) * kStage) + (64 * s + 8 * ks + j) * 128);
#pragma unroll
                for (int j = 0; j < 2; ++j) sc[j] = read(sc_at + (super & 1) * kScaleStage + (64 * s + 8 * ks + 4 * j) * 4);
            };
            auto convert = [&](int j) __attribute__((always_inline)) {
                const float scale = __uint_as_float(sc[j / 4][j % 4]);
                pair[j][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(raw[j], scale, 0));
                pair[j][1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(raw[j], scale, 1));
            };
            auto turn = [&](int set, int c) __attribute__((always_inline)) {
#pragma unroll
                for (int d = 0; d < 4; ++d)
                    fw[set][c][d] = __builtin_amdgcn_perm(pair[2 * d + 1][c / 2], pair[2 * d][c / 2], (c & 1) ? 0x07060302u : 0x05040100u);
            };
            auto raw_scales = [&](uint32_t super) __attribute__((always_inline)) {
                if constexpr (WHOLE)
                    scales_next = *reinterpret_cast<const uint32_t*>(lds + 4 * kStage + 2 * kScaleStage + (super & 1) * kRawScales + tid * 4);
                else asm volatile("" : "+v"(scales_next));
            };
            if constexpr (WHOLE) fetch_words(0);
            else fetch_scales(0);
#pragma unroll
            for (int i = 0; i < 4; ++i) fetch_w(i, 0);
            first_rows();
            raw_scales(0);                                   // what this wavefront fetched itself
            put_scales(0);
            __syncthreads();
            if constexpr (act > 0) {
                read_raw(0, 0, 0);
#pragma unroll
                for (int i = 0; i < act; ++i) fx[0][i] = read_x(i, 0, 0);
#pragma unroll
                for (int j = 0; j < 8; ++j) convert(j);
#pragma unroll
                for (int c = 0; c < 4; ++c) turn(0, c);
            }
            auto step = [&](auto S, auto MORE, uint32_t super) __attribute__((always_inline)) {
                constexpr int s = decltype(S)::value;
                constexpr bool load_w = decltype(MORE)::value != 0, next = load_w || s < 3, load = load_w || s + kXStages < 4;
                constexpr uint32_t stage = s % kXStages, stage_next = (s + 1) % kXStages;
                auto sub = [&](auto KS) __attribute__((always_inline)) {
                    constexpr int ks = decltype(KS)::value, set = ks & 1;
                    constexpr bool ahead = act > 0 && (ks < 3 || next);
                    if constexpr (!load_w && act > 0) {      // 0 past the last output, on both sides
                        const uint32_t mask = super * 256 + 64 * s + 32 * h + 8 * ks < a.N ? ~0u : 0u;
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) fw[set][j][c] &= mask;
#pragma unroll
                            for (int i = 0; i < act; ++i) fx[set][i][c] &= mask;
                        }
                    }
                    if constexpr (ahead) {
                        if (ks < 3) read_raw(super, s, ks + 1);
                        else read_raw(super + (s == 3), (s + 1) % 4, 0);
                    }
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int n = 0; n < 8; ++n) {
                        const int i = n / 4, j = n % 4;
                        if (i < act)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fx[set][i]), __builtin_bit_cast(bf16x8, fw[set][j]),
                                                                               acc[i][j], 0, 0, 0);
                        if constexpr (ahead) {
                            if (n < act) fx[set ^ 1][n] = ks < 3 ? read_x(n, ks + 1, stage) : read_x(n, 0, stage_next);
                            if (n == 2 || n == 3)
#pragma unroll
                                for (int k = 0; k < 4; ++k) convert(4 * (n - 2) + k);
                            if (n >= 4) turn(set ^ 1, n - 4);
                        }
                        // the next superblock's weights, in the first two steps of this one
                        if (ks == 0 && s < 2 && (n == 3 || n == 7) && load_w) fetch_w(s * 2 + n / 4, super + 1);
                        if (VEC && ks == 3 && load && (n & 1) && n / 2 < kXLoads)
                            fetch_x(n / 2, super + (s + kXStages) / 4, (s + kXStages) % 4, stage);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                };
                if constexpr (s == 0 && load_w) {
                    if constexpr (WHOLE) fetch_words(super + 1);
                    else fetch_scales(super + 1);
                }
                sub(Int<0>{});
                sub(Int<1>{});
                sub(Int<2>{});
                hand_over(S, MORE);
                wait_step(S, MORE);
                if constexpr (s == 3 && load_w) {
                    raw_scales(super + 1);
                    put_scales(super + 1);
                }
                __syncthreads();
                take_up(S, MORE, super);
                sub(Int<3>{});
            };
            uint32_t super = 0;
            for (; super + 1 < supers; ++super) {
                step(Int<0>{}, Int<1>{}, super);
                step(Int<1>{}, Int<1>{}, super);
                step(Int<2>{}, Int<1>{}, super);
                step(Int<3>{}, Int<1>{}, super);
            }
            step(Int<0>{}, Int<0>{}, super);
            step(Int<1>{}, Int<0>{}, super);
            step(Int<2>{}, Int<0>{}, super);
            step(Int<3>{}, Int<0>{}, super);
        } else {
            // A step is 64 columns: blocks s and 4 + s of a superblock, whose codes are in LDS for its four steps.  A sub-step is eight columns
            // of both blocks; its weights are converted in the sub-step before.
            uint32_t scales[4], scales_next[4];
            float sc[4];
            u32x4 codes[4], fx[2][RT];
            bf16x8 fw[2][4];
            auto fetch_scales = [&](uint32_t super) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < 4; ++j) scales_next[j] = w_scales(j, super);
            };
            auto scales_arrive = [&]() __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(scales_next[j]));
            };
            auto take_scales = [&](uint32_t super) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint8_t* from = lds + 4 * kStage + (super & 1) * kRawScales + (wn * 128 + j * 32 + q) * 8 + 4 * h;
                    scales[j] = WHOLE ? *reinterpret_cast<const uint32_t*>(from) : scales_next[j];
                }
            };
            if constexpr (WHOLE) fetch_words(0);
            else fetch_scales(0);
#pragma unroll
            for (int i = 0; i < 4; ++i) fetch_w(i, 0);
            first_rows();
            if constexpr (!WHOLE) scales_arrive();
            __syncthreads();
            take_scales(0);
            if constexpr (act > 0) {
#pragma unroll
                for (int j = 0; j < 4; ++j) codes[j] = read_w(j, 0, 0);
#pragma unroll
                for (int i = 0; i < act; ++i) fx[0][i] = read_x(i, 0, 0);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    sc[j] = scale_operand(scales[j] & 255);
                    fw[0][j] = codes_bf16(codes[j][0], sc[j]);
                }
            }
            // MORE: another superblock follows
            auto step = [&](auto S, auto MORE, uint32_t super) __attribute__((always_inline)) {
                constexpr int s = decltype(S)::value;
                constexpr bool load_w = decltype(MORE)::value != 0, next = load_w || s < 3, load = load_w || s + kXStages < 4;
                constexpr uint32_t stage = s % kXStages, stage_next = (s + 1) % kXStages;
                auto sub = [&](auto KS) __attribute__((always_inline)) {
                    constexpr int ks = decltype(KS)::value, set = ks & 1;
                    if constexpr (!load_w && act > 0) {      // 0 for blocks past the end, on both sides: a row may hold what is not finite
                        const uint32_t mask = super * 8 + 4 * h + s < blocks ? ~0u : 0u;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const u32x4 v = __builtin_bit_cast(u32x4, fw[set][j]);
                            fw[set][j] = __builtin_bit_cast(bf16x8, u32x4{v[0] & mask, v[1] & mask, v[2] & mask, v[3] & mask});
                        }
#pragma unroll
                        for (int i = 0; i < act; ++i)
#pragma unroll
                            for (int c = 0; c < 4; ++c) fx[set][i][c] &= mask;
                    }
                    if constexpr (ks == 3) {
                        if constexpr (next && act > 0) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) codes[j] = read_w(j, (s + 1) % 4, (super + (s == 3)) & 1);
#pragma unroll
                            for (int i = 0; i < act; ++i) fx[set ^ 1][i] = read_x(i, 0, stage_next);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
#pragma unroll
                    for (int n = 0; n < 8; ++n) {
                        const int i = n / 4, j = n % 4;
                        if (i < act)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fx[set][i]), fw[set][j], acc[i][j], 0, 0, 0);
                        if constexpr (ks < 3) {
                            if (n < act) fx[set ^ 1][n] = read_x(n, ks + 1, stage);
                            if (act > 0 && (n & 1)) fw[set ^ 1][n / 2] = codes_bf16(codes[n / 2][ks + 1], sc[n / 2]);
                            // the next superblock's weights, in the first two steps of this one
                            if (ks == 0 && s < 2 && (n == 3 || n == 7) && load_w) fetch_w(s * 2 + n / 4, super + 1);
                        } else {
                            if (VEC && load && (n & 1) && n / 2 < kXLoads) fetch_x(n / 2, super + (s + kXStages) / 4, (s + kXStages) % 4, stage);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    if constexpr (ks == 3) {
                        if constexpr (s == 3 && load_w) take_scales(super + 1);
                        if constexpr (next && act > 0) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                sc[j] = scale_operand((scales[j] >> (8 * ((s + 1) % 4))) & 255);
                                fw[set ^ 1][j] = codes_bf16(codes[j][0], sc[j]);
                            }
                        }
                    }
                };
                if constexpr (s == 0 && load_w) {
                    if constexpr (WHOLE) fetch_words(super + 1);
                    else fetch_scales(super + 1);
                }
                sub(Int<0>{});
                sub(Int<1>{});
                sub(Int<2>{});
                hand_over(S, MORE);
                wait_step(S, MORE);
                if constexpr (!WHOLE && s == 2 && load_w) scales_arrive();
                __syncthreads();
                take_up(S, MORE, super);
                sub(Int<3>{});
            };
            uint32_t super = 0;
            for (; super + 1 < supers; ++super) {
                step(Int<0>{}, Int<1>{}, super);
                step(Int<1>{}, Int<1>{}, super);
                step(Int<2>{}, Int<1>{}, super);
                step(Int<3>{}, Int<1>{}, super);
            }
            step(Int<0>{}, Int<0>{}, super);
            step(Int<1>{}, Int<0>{}, super);
            step(Int<2>{}, Int<0>{}, super);
            step(Int<3>{}, Int<0>{}, super);
        }
    };
    // (the same for a whole wavefront)
    if (RT == 2 && wm * 32 + 128 < t.rows) k_loop(Int<RT>{});
    else if (wm * 32 < t.rows) k_loop(Int<1>{});
    else k_loop(Int<0>{});

    // Column q of a 32 x 32 result lies in lane q and q + 32, its rows 8 (r / 4) + 4 h + r % 4 in their 16 numbers.  For BF16 neighbouring
    // lanes swap numbers, so that an even lane has two columns of an even row and an odd one of the next: 4-byte stores.
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        const uint32_t row0 = (wm + 4 * i) * 32 + 4 * h;
        if ((wm + 4 * i) * 32 >= t.rows) break;
        if constexpr (GRAD) {                                // the lane's four columns are those of the four tiles
            const uint32_t n = n0 + wn * 128 + 4 * q;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const uint32_t row = row0 + 8 * (r / 4) + r % 4;
                if (row >= t.rows || n >= outs) continue;
                OUT* const dst = reinterpret_cast<OUT*>(static_cast<char*>(a.out) + uint64_t(t.first + row) * a.out_stride) + n;
                if (a.out_vec) {
                    if constexpr (sizeof(OUT) == 2)
                        *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16_rne(acc[i][0][r], acc[i][1][r]), pack_bf16_rne(acc[i][2][r], acc[i][3][r]));
                    else
                        *reinterpret_cast<float4*>(dst) = make_float4(acc[i][0][r], acc[i][1][r], acc[i][2][r], acc[i][3][r]);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) from_float(dst + j, acc[i][j][r]);
                }
            }
            continue;
        }
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
            if constexpr (sizeof(OUT) == 2) {
                const uint32_t row = row0 + 8 * (r / 4) + r % 4 + (q & 1);
                char* const dst = static_cast<char*>(a.out) + uint64_t(t.first + min(row, t.rows - 1)) * a.out_stride;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t mine = pack_bf16_rne(acc[i][j][r], acc[i][j][r + 1]), other = dpp<kDppXor1>(mine);
                    const uint32_t both = __builtin_amdgcn_perm(other, mine, (q & 1) ? 0x03020706u : 0x05040100u);
                    const uint32_t n = n0 + wn * 128 + j * 32 + (q & ~1u);
                    if (row >= t.rows || n >= a.N) continue;
                    if (a.out_vec && n + 1 < a.N) {
                        *reinterpret_cast<uint32_t*>(dst + 2 * n) = both;
                    } else {
                        reinterpret_cast<uint16_t*>(dst)[n] = uint16_t(both);
                        if (n + 1 < a.N) reinterpret_cast<uint16_t*>(dst)[n + 1] = uint16_t(both >> 16);
                    }
                }
            } else {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const uint32_t row = row0 + 8 * (r / 4) + (r + c) % 4;
                    if (row >= t.rows) continue;
                    float* const dst = reinterpret_cast<float*>(static_cast<char*>(a.out) + uint64_t(t.first + row) * a.out_stride);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t n = n0 + wn * 128 + j * 32 + q;
                        if (n < a.N) dst[n] = acc[i][j][r + c];
                    }
                }
            }
        }
    }
}

template <Mode MODE, int RT, typename OUT>
void go(const MxProductArgs& a, const MxChoice& choice, hipStream_t stream) {
    const WideGrid grid(a, 128 * RT, MODE == kGradRows ? a.K : a.N);
    const dim3 wgs(grid.total), threads(kThreads);
    constexpr uint32_t lds = 4 * kStage + scale_bytes(MODE) + 4 * kTileWords;
    if constexpr (MODE == kGradRows || (MODE == kBf16Rows && RT == 1)) {
        if (!choice.vec) {
            hipLaunchKernelGGL((mx_wide_kernel<MODE, RT, false, false, OUT>), wgs, threads, lds, stream, a, grid);
            return;
        }
    }
    if (choice.whole) hipLaunchKernelGGL((mx_wide_kernel<MODE, RT, true, true, OUT>), wgs, threads, lds, stream, a, grid);
    else hipLaunchKernelGGL((mx_wide_kernel<MODE, RT, false, true, OUT>), wgs, threads, lds, stream, a, grid);
}
template <Mode MODE, int RT>
hipError_t go(const MxProductArgs& a, const MxChoice& choice, bool out_f32, hipStream_t stream) {
    out_f32 ? go<MODE, RT, float>(a, choice, stream) : go<MODE, RT, bf16_t>(a, choice, stream);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_wide(const MxProductArgs& a, const MxChoice& choice, bool mx_rows, bool out_f32, hipStream_t stream) {
    if (mx_rows) return go<kMxRows, 2>(a, choice, out_f32, stream);
    return choice.rows == 128 ? go<kBf16Rows, 1>(a, choice, out_f32, stream) : go<kBf16Rows, 2>(a, choice, out_f32, stream);
}
hipError_t launch_mx_wide_grad(const MxProductArgs& a, const MxChoice& choice, bool out_f32, hipStream_t stream) {
    return choice.rows == 128 ? go<kGradRows, 1>(a, choice, out_f32, stream) : go<kGradRows, 2>(a, choice, out_f32, stream);
}

}  // namespace fluxmoe
