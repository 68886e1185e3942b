// Products of rows sorted by expert with their expert's weights in 4-bit floating point (MXFP4), and the gradient to the rows.
//
//   out[r][n]    = sum over k of rows[r][k] W_e[n][k]         W_e[n][k] = code * 2^(scale - 127)
//   d_rows[r][k] = sum over n of d_out[r][n] W_e[n][k]
//
// Codes become BF16 in v_cvt_scalef32_pk_bf16_fp4, two at a time and exactly (a code has two significant bits), and meet BF16
// rows in the BF16 matrix instructions; rows in 4 bits themselves go to the scaled ones as they are.  Sums are FP32.
//
// Which rows are whose is known on the device only: a workgroup adds up the experts' tiles and finds its own (find_tile).
#include "mx_device.h"

namespace fluxmoe {
namespace {

constexpr uint32_t kThreads = 256;
constexpr uint32_t kMaxGrid = 1u << 22;

// `n` (1 .. 4) neighbouring outputs of a row
template <typename OUT>
__device__ __forceinline__ void store_outputs(const MxProductArgs& a, uint32_t row, uint32_t at, uint32_t n, f32x4 v) {
    OUT* const dst = reinterpret_cast<OUT*>(static_cast<char*>(a.out) + uint64_t(row) * a.out_stride) + at;
    if (a.out_vec && n == 4) {
        if constexpr (sizeof(OUT) == 2) *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16_rne(v[0], v[1]), pack_bf16_rne(v[2], v[3]));
        else *reinterpret_cast<f32x4*>(dst) = v;
    } else {
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k)
            if (k < n) from_float(dst + k, v[k]);
    }
}

// ---------------------------------------------------------------- few rows to an expert: bound by the weights' bytes
// A workgroup has 16 MI rows and 16 NI outputs, and its four wavefronts a quarter of the columns each, 512 at a time.  Lane (r, q) of a
// wavefront holds blocks q, 4 + q, 8 + q and 12 + q of output r's 512 columns, as they lie in memory: 16 bytes of codes and a scale
// each.  Which columns a matrix instruction's k numbers stand for is free as long as both operands agree, so the weights go from memory
// to registers to the matrix cores with nothing between; a row's columns are loaded likewise.  A load takes 64 bytes of each of 16
// outputs, and the next one the other half of their lines, which it finds in the first cache: 647 MB of 160 experts 132 us, 198 where
// loads pass it by, 141 where a lane's four blocks lie next to each other.
// VEC: rows at 16-byte addresses, not too far apart.  WHOLE: a row's scales are read as words.
template <int MI, int NI, bool MX, bool VEC, bool WHOLE, typename OUT>
__global__ __launch_bounds__(kThreads) void mx_stream_kernel(MxProductArgs a, uint32_t strips, uint64_t items) {
    __shared__ uint32_t s_tile[kTileWords];
    __shared__ f32x4 s_acc[4][MI * NI][64];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, q = lane >> 4;
    const uint32_t blocks = a.K / kMxBlock, supers = (blocks + 15) / 16;
    for (uint64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const auto [tile_at, strip] = item_at(item, strips);
        const Tile t = find_tile<kThreads>(a, 16 * MI, tile_at, s_tile);
        if (t.rows == 0) return;                         // nor are there any behind it
        const uint32_t n0 = strip * (16 * NI), outs = min(a.N - n0, uint32_t(16 * NI));
        const uint64_t w_row = uint64_t(t.expert) * a.N + n0;
        const row_t w = bytes_at(a.w, w_row * (a.K / 2), outs * (a.K / 2));
        const row_t ws = bytes_at(a.ws, w_row * blocks, outs * blocks);

        f32x4 acc[MI][NI];
#pragma unroll
        for (int m = 0; m < MI; ++m)
#pragma unroll
            for (int n = 0; n < NI; ++n) acc[m][n] = f32x4{0, 0, 0, 0};

        for (uint32_t super = wave; super < supers; super += 4) {
            const uint32_t block = super * 16 + q;           // and 4, 8, 12 behind it
            u32x4 wv[NI][4];
            uint32_t wsv[NI];
#pragma unroll
            for (int n = 0; n < NI; ++n) {
                const uint32_t row = n * 16 + r;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    wv[n][i] = piece_at(w, block + 4 * i < blocks, row * (a.K / 2) + (block + 4 * i) * 16);
                wsv[n] = spread_scales<WHOLE>(ws, row * blocks, block, q, blocks);
            }
            const char* src[MI];
            bool have[MI];
#pragma unroll
            for (int m = 0; m < MI; ++m) {
                have[m] = m * 16 + r < t.rows;
                src[m] = static_cast<const char*>(a.rows) + uint64_t(t.first + (have[m] ? m * 16 + r : 0)) * a.row_stride;
            }
            if constexpr (MX) {
                u32x4 xv[MI][4];
                uint32_t xs[MI];
#pragma unroll
                for (int m = 0; m < MI; ++m) {
                    xs[m] = 0;
                    if constexpr (WHOLE) {
                        const uint32_t stride = uint32_t(a.row_scales_stride);
                        const row_t scales = bytes_at(a.row_scales, uint64_t(t.first) * stride, (t.rows - 1) * stride + blocks);
                        if (have[m]) xs[m] = spread_scales<true>(scales, (m * 16 + r) * stride, block, q, blocks);
                    } else {
                        const uint8_t* scales = a.row_scales + uint64_t(t.first + (have[m] ? m * 16 + r : 0)) * a.row_scales_stride;
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (have[m] && block + 4 * i < blocks) xs[m] |= uint32_t(scales[block + 4 * i]) << (8 * i);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        xv[m][i] = u32x4{0, 0, 0, 0};
                        if (have[m] && block + 4 * i < blocks) {
                            if constexpr (VEC) xv[m][i] = *reinterpret_cast<const u32x4*>(src[m] + (block + 4 * i) * 16);
                            else __builtin_memcpy(&xv[m][i], src[m] + (block + 4 * i) * 16, 16);
                        }
                    }
                }
                auto multiply = [&](auto I) __attribute__((always_inline)) {
                    constexpr int i = decltype(I)::value;
#pragma unroll
                    for (int n = 0; n < NI; ++n) {
                        const i32x8 wa = {int(wv[n][i][0]), int(wv[n][i][1]), int(wv[n][i][2]), int(wv[n][i][3]), 0, 0, 0, 0};
#pragma unroll
                        for (int m = 0; m < MI; ++m) {
                            const i32x8 xb = {int(xv[m][i][0]), int(xv[m][i][1]), int(xv[m][i][2]), int(xv[m][i][3]), 0, 0, 0, 0};
                            acc[m][n] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wa, xb, acc[m][n], 4, 4, i, int(wsv[n]), i, int(xs[m]));
                        }
                    }
                };
                multiply(Int<0>{});
                multiply(Int<1>{});
                multiply(Int<2>{});
                multiply(Int<3>{});
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    u32x4 xv[MI][4];
#pragma unroll
                    for (int m = 0; m < MI; ++m)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            xv[m][j] = u32x4{0, 0, 0, 0};
                            if (have[m] && block + 4 * i < blocks) {
                                if constexpr (VEC) xv[m][j] = *reinterpret_cast<const u32x4*>(src[m] + (block + 4 * i) * 64 + j * 16);
                                else __builtin_memcpy(&xv[m][j], src[m] + (block + 4 * i) * 64 + j * 16, 16);
                            }
                        }
#pragma unroll
                    for (int n = 0; n < NI; ++n) {
                        const float scale = scale_operand((wsv[n] >> (8 * i)) & 255);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const bf16x8 f = codes_bf16(wv[n][i][j], scale);
#pragma unroll
                            for (int m = 0; m < MI; ++m)
                                acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, __builtin_bit_cast(bf16x8, xv[m][j]), acc[m][n], 0, 0, 0);
                        }
                    }
                }
            }
        }

        // The quarters' sums in their order; then neighbouring threads have neighbouring outputs of a row, four to each.
#pragma unroll
        for (int m = 0; m < MI; ++m)
#pragma unroll
            for (int n = 0; n < NI; ++n) s_acc[wave][m * NI + n][lane] = acc[m][n];
        __syncthreads();
        for (uint32_t i = tid; i < 64 * MI * NI; i += kThreads) {
            const uint32_t row = i / (4 * NI), quad = i % (4 * NI);
            if (row >= t.rows) break;
            const uint32_t at = (quad & 3) * 16 + (row & 15), part = (row >> 4) * NI + (quad >> 2);
            f32x4 v = s_acc[0][part][at];
#pragma unroll
            for (int k = 1; k < 4; ++k) v += s_acc[k][part][at];
            if (quad * 4 < outs) store_outputs<OUT>(a, t.first + row, n0 + quad * 4, min(outs - quad * 4, 4u), v);
        }
    }
}

// The same for more bytes: four wavefronts side by side, 16 NI outputs each, over all columns.  The rows' columns come through LDS, for all
// four, and the weights of the next 256 columns are on their way while these are multiplied: loads return in the order of their issue, so
// rows that a wavefront fetched for itself would be waited for behind those weights.  A row's 16-byte pieces are placed so that 16 rows'
// pieces of one number lie in different banks.
template <int MI, int NI, bool MX, bool WHOLE, typename OUT>
__global__ __launch_bounds__(kThreads, 2) void mx_strip_kernel(MxProductArgs a, uint32_t strips, uint64_t items) {
    constexpr uint32_t kPieces = MX ? 8 : 32;                // 16-byte pieces of a row's 256 columns
    constexpr int kMine = (16 * MI * kPieces + kThreads - 1) / kThreads;      // that a thread brings to LDS
    __shared__ uint32_t s_tile[kTileWords];
    __shared__ u32x4 s_x[2][16 * MI * kPieces];
    __shared__ f32x4 s_acc[4][NI][64];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, q = lane >> 4;
    const uint32_t blocks = a.K / kMxBlock, steps = (blocks + 7) / 8;
    for (uint64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const auto [tile_at, strip] = item_at(item, strips);
        const Tile t = find_tile<kThreads>(a, 16 * MI, tile_at, s_tile);
        if (t.rows == 0) return;
        const uint32_t n0 = (strip * 4 + wave) * (16 * NI), outs = n0 < a.N ? min(a.N - n0, uint32_t(16 * NI)) : 0;
        const uint64_t w_row = uint64_t(t.expert) * a.N + min(n0, a.N - 1);
        const row_t w = bytes_at(a.w, w_row * (a.K / 2), outs * (a.K / 2)), ws = bytes_at(a.ws, w_row * blocks, outs * blocks);
        const row_t x = bytes_at(a.rows, uint64_t(t.first) * a.row_stride, (t.rows - 1) * uint32_t(a.row_stride) + (MX ? a.K / 2 : a.K * 2));
        const row_t xs = bytes_at(a.row_scales, uint64_t(t.first) * a.row_scales_stride,
                                  MX ? (t.rows - 1) * uint32_t(a.row_scales_stride) + blocks : 0);

        auto swizzle = [](uint32_t row) __attribute__((always_inline)) { return MX ? (row >> 1) & 7 : row & 15; };
        struct Operands {
            u32x4 w[NI][2];
            uint32_t ws[NI], xs[MI];
        };
        Operands one, two;
        u32x4 mine[kMine];
        auto load = [&](Operands& o, uint32_t step) __attribute__((always_inline)) {
#pragma unroll
            for (int c = 0; c < kMine; ++c) {                // ahead of the weights, to be waited for without them
                const uint32_t at = tid + c * kThreads, row = at / kPieces, piece = step * kPieces + at % kPieces;
                mine[c] = piece_at(x, row < t.rows && piece < blocks * (MX ? 1 : 4), row * uint32_t(a.row_stride) + piece * 16);
            }
            const uint32_t block = step * 8 + q;
            if constexpr (MX) {
#pragma unroll
                for (int m = 0; m < MI; ++m)
                    o.xs[m] = pair_scales<WHOLE>(xs, min(m * 16 + r, t.rows - 1) * uint32_t(a.row_scales_stride), block, q, blocks);
            }
#pragma unroll
            for (int n = 0; n < NI; ++n) {
                const uint32_t row = n * 16 + r;
                o.ws[n] = pair_scales<WHOLE>(ws, row * blocks, block, q, blocks);
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    o.w[n][i] = piece_at(w, block + 4 * i < blocks, row * (a.K / 2) + (block + 4 * i) * 16);
            }
        };
        auto put = [&](uint32_t stage) __attribute__((always_inline)) {
#pragma unroll
            for (int c = 0; c < kMine; ++c) {
                const uint32_t at = tid + c * kThreads, row = at / kPieces, piece = at % kPieces;
                if (16 * MI * kPieces % kThreads == 0 || at < 16 * MI * kPieces) s_x[stage][row * kPieces + (piece ^ swizzle(row))] = mine[c];
            }
        };
        f32x4 acc[MI][NI];
#pragma unroll
        for (int m = 0; m < MI; ++m)
#pragma unroll
            for (int n = 0; n < NI; ++n) acc[m][n] = f32x4{0, 0, 0, 0};
        auto multiply = [&](const Operands& o, uint32_t stage) __attribute__((always_inline)) {
            auto part = [&](auto I) __attribute__((always_inline)) {
                constexpr int i = decltype(I)::value;
                if constexpr (MX) {
                    u32x4 xv[MI];
#pragma unroll
                    for (int m = 0; m < MI; ++m) xv[m] = s_x[stage][(m * 16 + r) * kPieces + ((4 * i + q) ^ swizzle(r))];
#pragma unroll
                    for (int n = 0; n < NI; ++n) {
                        const i32x8 wa = {int(o.w[n][i][0]), int(o.w[n][i][1]), int(o.w[n][i][2]), int(o.w[n][i][3]), 0, 0, 0, 0};
#pragma unroll
                        for (int m = 0; m < MI; ++m) {
                            const i32x8 xb = {int(xv[m][0]), int(xv[m][1]), int(xv[m][2]), int(xv[m][3]), 0, 0, 0, 0};
                            acc[m][n] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wa, xb, acc[m][n], 4, 4, i, int(o.ws[n]), i, int(o.xs[m]));
                        }
                    }
                } else {
                    float scale[NI];
#pragma unroll
                    for (int n = 0; n < NI; ++n) scale[n] = scale_operand((o.ws[n] >> (8 * i)) & 255);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        bf16x8 xv[MI];
#pragma unroll
                        for (int m = 0; m < MI; ++m)
                            xv[m] = __builtin_bit_cast(bf16x8, s_x[stage][(m * 16 + r) * kPieces + ((16 * i + 4 * q + j) ^ swizzle(r))]);
#pragma unroll
                        for (int n = 0; n < NI; ++n) {
                            const bf16x8 f = codes_bf16(o.w[n][i][j], scale[n]);
#pragma unroll
                            for (int m = 0; m < MI; ++m) acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, xv[m], acc[m][n], 0, 0, 0);
                        }
                    }
                }
            };
            part(Int<0>{});
            part(Int<1>{});
        };
        load(one, 0);
        put(0);
        __syncthreads();
        for (uint32_t step = 0;; step += 2) {
            if (step + 1 < steps) load(two, step + 1);
            multiply(one, 0);
            if (step + 1 >= steps) break;
            put(1);
            __syncthreads();
            if (step + 2 < steps) load(one, step + 2);
            multiply(two, 1);
            if (step + 2 >= steps) break;
            put(0);
            __syncthreads();
        }

        // Through LDS to where neighbouring lanes have neighbouring outputs of a row, four to each.
#pragma unroll
        for (int m = 0; m < MI; ++m) {
            if (m * 16 >= t.rows) break;
            wave_fence();
#pragma unroll
            for (int n = 0; n < NI; ++n) s_acc[wave][n][lane] = acc[m][n];
            wave_fence();
#pragma unroll
            for (int c = 0; c < NI; ++c) {
                const uint32_t row = (c * 64 + lane) / (4 * NI), quad = lane % (4 * NI);
                const f32x4 v = s_acc[wave][quad >> 2][(quad & 3) * 16 + row];
                if (m * 16 + row >= t.rows || quad * 4 >= outs) continue;
                store_outputs<OUT>(a, t.first + m * 16 + row, n0 + quad * 4, min(outs - quad * 4, 4u), v);
            }
        }
    }
}

// The gradient likewise.  A workgroup has 16 MI rows and 256 columns, its four or eight wavefronts share out the outputs, 32 at a time.
// Lane (r, q) loads 16 neighbouring columns of eight outputs, eight bytes of each, turns them into sixteen fragments of eight outputs by a
// conversion and a permutation to each two numbers, and fragment c goes to a matrix instruction whose results are column c of every lane's.
// A wavefront waits for its loads, so what counts is how many there are: three to a SIMD with 16 rows, two with 32 (900 tokens of 512 experts,
// 512 columns 163 -> 91 us, 100 tokens 47 -> 41; fetching the next outputs ahead, with fewer wavefronts, 98 and 52).
template <int MI, int WAVES, bool VEC, typename OUT>
__global__ __launch_bounds__(64 * WAVES, MI == 1 && WAVES == 4 ? 3 : 2) void mx_stream_grad_kernel(MxProductArgs a, uint32_t strips, uint64_t items) {
    __shared__ uint32_t s_tile[kTileWords];
    __shared__ f32x4 s_acc[WAVES - 1][8][64];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, q = lane >> 4;
    const uint32_t blocks = a.K / kMxBlock, chunks = (a.N + 31) / 32;
    for (uint64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const auto [tile_at, strip] = item_at(item, strips);
        const Tile t = find_tile<64 * WAVES>(a, 16 * MI, tile_at, s_tile);
        if (t.rows == 0) return;
        const uint32_t k0 = strip * 256, column = k0 + r * 16;
        f32x4 acc[MI][16];
#pragma unroll
        for (int m = 0; m < MI; ++m)
#pragma unroll
            for (int c = 0; c < 16; ++c) acc[m][c] = f32x4{0, 0, 0, 0};
        for (uint32_t chunk = wave; chunk < chunks; chunk += WAVES) {
            const uint64_t row = uint64_t(t.expert) * a.N + chunk * 32;
            const uint32_t left = min(a.N - chunk * 32, 32u);
            const row_t w = bytes_at(a.w, row * (a.K / 2), left * (a.K / 2)), ws = bytes_at(a.ws, row * blocks, left * blocks);
            uint32_t w_at = column < a.K ? 8 * q * (a.K / 2) + column / 2 : kNowhere;
            uint32_t s_at = column < a.K ? 8 * q * blocks + column / kMxBlock : kNowhere;
            // (made anew for each chunk: kept for all of them, the sixteen places below cost a wavefront to a SIMD)
            asm volatile("" : "+v"(w_at), "+v"(s_at));
            u32x2 codes[8];
            uint32_t scales[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                codes[j] = __builtin_amdgcn_raw_buffer_load_b64(w, w_at + j * (a.K / 2), 0, kStream);
                scales[j] = __builtin_amdgcn_raw_buffer_load_b8(ws, s_at + j * blocks, 0, kCached);
            }
            u32x4 x[MI];
            const uint32_t n = chunk * 32 + 8 * q;
#pragma unroll
            for (int m = 0; m < MI; ++m) {
                x[m] = u32x4{0, 0, 0, 0};
                const uint64_t at = uint64_t(t.first + min(m * 16 + r, t.rows - 1)) * a.row_stride;
                const uint16_t* p = reinterpret_cast<const uint16_t*>(static_cast<const char*>(a.rows) + at) + n;
                if (m * 16 + r < t.rows) {
                    if (VEC && n < a.N) x[m] = *reinterpret_cast<const u32x4*>(p);
                    if constexpr (!VEC) {
                        if (n + 8 <= a.N) {
                            __builtin_memcpy(&x[m], p, 16);
                        } else {
#pragma unroll
                            for (uint32_t j = 0; j < 8; ++j)
                                if (n + j < a.N) x[m][j / 2] |= uint32_t(p[j]) << (16 * (j & 1));
                        }
                    }
                }
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {           // eight of the sixteen columns
                uint32_t pair[8][4];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float scale = scale_operand(scales[j]);
                    pair[j][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[j][half], scale, 0));
                    pair[j][1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[j][half], scale, 1));
                    pair[j][2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[j][half], scale, 2));
                    pair[j][3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[j][half], scale, 3));
                }
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    u32x4 f;
#pragma unroll
                    for (int d = 0; d < 4; ++d) f[d] = __builtin_amdgcn_perm(pair[2 * d + 1][c / 2], pair[2 * d][c / 2], (c & 1) ? 0x07060302u : 0x05040100u);
#pragma unroll
                    for (int m = 0; m < MI; ++m)
                        acc[m][half * 8 + c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), __builtin_bit_cast(bf16x8, x[m]),
                                                                                      acc[m][half * 8 + c], 0, 0, 0);
                }
            }
        }
        // The wavefronts' sums in their order, 16 rows at a time and half of the columns; a lane then has 16 neighbouring columns of four
        // lanes' for its row.
#pragma unroll
        for (int m = 0; m < MI; ++m) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                if (m || half) __syncthreads();
                if (wave) {
#pragma unroll
                    for (int c = 0; c < 8; ++c) s_acc[wave - 1][c][lane] = acc[m][half * 8 + c];
                }
                __syncthreads();
                if (wave == 0) {
#pragma unroll
                    for (int c = 0; c < 8; ++c)
#pragma unroll
                        for (int k = 0; k < WAVES - 1; ++k) acc[m][half * 8 + c] += s_acc[k][c][lane];
                }
            }
            if (wave != 0 || m * 16 + r >= t.rows) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t k = k0 + (4 * q + i) * 16;
                if (k >= a.K) continue;
#pragma unroll
                for (int c = 0; c < 16; c += 4)
                    store_outputs<OUT>(a, t.first + m * 16 + r, k + c, 4, f32x4{acc[m][c][i], acc[m][c + 1][i], acc[m][c + 2][i], acc[m][c + 3][i]});
            }
        }
    }
}

struct Grid {
    uint32_t strips;
    uint64_t items;
    uint32_t workgroups;
    Grid(const MxCall& c, uint32_t rows, uint32_t outs, uint32_t width) {
        strips = (outs + width - 1) / width;
        items = mx_most_tiles(c, rows) * strips;
        workgroups = uint32_t(items < kMaxGrid ? items : kMaxGrid);
    }
};

MxCall call_of(const MxProductArgs& a, bool mx_rows) {
    const auto words = [](const void* p, uint64_t stride) { return reinterpret_cast<uintptr_t>(p) % 4 == 0 && stride % 4 == 0; };
    return {a.cap, a.E, a.N, a.K, a.row_stride, a.row_scales_stride, mx_rows, a.rows_vec != 0, words(a.ws, a.K / kMxBlock),
            words(a.row_scales, a.row_scales_stride)};
}

template <int MI, int NI, bool MX, bool VEC, typename OUT>
void go_stream(const MxProductArgs& a, const MxCall& c, bool whole, hipStream_t stream) {
    const Grid g(c, 16 * MI, a.N, 16 * NI);
    if (VEC && whole) hipLaunchKernelGGL((mx_stream_kernel<MI, NI, MX, VEC, VEC, OUT>), dim3(g.workgroups), dim3(kThreads), 0, stream, a, g.strips, g.items);
    else hipLaunchKernelGGL((mx_stream_kernel<MI, NI, MX, VEC, false, OUT>), dim3(g.workgroups), dim3(kThreads), 0, stream, a, g.strips, g.items);
}
template <int MI, bool MX, typename OUT>
void go_strip(const MxProductArgs& a, const MxCall& c, bool whole, hipStream_t stream) {
    constexpr int NI = mx_strip_outs(MX, 16 * MI) / 16;
    const Grid g(c, 16 * MI, a.N, 64 * NI);
    if (whole) hipLaunchKernelGGL((mx_strip_kernel<MI, NI, MX, true, OUT>), dim3(g.workgroups), dim3(kThreads), 0, stream, a, g.strips, g.items);
    else hipLaunchKernelGGL((mx_strip_kernel<MI, NI, MX, false, OUT>), dim3(g.workgroups), dim3(kThreads), 0, stream, a, g.strips, g.items);
}
template <int MI, bool VEC, typename OUT>
void go_stream_grad(const MxProductArgs& a, const MxCall& c, uint32_t waves, hipStream_t stream) {
    const Grid g(c, 16 * MI, a.K, 256);
    if (waves == 8) hipLaunchKernelGGL((mx_stream_grad_kernel<MI, 8, VEC, OUT>), dim3(g.workgroups), dim3(512), 0, stream, a, g.strips, g.items);
    else hipLaunchKernelGGL((mx_stream_grad_kernel<MI, 4, VEC, OUT>), dim3(g.workgroups), dim3(256), 0, stream, a, g.strips, g.items);
}

template <bool MX, typename OUT>
hipError_t product(const MxProductArgs& a, hipStream_t stream) {
    const MxCall c = call_of(a, MX);
    const MxChoice k = mx_choose_product(c);
    if (k.kernel == kMxWide) return launch_mx_wide(a, k, MX, sizeof(OUT) == 4, stream);
    if (k.kernel == kMxStrip) {
        if (k.rows == 64) go_strip<4, MX, OUT>(a, c, k.whole, stream);
        else if (k.rows == 32) go_strip<2, MX, OUT>(a, c, k.whole, stream);
        else go_strip<1, MX, OUT>(a, c, k.whole, stream);
    } else if (!k.vec) {
        go_stream<2, 4, MX, false, OUT>(a, c, false, stream);
    } else if (k.rows == 32) {
        k.outs == 64 ? go_stream<2, 4, MX, true, OUT>(a, c, k.whole, stream) : go_stream<2, 1, MX, true, OUT>(a, c, k.whole, stream);
    } else {
        k.outs == 64 ? go_stream<1, 4, MX, true, OUT>(a, c, k.whole, stream) : go_stream<1, 1, MX, true, OUT>(a, c, k.whole, stream);
    }
    return hipGetLastError();
}

template <typename OUT>
hipError_t product_grad(const MxProductArgs& a, hipStream_t stream) {
    const MxCall c = call_of(a, false);
    const MxChoice k = mx_choose_grad(c);
    if (k.kernel == kMxWide) return launch_mx_wide_grad(a, k, sizeof(OUT) == 4, stream);
    if (k.rows == 32) k.vec ? go_stream_grad<2, true, OUT>(a, c, k.waves, stream) : go_stream_grad<2, false, OUT>(a, c, k.waves, stream);
    else k.vec ? go_stream_grad<1, true, OUT>(a, c, k.waves, stream) : go_stream_grad<1, false, OUT>(a, c, k.waves, stream);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_product(const MxProductArgs& a, bool mx_rows, bool out_f32, hipStream_t stream) {
    if (mx_rows) return out_f32 ? product<true, float>(a, stream) : product<true, bf16_t>(a, stream);
    return out_f32 ? product<false, float>(a, stream) : product<false, bf16_t>(a, stream);
}
hipError_t launch_mx_product_grad(const MxProductArgs& a, bool out_f32, hipStream_t stream) {
    return out_f32 ? product_grad<float>(a, stream) : product_grad<bf16_t>(a, stream);
}

}  // namespace fluxmoe
