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

// ---------------------------------------------------------------- few rows to an expert: bound by the weights' bytes
// A workgroup has a tile of 16 MI rows and 16 NI outputs; its four wavefronts share out the columns, 128 at a time.  Lane
// (r, q) of a wavefront holds the block of 32 columns number q of output r's 128, as it lies in memory: one 16-byte load
// and one scale.  Which columns a matrix instruction's k numbers stand for is free as long as both operands agree, so the
// weights go from memory to registers to the matrix cores with nothing between; a row's columns are loaded likewise.
template <int MI, int NI, bool MX, bool VEC, typename OUT>
__global__ __launch_bounds__(kThreads) void mx_stream_kernel(MxProductArgs a, uint32_t strips, uint64_t items) {
    __shared__ uint32_t s_tile[kTileWords];
    __shared__ f32x4 s_acc[4][MI * NI][64];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 15, q = lane >> 4;
    const uint32_t blocks = a.K / kMxBlock, groups = (blocks + 3) / 4;
    for (uint64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const uint32_t tile_at = uint32_t(item / strips), strip = uint32_t(item - uint64_t(tile_at) * strips);
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

        for (uint32_t g = wave; g < groups; g += 4) {
            const uint32_t block = g * 4 + q;
            const bool in = block < blocks;
            u32x4 wv[NI];
            uint32_t wsv[NI];
#pragma unroll
            for (int n = 0; n < NI; ++n) {
                const uint32_t row = n * 16 + r;
                wv[n] = __builtin_amdgcn_raw_buffer_load_b128(w, in ? row * (a.K / 2) + block * 16 : kNowhere, 0, kStream);
                wsv[n] = __builtin_amdgcn_raw_buffer_load_b8(ws, in ? row * blocks + block : kNowhere, 0, kCached);
            }
#pragma unroll
            for (int m = 0; m < MI; ++m) {
                const uint32_t row = m * 16 + r;
                const bool have = in && row < t.rows;
                const char* src = static_cast<const char*>(a.rows) + uint64_t(t.first + (have ? row : 0)) * a.row_stride;
                if constexpr (MX) {
                    u32x4 xv = {0, 0, 0, 0};
                    uint32_t xs = 0;
                    if (have) {
                        if constexpr (VEC) xv = *reinterpret_cast<const u32x4*>(src + block * 16);
                        else {
#pragma unroll
                            for (int j = 0; j < 16; ++j) xv[j / 4] |= uint32_t(uint8_t(src[block * 16 + j])) << (8 * (j & 3));
                        }
                        xs = a.row_scales[uint64_t(t.first + row) * a.row_scales_stride + block];
                    }
                    const i32x8 xb = {int(xv[0]), int(xv[1]), int(xv[2]), int(xv[3]), 0, 0, 0, 0};
#pragma unroll
                    for (int n = 0; n < NI; ++n) {
                        const i32x8 wa = {int(wv[n][0]), int(wv[n][1]), int(wv[n][2]), int(wv[n][3]), 0, 0, 0, 0};
                        acc[m][n] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wa, xb, acc[m][n], 4, 4, 0, int(wsv[n]), 0, int(xs));
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        u32x4 xv = {0, 0, 0, 0};
                        if (have) {
                            if constexpr (VEC) xv = *reinterpret_cast<const u32x4*>(src + block * 64 + j * 16);
                            else {
                                const uint16_t* p = reinterpret_cast<const uint16_t*>(src) + block * 32 + j * 8;
#pragma unroll
                                for (int i = 0; i < 8; ++i) xv[i / 2] |= uint32_t(p[i]) << (16 * (i & 1));
                            }
                        }
#pragma unroll
                        for (int n = 0; n < NI; ++n)
                            acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_bf16(wv[n][j], scale_operand(wsv[n])),
                                                                               __builtin_bit_cast(bf16x8, xv), acc[m][n], 0, 0, 0);
                    }
                }
            }
        }

        // the wavefronts' sums in their order; then neighbouring threads have neighbouring outputs of a row, four to each
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
            OUT* dst = reinterpret_cast<OUT*>(static_cast<char*>(a.out) + uint64_t(t.first + row) * a.out_stride) + n0 + quad * 4;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (quad * 4 + k < outs) from_float(dst + k, v[k]);
        }
    }
}

// ---------------------------------------------------------------- many rows: tiles in LDS
// Both operands lie in LDS as BF16 rows of 64 summed columns (128 bytes), the weights converted on their way there; a 16-byte
// piece lies at its number xor swizzle(row), which spreads the rows' pieces over the banks.  GRAD sums over the outputs: the
// weights are turned round on their way, eight outputs by four columns to a thread.
__device__ __forceinline__ uint32_t piece_at(uint32_t row, uint32_t piece) { return row * 8 + (piece ^ ((row ^ (row >> 3)) & 7)); }

template <bool GRAD, typename OUT>
__global__ __launch_bounds__(kThreads) void mx_tile_kernel(MxProductArgs a, uint32_t strips, uint64_t items) {
    constexpr uint32_t BM = 128, BN = 128;
    __shared__ uint32_t s_tile[kTileWords];
    __shared__ u32x4 s_x[BM * 8], s_w[BN * 8];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t sum = GRAD ? a.N : a.K, outs = GRAD ? a.K : a.N, blocks = a.K / kMxBlock;
    const uint32_t m_wave = (wave >> 1) * 64, n_wave = (wave & 1) * 64;
    for (uint64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const uint32_t tile_at = uint32_t(item / strips), strip = uint32_t(item - uint64_t(tile_at) * strips);
        const Tile t = find_tile<kThreads>(a, BM, tile_at, s_tile);
        if (t.rows == 0) return;
        const uint32_t n0 = strip * BN;
        const char* x = static_cast<const char*>(a.rows) + uint64_t(t.first) * a.row_stride;
        const uint8_t* w = a.w + uint64_t(t.expert) * a.N * (a.K / 2);
        const uint8_t* ws = a.ws + uint64_t(t.expert) * a.N * blocks;
        f32x16 acc[2][2];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[i / 2][i % 2][j] = 0.0f;

        for (uint32_t k0 = 0; k0 < sum; k0 += 64) {
            u32x4 xv[4], wv[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t at = tid + i * kThreads, row = at / 8, k = k0 + (at & 7) * 8;
                xv[i] = u32x4{0, 0, 0, 0};
                if (row < t.rows && k < sum) {
                    const uint16_t* p = reinterpret_cast<const uint16_t*>(x + uint64_t(row) * a.row_stride) + k;
                    if (a.rows_vec && k + 8 <= sum) xv[i] = *reinterpret_cast<const u32x4*>(p);
                    else {
#pragma unroll
                        for (uint32_t j = 0; j < 8; ++j)
                            if (k + j < sum) xv[i][j / 2] |= uint32_t(p[j]) << (16 * (j & 1));
                    }
                }
            }
            if constexpr (GRAD) {
                const uint32_t ng = tid >> 5, k4 = n0 + (tid & 31) * 4;
                uint32_t v[8][2];
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) {
                    const uint64_t n = k0 + ng * 8 + j;
                    uint32_t codes = 0, s = 0;
                    if (n < sum && k4 < outs) {
                        codes = *reinterpret_cast<const uint16_t*>(w + n * (a.K / 2) + k4 / 2);
                        s = ws[n * blocks + k4 / kMxBlock];
                    }
                    v[j][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale_operand(s), 0));
                    v[j][1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale_operand(s), 1));
                }
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        const uint32_t lo = v[2 * d][c / 2], hi = v[2 * d + 1][c / 2];
                        wv[c][d] = (c & 1) ? (lo >> 16) | (hi & 0xFFFF0000u) : (lo & 0xFFFFu) | (hi << 16);
                    }
            } else {
                const uint32_t n = n0 + tid / 2, block = k0 / kMxBlock + (tid & 1);
                u32x4 codes = {0, 0, 0, 0};
                uint32_t s = 0;
                if (n < outs && block < blocks) {
                    codes = *reinterpret_cast<const u32x4*>(w + uint64_t(n) * (a.K / 2) + block * 16);
                    s = ws[uint64_t(n) * blocks + block];
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) wv[j] = __builtin_bit_cast(u32x4, codes_bf16(codes[j], scale_operand(s)));
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t at = tid + i * kThreads;
                s_x[piece_at(at / 8, at & 7)] = xv[i];
                if constexpr (GRAD) s_w[piece_at((tid & 31) * 4 + i, tid >> 5)] = wv[i];
                else s_w[piece_at(tid / 2, (tid & 1) * 4 + i)] = wv[i];
            }
            __syncthreads();
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                bf16x8 xf[2], wf[2];
                const uint32_t piece = ks * 2 + lane / 32;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    xf[i] = __builtin_bit_cast(bf16x8, s_x[piece_at(m_wave + i * 32 + (lane & 31), piece)]);
                    wf[i] = __builtin_bit_cast(bf16x8, s_w[piece_at(n_wave + i * 32 + (lane & 31), piece)]);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xf[i], wf[j], acc[i][j], 0, 0, 0);
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t n = n0 + n_wave + j * 32 + (lane & 31);
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                    const uint32_t row = m_wave + i * 32 + (c / 4) * 8 + (lane / 32) * 4 + c % 4;
                    if (row < t.rows && n < outs)
                        from_float(reinterpret_cast<OUT*>(static_cast<char*>(a.out) + uint64_t(t.first + row) * a.out_stride) + n, acc[i][j][c]);
                }
            }
    }
}

// Tiles that the groups can have: full ones and one unfinished one for each expert that has rows.
uint64_t most_tiles(const MxProductArgs& a, uint32_t size) { return a.cap / size + (a.cap < a.E ? a.cap : a.E); }

struct Plan {
    uint32_t strips;
    uint64_t items;
    uint32_t grid;
    Plan(const MxProductArgs& a, uint32_t rows, uint32_t outs, uint32_t width) {
        strips = (outs + width - 1) / width;
        items = most_tiles(a, rows) * strips;
        grid = uint32_t(items < kMaxGrid ? items : kMaxGrid);
    }
};

template <int MI, int NI, bool MX, bool VEC, typename OUT>
void go_stream(const MxProductArgs& a, hipStream_t stream) {
    const Plan p(a, 16 * MI, a.N, 16 * NI);
    hipLaunchKernelGGL((mx_stream_kernel<MI, NI, MX, VEC, OUT>), dim3(p.grid), dim3(kThreads), 0, stream, a, p.strips, p.items);
}
template <bool GRAD, typename OUT>
void go_tile(const MxProductArgs& a, hipStream_t stream) {
    const Plan p(a, 128, GRAD ? a.K : a.N, 128);
    hipLaunchKernelGGL((mx_tile_kernel<GRAD, OUT>), dim3(p.grid), dim3(kThreads), 0, stream, a, p.strips, p.items);
}

template <typename OUT>
hipError_t product(const MxProductArgs& a, bool mx_rows, hipStream_t stream) {
    const uint32_t per_expert = a.cap / a.E;
    if (per_expert > 32 && mx_wide_takes(a, mx_rows)) return launch_mx_wide(a, mx_rows, sizeof(OUT) == 4, stream);
    if (mx_rows) {
        if (a.rows_vec) go_stream<2, 4, true, true, OUT>(a, stream);
        else go_stream<2, 4, true, false, OUT>(a, stream);
    } else if (per_expert > 32) {
        go_tile<false, OUT>(a, stream);
    } else {
        if (a.rows_vec) go_stream<1, 4, false, true, OUT>(a, stream);
        else go_stream<1, 4, false, false, OUT>(a, stream);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_product(const MxProductArgs& a, bool mx_rows, bool out_f32, hipStream_t stream) {
    return out_f32 ? product<float>(a, mx_rows, stream) : product<bf16_t>(a, mx_rows, stream);
}
hipError_t launch_mx_product_grad(const MxProductArgs& a, bool out_f32, hipStream_t stream) {
    if (a.cap / a.E > 32 && mx_wide_grad_takes(a)) return launch_mx_wide_grad(a, out_f32, stream);
    if (out_f32) go_tile<true, float>(a, stream);
    else go_tile<true, bf16_t>(a, stream);
    return hipGetLastError();
}

}  // namespace fluxmoe
