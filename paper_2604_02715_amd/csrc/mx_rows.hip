// Rows to 4-bit floating point with shared scales (MXFP4) and back, and SwiGLU between an expert's two products: all of them
// pass over their rows once.
//
// 32 neighbouring numbers share a scale 2^e, e = floor(log2(largest magnitude)) - 2, so that the largest lies in [4, 8) of the
// code's 0 .. 6; each number over 2^e goes to its nearest code, ties to the even one, and past 6 to 6.  The largest is found
// on the bits (as integers they have the magnitudes' order, NaN on top), and e is its exponent field less 2: nothing is rounded
// but the number itself, once, in v_cvt_scalef32_pk_fp4_*, which does scale, rounding and saturation of two.
#include <type_traits>

#include "block_device.h"
#include "mx_ops.h"

namespace fluxmoe {
namespace {

constexpr uint32_t kThreads = 256;
constexpr uint32_t kMaxGrid = 1u << 22;      // workgroups of a launch; they go on past that many shares

// 2^(s - 127) as v_cvt_scalef32 takes it: by the exponent field alone, 0 for 2^-127 and 255 for not-a-number
__device__ __forceinline__ float scale_operand(uint32_t s) { return __uint_as_float(s << 23); }

// A workgroup's share of a matrix of rows: 256 pieces of a row side by side, or whole rows of fewer pieces, as many as fit.
struct Share {
    uint64_t row, piece;
    bool valid;
};
struct Shares {
    uint64_t rows, pieces;       // pieces of a row
    uint64_t chunks;             // workgroups to a row
    uint64_t items;
    uint32_t log2_lanes;         // lanes to a row
    __host__ Shares(uint64_t rows, uint64_t pieces) : rows(rows), pieces(pieces) {
        log2_lanes = 0;
        while (log2_lanes < 8 && (1ull << log2_lanes) < pieces) ++log2_lanes;
        chunks = (pieces + kThreads - 1) / kThreads;
        const uint64_t rows_per_wg = kThreads >> log2_lanes;
        items = chunks * ((rows + rows_per_wg - 1) / rows_per_wg);
    }
    // workgroups, with so many neighbouring shares to each at a time
    __host__ uint32_t grid(uint32_t at_once) const {
        const uint64_t n = (items + at_once - 1) / at_once;
        return uint32_t(n < kMaxGrid ? n : kMaxGrid);
    }
    // `item` may lie past the end
    __device__ __forceinline__ Share operator()(uint64_t item) const {
        // nearly always within 32 bits, where a division is a tenth as long
        const uint64_t group = (item | chunks) >> 32 ? item / chunks : uint32_t(item) / uint32_t(chunks);
        const uint64_t chunk = item - group * chunks;
        Share s;
        s.row = group * (kThreads >> log2_lanes) + (threadIdx.x >> log2_lanes);
        s.piece = chunk * kThreads + (threadIdx.x & ((1u << log2_lanes) - 1));
        s.valid = item < items && s.row < rows && s.piece < pieces;
        return s;
    }
};

// ---------------------------------------------------------------- to 4 bits
// Four lanes to a block, eight columns to a lane: a wavefront reads 1 or 2 KiB and writes 256 bytes of codes without gaps.
// Two shares at a time, so that a lane has two loads under way: 32768 x 14336 BF16 176 us (6.8 TB/s), with one 194, with four 179; with shares that
// lie far from each other 242.
// Likewise SwiGLU's gradient (32768 x 1536 FP32 158 -> 147 us, four 151); the others are level.
constexpr int kQuantizeAtOnce = 2, kSwigluGradAtOnce = 2;
template <typename T, bool VEC>
__global__ __launch_bounds__(kThreads) void mx_quantize_kernel(MxRowsArgs a, Shares shares) {
    constexpr int kAtOnce = kQuantizeAtOnce, kLoads = sizeof(T) / 2;
    for (uint64_t item = uint64_t(blockIdx.x) * kAtOnce; item < shares.items; item += uint64_t(kAtOnce) * gridDim.x) {
        Share share[kAtOnce];
        uint4 in[kAtOnce][kLoads];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            share[u] = shares(item + u);
            const T* x = static_cast<const T*>(a.x) + share[u].row * a.x_stride + share[u].piece * 8;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) in[u][i] = make_uint4(0, 0, 0, 0);
            if (VEC && share[u].valid) {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) in[u][i] = load_stream16(x + i * (16 / sizeof(T)));
            }
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const Share s = share[u];
            uint32_t v[8];                               // FP32 bits
            if constexpr (VEC) {
                const uint32_t w[4] = {in[u][0].x, in[u][0].y, in[u][0].z, in[u][0].w};
                if constexpr (sizeof(T) == 2) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = (j & 1) ? (w[j / 2] & 0xFFFF0000u) : (w[j / 2] << 16);
                } else {
                    const uint4 q = in[u][kLoads - 1];
                    const uint32_t z[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        v[j] = w[j];
                        v[j + 4] = z[j];
                    }
                }
            } else {
                const T* x = static_cast<const T*>(a.x) + s.row * a.x_stride + s.piece * 8;
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = s.valid ? __float_as_uint(to_float(x[j])) : 0u;
            }
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) top = max(top, v[j] & 0x7FFFFFFFu);
            top = group_max<4>(top);                     // rows are whole blocks: the four lanes are valid together
            const uint32_t field = top >> 23;
            const uint32_t scale = field == 255 ? 255 : field > 2 ? field - 2 : 0;
            uint32_t codes = 0;
            const float sc = scale_operand(scale);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(v[0]), __uint_as_float(v[1]), sc, 0);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(v[2]), __uint_as_float(v[3]), sc, 1);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(v[4]), __uint_as_float(v[5]), sc, 2);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(v[6]), __uint_as_float(v[7]), sc, 3);
            if (field == 255) codes = 0;
            if (!s.valid) continue;
            uint8_t* dst = a.codes + s.row * a.codes_stride + s.piece * 4;
            if constexpr (VEC) {
                *reinterpret_cast<uint32_t*>(dst) = codes;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) dst[j] = uint8_t(codes >> (8 * j));
            }
            if ((s.piece & 3) == 0) a.scales[s.row * a.scales_stride + s.piece / 4] = uint8_t(scale);
        }
    }
}

// ---------------------------------------------------------------- from 4 bits
// 16 bytes of output to a lane.
template <typename T, bool VEC>
__global__ __launch_bounds__(kThreads) void mx_dequantize_kernel(MxRowsArgs a, Shares shares) {
    constexpr int N = sizeof(T) == 2 ? 8 : 4;            // columns to a lane
    for (uint64_t item = blockIdx.x; item < shares.items; item += gridDim.x) {
        const Share s = shares(item);
        if (!s.valid) continue;
        const uint8_t* src = a.codes + s.row * a.codes_stride + s.piece * (N / 2);
        uint32_t codes = 0;
        if constexpr (VEC && N == 8) codes = *reinterpret_cast<const uint32_t*>(src);
        else if constexpr (VEC) codes = *reinterpret_cast<const uint16_t*>(src);
        else {
#pragma unroll
            for (int j = 0; j < N / 2; ++j) codes |= uint32_t(src[j]) << (8 * j);
        }
        const float sc = scale_operand(a.scales[s.row * a.scales_stride + s.piece * N / kMxBlock]);
        T* dst = static_cast<T*>(a.out) + s.row * a.x_stride + s.piece * N;
        uint32_t o[4];
        if constexpr (N == 8) {
            o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, sc, 0));
            o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, sc, 1));
            o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, sc, 2));
            o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, sc, 3));
        } else {
            const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, sc, 0), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, sc, 1);
            o[0] = __float_as_uint(lo[0]);
            o[1] = __float_as_uint(lo[1]);
            o[2] = __float_as_uint(hi[0]);
            o[3] = __float_as_uint(hi[1]);
        }
        if constexpr (VEC) {
            store_stream16(dst, make_uint4(o[0], o[1], o[2], o[3]));
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                if constexpr (N == 8) dst[j].bits = uint16_t(o[j / 2] >> (16 * (j & 1)));
                else dst[j] = __uint_as_float(o[j]);
            }
        }
    }
}

// ---------------------------------------------------------------- SwiGLU
// Pieces of a half row: N neighbouring elements, or one where the halves are not at 16-byte addresses.
template <typename T, int N>
struct Piece {
    float f[N];
    __device__ __forceinline__ void load(const T* p) {
        if constexpr (N == 1) {
            f[0] = to_float(*p);
        } else if constexpr (sizeof(T) == 2) {
            static_assert(N == 8 || N == 4, "pieces of 8 or 16 bytes");
            uint32_t w[4] = {0, 0, 0, 0};
            if constexpr (N == 8) {
                const uint4 v = load_stream16(p);
                w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
            } else {
                const uint2 v = *reinterpret_cast<const uint2*>(p);
                w[0] = v.x; w[1] = v.y;
            }
#pragma unroll
            for (int j = 0; j < N; ++j) f[j] = __uint_as_float((j & 1) ? (w[j / 2] & 0xFFFF0000u) : (w[j / 2] << 16));
        } else {
#pragma unroll
            for (int i = 0; i < N; i += 4) {
                const uint4 v = load_stream16(p + i);
                f[i] = __uint_as_float(v.x);
                f[i + 1] = __uint_as_float(v.y);
                f[i + 2] = __uint_as_float(v.z);
                f[i + 3] = __uint_as_float(v.w);
            }
        }
    }
    __device__ __forceinline__ void store(T* p) const {
        if constexpr (N == 1) {
            from_float(p, f[0]);
        } else if constexpr (sizeof(T) == 2) {
            if constexpr (N == 8)
                store_stream16(p, make_uint4(pack_bf16_rne(f[0], f[1]), pack_bf16_rne(f[2], f[3]), pack_bf16_rne(f[4], f[5]), pack_bf16_rne(f[6], f[7])));
            else
                *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16_rne(f[0], f[1]), pack_bf16_rne(f[2], f[3]));
        } else {
#pragma unroll
            for (int i = 0; i < N; i += 4)
                store_stream16(p + i, make_uint4(__float_as_uint(f[i]), __float_as_uint(f[i + 1]), __float_as_uint(f[i + 2]), __float_as_uint(f[i + 3])));
        }
    }
};

// e^x as a power of 2: 1 / ln 2 in two parts, the second, and what the first rounds off, multiplied on behind the power
constexpr float kLog2E = 0x1.715476p+0f, kLog2ELow = 0x1.4ae0cp-26f, kLn2 = 0x1.62e43p-1f;

// p = 1 / (1 + e^-g) and q = 1 - p, both from t = e^-|g| <= 1, the smaller one as t / (1 + t): neither overflows or is a difference of rounded
// numbers.  The power is the hardware's of 2, the quotient one Newton step on its reciprocal.  Both good to 2 ulp, with half of expf's and the
// division's instructions, of which there were more than memory leaves time for (4097 x 14336 BF16 69 us).  t is 0 where it would be below the
// normal numbers: gates below kFar are not for this.
constexpr float kFar = -87.0f;
__device__ __forceinline__ void sigmoids(float g, float& p, float& q) {
    const float x = -fminf(fabsf(g), 200.0f), y = x * kLog2E, low = fmaf(x, kLog2ELow, fmaf(x, kLog2E, -y));
    float t = __builtin_amdgcn_exp2f(y);
    t = fmaf(t, low * kLn2, t);
    const float d = 1.0f + t;
    float r = __builtin_amdgcn_rcpf(d);
    r = fmaf(fmaf(-d, r, 1.0f), r, r);
    const float s = t * r;
    p = g >= 0.0f ? r : s;
    q = g >= 0.0f ? s : r;
}

// p for gates below kFar, where it is e^g to more digits than are kept.  It may be far below FP32's numbers and h, or a gradient, not: what
// it is multiplied by is in 64 bits, too, and rounded behind the last product.
__device__ __forceinline__ double far_sigmoid(float g) {
    const float x = fmaxf(g, -2000.0f), whole = rintf(x * kLog2E), t = __builtin_amdgcn_exp2f(fmaf(x, kLog2E, -whole));
    return __builtin_amdgcn_ldexp(double(fmaf(t, x * kLog2ELow * kLn2, t)), int(whole));
}
__device__ __forceinline__ bool is_far(float g) { return g < kFar && g > -INFINITY; }    // (of minus infinity all is NaN, as written)
template <int N>
__device__ __forceinline__ bool any_far(const float (&g)[N]) {
    float least = g[0];
#pragma unroll
    for (int j = 1; j < N; ++j) least = fminf(least, g[j]);
    return least < kFar;
}

// h = g / (1 + e^-g) u
template <typename T, typename H, int N>
__global__ __launch_bounds__(kThreads) void swiglu_kernel(SwigluArgs a, Shares shares) {
    for (uint64_t item = blockIdx.x; item < shares.items; item += gridDim.x) {
        const Share s = shares(item);
        if (!s.valid) continue;
        const T* row = static_cast<const T*>(a.gate_up) + s.row * a.in_stride + s.piece * N;
        Piece<T, N> g, u;
        Piece<H, N> h;
        g.load(row);
        u.load(row + a.F);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float p, q;
            sigmoids(g.f[j], p, q);
            h.f[j] = g.f[j] * p * u.f[j];
        }
        if (any_far(g.f)) {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (is_far(g.f[j])) h.f[j] = float(double(g.f[j]) * far_sigmoid(g.f[j]) * double(u.f[j]));
        }
        h.store(static_cast<H*>(a.out) + s.row * a.out_stride + s.piece * N);
    }
}

// d_u = d g p, d_g = d u p (1 + g q) with the sigmoids p and q of g and -g
template <typename T, typename H, int N>
__global__ __launch_bounds__(kThreads) void swiglu_grad_kernel(SwigluArgs a, Shares shares) {
    constexpr int kAtOnce = kSwigluGradAtOnce;
    for (uint64_t item = uint64_t(blockIdx.x) * kAtOnce; item < shares.items; item += uint64_t(kAtOnce) * gridDim.x) {
        Share share[kAtOnce];
        Piece<T, N> g[kAtOnce], up[kAtOnce];
        Piece<H, N> d[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            share[u] = shares(item + u);
            if (!share[u].valid) continue;
            const T* row = static_cast<const T*>(a.gate_up) + share[u].row * a.in_stride + share[u].piece * N;
            g[u].load(row);
            up[u].load(row + a.F);
            d[u].load(static_cast<const H*>(a.d_h) + share[u].row * a.d_stride + share[u].piece * N);
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            if (!share[u].valid) continue;
            Piece<T, N> dg, du;
            auto derive = [&](auto FAR) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    float p, q;
                    sigmoids(g[u].f[j], p, q);
                    du.f[j] = d[u].f[j] * (g[u].f[j] * p);
                    dg.f[j] = d[u].f[j] * up[u].f[j] * (p * fmaf(g[u].f[j], q, 1.0f));
                    if (decltype(FAR)::value && is_far(g[u].f[j])) {
                        const double gate = double(g[u].f[j]), dp = far_sigmoid(g[u].f[j]) * double(d[u].f[j]);
                        du.f[j] = float(gate * dp);
                        dg.f[j] = float((1.0 + gate) * dp * double(up[u].f[j]));
                    }
                }
            };
            // two bodies for the whole wavefront: with a branch behind one (BF16, 4097 x 14336) 97 -> 104 us, so 97 -> 100
            if (__any(any_far(g[u].f))) derive(std::true_type{});
            else derive(std::false_type{});
            T* out = static_cast<T*>(a.out) + share[u].row * a.out_stride + share[u].piece * N;
            dg.store(out);
            du.store(out + a.F);
        }
    }
}

template <typename T>
void go_rows(const MxRowsArgs& a, bool back, hipStream_t stream) {
    const Shares shares(a.rows, a.cols / (back ? (sizeof(T) == 2 ? 8 : 4) : 8));
    const dim3 grid(shares.grid(back ? 1 : kQuantizeAtOnce)), wg(kThreads);
    if (back) {
        if (a.vec) hipLaunchKernelGGL((mx_dequantize_kernel<T, true>), grid, wg, 0, stream, a, shares);
        else hipLaunchKernelGGL((mx_dequantize_kernel<T, false>), grid, wg, 0, stream, a, shares);
    } else {
        if (a.vec) hipLaunchKernelGGL((mx_quantize_kernel<T, true>), grid, wg, 0, stream, a, shares);
        else hipLaunchKernelGGL((mx_quantize_kernel<T, false>), grid, wg, 0, stream, a, shares);
    }
}
hipError_t launch_rows(MxRowsArgs a, bool f32, bool back, hipStream_t stream) {
    // rows without gaps are one long row: no lanes are left over at the ends of short ones
    if (a.x_stride == a.cols && a.codes_stride == a.cols / 2 && a.scales_stride == a.cols / kMxBlock) {
        a.cols *= a.rows;
        a.rows = 1;
    }
    if (f32) go_rows<float>(a, back, stream);
    else go_rows<bf16_t>(a, back, stream);
    return hipGetLastError();
}

template <typename T, typename H>
void go_swiglu(const SwigluArgs& a, bool grad, hipStream_t stream) {
    constexpr int N = kPiece<T, H>;
    const Shares shares(a.rows, a.vec ? a.F / N : a.F);
    const dim3 grid(shares.grid(grad ? kSwigluGradAtOnce : 1)), wg(kThreads);
    if (grad) {
        if (a.vec) hipLaunchKernelGGL((swiglu_grad_kernel<T, H, N>), grid, wg, 0, stream, a, shares);
        else hipLaunchKernelGGL((swiglu_grad_kernel<T, H, 1>), grid, wg, 0, stream, a, shares);
    } else {
        if (a.vec) hipLaunchKernelGGL((swiglu_kernel<T, H, N>), grid, wg, 0, stream, a, shares);
        else hipLaunchKernelGGL((swiglu_kernel<T, H, 1>), grid, wg, 0, stream, a, shares);
    }
}
hipError_t launch_act(const SwigluArgs& a, bool in_f32, bool h_f32, bool grad, hipStream_t stream) {
    if (in_f32) h_f32 ? go_swiglu<float, float>(a, grad, stream) : go_swiglu<float, bf16_t>(a, grad, stream);
    else h_f32 ? go_swiglu<bf16_t, float>(a, grad, stream) : go_swiglu<bf16_t, bf16_t>(a, grad, stream);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_quantize(const MxRowsArgs& a, bool f32, hipStream_t stream) { return launch_rows(a, f32, false, stream); }
hipError_t launch_mx_dequantize(const MxRowsArgs& a, bool f32, hipStream_t stream) { return launch_rows(a, f32, true, stream); }
hipError_t launch_swiglu(const SwigluArgs& a, bool in_f32, bool h_f32, hipStream_t stream) { return launch_act(a, in_f32, h_f32, false, stream); }
hipError_t launch_swiglu_grad(const SwigluArgs& a, bool in_f32, bool h_f32, hipStream_t stream) { return launch_act(a, in_f32, h_f32, true, stream); }

}  // namespace fluxmoe
