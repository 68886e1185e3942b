// The norms around a block and what lies between them, for a row y of the block's output and the residual stream's row x:
//   y' = y * rstd(y) * w_post       (y itself where there is no norm behind the block)
//   r  = x + scale * g * y'         (g: 1, one number for the token, or one for each channel; raw or through a sigmoid)
//   n  = r * rstd(r) * w_pre        rstd(v) = 1 / sqrt(mean(v^2) + eps)
// and the gradients of x, y, g, w_pre and w_post.  All in FP32 between one read of the inputs and one write of the outputs; n
// is taken from r before r is rounded.
//
// A row is a few hundred wide additions and one or two reductions: bound by memory.  A lane holds eight columns in registers from
// load to store, a row is spread over as many wavefronts as that takes (up to 16: 8192 columns), and a workgroup has several
// rows where a row is short.  One to three workgroups run on a CU; each keeps its columns' weights in registers and walks through
// the rows, the next row's loads under way while it works on one.  With a workgroup for every row instead, a row's loads,
// reductions and stores follow each other and the weights come again from the caches: 8192 x 5120 118 us against 84.
// Measured, of 6.6 TB/s that a copy reaches (us): 8192 x 5120, BF16 y, FP32 stream, norms on both sides and a channel's gate
// 84 (6.0 TB/s); 256 x 4096 4.2, of which 2.1 are the launch's; 1 x 2048 2.3.  Gradient of 8192 x 4096, all BF16, both norms, channel's
// gate 68 (5.9 TB/s) and 4.8 for the sums over the tokens.
#include "block_device.h"
#include "block_ops.h"

namespace fluxmoe {
namespace {

constexpr uint32_t kRowColumns = 8192;       // what 16 wavefronts hold in registers

// What a call has beside the residual stream and the norm of it.
enum Mode {
    kAlone,      // nothing: the norm alone
    kAdd,        // y, with one factor for a token at most
    kScaled,     // y with a gate for each channel
    kPost,       // y through a norm of its own, with or without a gate
};

// N sums over the `waves` wavefronts of a row, in a fixed order, to all lanes.  `s`: LDS that no wavefront of the row may still be
// reading from a call before.  The wavefronts' parts are fetched by 16 lanes each and added up between them.
template <int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*s)[16], uint32_t waves) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = group_sum<64>(v[i]);
    if (waves == 1) return;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = __builtin_amdgcn_readfirstlane(wave / waves * waves);
    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) s[i][wave] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const uint32_t which = i + (lane >> 4), w = lane & 15;
        const float part = group_sum<16>(which < N && w < waves ? s[which < N ? which : 0][first + (w < waves ? w : 0)] : 0.0f);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k < N) v[i + k] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(part), 16 * k));
    }
}

__device__ __forceinline__ float weight_at(const NormArgs& a, const void* w, uint32_t c) {
    const float v = a.weight_f32 ? static_cast<const float*>(w)[c] : to_float(static_cast<const bf16_t*>(w)[c]);
    return a.zero_centred ? v + 1.0f : v;
}
template <int N>
__device__ __forceinline__ void weights_at(const NormArgs& a, const void* w, uint32_t c, float* f) {
    const float one = a.zero_centred ? 1.0f : 0.0f;
    if (a.weight_f32) {
        Pack<float, N> p;
        p.template load<kCached>(row_at(static_cast<const float*>(w), 0, 0, a.H), c);
#pragma unroll
        for (int j = 0; j < N; ++j) f[j] = p[j] + one;
    } else {
        Pack<bf16_t, N> p;
        p.template load<kCached>(row_at(static_cast<const bf16_t*>(w), 0, 0, a.H), c);
#pragma unroll
        for (int j = 0; j < N; ++j) f[j] = p[j] + one;
    }
}
__device__ __forceinline__ float gate_value(const NormArgs& a, float v) { return a.gate_sigmoid ? sigmoid(v) : v; }
// The gate's derivative by what is read: a sigmoid's by e = e^-|v|, as 1 - g of a rounded g has three digits left at v = 10 and none
// from 17 on.
__device__ __forceinline__ float gate_slope(const NormArgs& a, float v) {
    if (!a.gate_sigmoid) return 1.0f;
    const float e = expf(-fabsf(v)), one_e = 1.0f + e;
    return e / (one_e * one_e);
}
template <int N>
__device__ __forceinline__ void gates_at(const NormArgs& a, uint32_t c, float* f) {
    Pack<float, N> p;
    p.template load<kCached>(row_at(a.gate, 0, 0, a.H), c);
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = gate_value(a, p[j]);
}
__device__ __forceinline__ float rstd_of(const NormArgs& a, float squares) { return rsqrtf(squares / float(a.H) + a.eps); }
// What y is multiplied by in a column: the weight of the norm behind the block times the channel's gate.
template <int N>
__device__ __forceinline__ void column_factors(const NormArgs& a, uint32_t c, float* f) {
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = 1.0f;
    if (a.w_post) weights_at<N>(a, a.w_post, c, f);
    if (a.gate_channel) {
        float g[N];
        gates_at<N>(a, c, g);
#pragma unroll
        for (int j = 0; j < N; ++j) f[j] *= g[j];
    }
}

// ================================================================ forward
template <typename Y, typename R, Mode MODE>
__global__ __launch_bounds__(1024) void norm_kernel(NormArgs a, uint32_t waves, uint32_t rows_per_wg) {
    constexpr int N = kPiece<Y, R>, P = 8 / N;           // columns of a piece, pieces of a lane
    __shared__ float s_y[2][1][16], s_r[2][1][16];       // of rows that follow each other, in turn
    const uint32_t per_row = waves * 64, step = gridDim.x * rows_per_wg;
    const uint32_t mine = __builtin_amdgcn_readfirstlane(threadIdx.x / per_row);
    uint32_t c[P];
    float w_pre[P][N], w_y[P][N];
    Pack<Y, N> next_y[P];
    Pack<R, N> next_x[P];
    auto fetch = [&](uint32_t t) {
        const uint32_t columns = t < a.T ? a.H : 0;
        const row_t x = row_at(static_cast<const R*>(a.residual), t, a.residual_stride, columns);
        const row_t y = row_at(static_cast<const Y*>(a.y), t, a.y_stride, columns);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            next_x[p].template load<kStream>(x, c[p]);
            if (MODE != kAlone) next_y[p].template load<kStream>(y, c[p]);
        }
    };
#pragma unroll
    for (int p = 0; p < P; ++p) c[p] = (p * per_row + threadIdx.x % per_row) * N;
    fetch(blockIdx.x * rows_per_wg + mine);
#pragma unroll
    for (int p = 0; p < P; ++p) {
        weights_at<N>(a, a.w_pre, c[p], w_pre[p]);
        if (MODE == kScaled || MODE == kPost) column_factors<N>(a, c[p], w_y[p]);
    }
    uint32_t turn = 0;
    for (uint32_t base = blockIdx.x * rows_per_wg; base < a.T; base += step, turn ^= 1) {   // as often for the whole workgroup
        const uint32_t t = base + mine;
        Pack<Y, N> y[P];
        float r[P][N];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            y[p] = next_y[p];
#pragma unroll
            for (int j = 0; j < N; ++j) r[p][j] = next_x[p][j];
        }
        fetch(t + step);
        if constexpr (MODE != kAlone) {
            float scale = a.scale;
            if (a.gate_token) scale *= gate_value(a, scalar_at(a.gate, min(t, a.T - 1)));
            if constexpr (MODE == kPost) {
                float sq[1] = {0.0f};
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int j = 0; j < N; ++j) sq[0] += y[p][j] * y[p][j];
                row_sums<1>(sq, s_y[turn], waves);
                scale *= rstd_of(a, sq[0]);
            }
#pragma unroll
            for (int p = 0; p < P; ++p) {
#pragma unroll
                for (int j = 0; j < N; ++j) r[p][j] += y[p][j] * scale * (MODE == kAdd ? 1.0f : w_y[p][j]);
            }
        }
        float sq[1] = {0.0f};
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int j = 0; j < N; ++j) sq[0] += r[p][j] * r[p][j];
        row_sums<1>(sq, s_r[turn], waves);
        const float rstd = rstd_of(a, sq[0]);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            next_x[p].arrive();
            if (MODE != kAlone) next_y[p].arrive();
        }
        const uint32_t columns = t < a.T ? a.H : 0;
        const row_t r_out = row_at(static_cast<R*>(a.residual_out), t, a.residual_out_stride, columns);
        const row_t n_out = row_at(reinterpret_cast<bf16_t*>(a.normed), t, a.normed_stride, columns);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (MODE != kAlone) store<R, N, kStream>(r_out, c[p], r[p]);
#pragma unroll
            for (int j = 0; j < N; ++j) r[p][j] *= rstd * w_pre[p][j];
            store<bf16_t, N, kStream>(n_out, c[p], r[p]);
        }
    }
}

// Any width and alignment: a column at a time, the row read again for each reduction.  Slower where rows outgrow the caches.
template <typename Y, typename R>
__global__ __launch_bounds__(1024) void norm_any_kernel(NormArgs a) {
    __shared__ float s_y[1][16], s_r[1][16];
    const uint32_t t = blockIdx.x, waves = blockDim.x / 64;
    const Y* y = static_cast<const Y*>(a.y) + t * a.y_stride;
    const R* x = static_cast<const R*>(a.residual) + t * a.residual_stride;
    float scale = a.scale;
    if (a.gate_token) scale *= gate_value(a, a.gate[t]);
    if (a.w_post) {
        float sq[1] = {0.0f};
        for (uint32_t c = threadIdx.x; c < a.H; c += blockDim.x) sq[0] += to_float(y[c]) * to_float(y[c]);
        row_sums<1>(sq, s_y, waves);
        scale *= rstd_of(a, sq[0]);
    }
    auto sum_at = [&](uint32_t c) {
        float v = to_float(x[c]);
        if (a.y) {
            float p = to_float(y[c]) * scale;
            if (a.w_post) p *= weight_at(a, a.w_post, c);
            if (a.gate_channel) p *= gate_value(a, a.gate[c]);
            v += p;
        }
        return v;
    };
    float sq[1] = {0.0f};
    for (uint32_t c = threadIdx.x; c < a.H; c += blockDim.x) {
        const float v = sum_at(c);
        sq[0] += v * v;
    }
    row_sums<1>(sq, s_r, waves);
    const float rstd = rstd_of(a, sq[0]);
    for (uint32_t c = threadIdx.x; c < a.H; c += blockDim.x) {
        const float v = sum_at(c);
        if (a.y && a.residual_out) from_float(static_cast<R*>(a.residual_out) + t * a.residual_out_stride + c, v);
        from_float(reinterpret_cast<bf16_t*>(a.normed) + t * a.normed_stride + c, v * (rstd * weight_at(a, a.w_pre, c)));
    }
}

// ================================================================ gradient
// With h = r rstd(r) and dn, dr_out the gradients of n and r:
//   dr = dr_out + rstd (dn w_pre - h mean(dn w_pre h)) = dx        d w_pre = sum_t dn h
//   dg = scale sum dr y' (over the channels for a token's gate, over the tokens for a channel's)
//   dy' = scale g dr, and through the norm behind the block as above: dy and d w_post.
// With hy = y rstd(y) (y where there is no norm behind the block) the sums over the tokens for w_post and a channel's gate are
// one sum s_y = sum_t scale g_token dr hy: d w_post = g_channel s_y, d g_channel = w_post s_y.
// dr is linear in rstd and the mean, so that what dy and a token's gate need of dr is put together from sums that need no dr:
// one reduction, and one barrier, for a row.  With q = y w_post g_channel:
//   sum dr q = sum dr_out q + rstd (sum dn w_pre q - rstd mean sum r q)
// A workgroup takes every grid-th row and keeps its columns' sums over the tokens in registers; column_sum_kernel adds up the
// workgroups' sums in a fixed order.
template <typename Y, typename R, Mode MODE, bool D_OUT>
struct GradRow {
    static constexpr int N = kPiece<Y, R>, P = 8 / N;    // columns of a piece, pieces of a lane
    Pack<R, N> r[P], d_out[P];
    Pack<bf16_t, N> dn[P];
    Pack<Y, N> y[P];
    __device__ __forceinline__ void arrive() {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            r[p].arrive();
            dn[p].arrive();
            if (D_OUT) d_out[p].arrive();
            if (MODE != kAlone) y[p].arrive();
        }
    }
    __device__ __forceinline__ void load(const NormArgs& a, uint32_t t, const uint32_t (&c)[P]) {
        const uint32_t columns = t < a.T ? a.H : 0;
        const row_t br = row_at(static_cast<const R*>(a.residual), t, a.residual_stride, columns);
        const row_t bn = row_at(reinterpret_cast<const bf16_t*>(a.d_normed), t, a.d_normed_stride, columns);
        const row_t bo = row_at(static_cast<const R*>(a.d_residual_out), t, a.d_residual_out_stride, columns);
        const row_t by = row_at(static_cast<const Y*>(a.y), t, a.y_stride, columns);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            r[p].template load<kStream>(br, c[p]);
            dn[p].template load<kStream>(bn, c[p]);
            if (D_OUT) d_out[p].template load<kStream>(bo, c[p]);
            if (MODE != kAlone) y[p].template load<kStream>(by, c[p]);
        }
    }
};

__device__ __forceinline__ float* partial_row(const NormArgs& a, uint32_t sum, uint32_t part) {
    return a.partials + (uint64_t(sum) * a.n_partials + part) * a.H;
}

// WAVES: the most wavefronts of a workgroup, 8 or 16.  With FP32 rows no more than 8 run on a CU where a row needs no more, and
// each lane may have 256 registers: within the 128 of 16 wavefronts the form with all its parts spills (20480 x 2048 FP32 151 us,
// spilling 175).  BF16 rows fit 128, and are faster compiled for them (10240 x 4096 89 us, compiled for 256 98).
template <typename Y, typename R, Mode MODE, bool D_OUT, int WAVES>
__global__ __launch_bounds__((kPiece<Y, R> == 8 ? 1024 : WAVES * 64)) void norm_grad_kernel(NormArgs a, uint32_t waves, uint32_t rows_per_wg) {
    typedef GradRow<Y, R, MODE, D_OUT> Row;
    constexpr int N = Row::N, P = Row::P;
    constexpr bool FACTORS = MODE == kScaled || MODE == kPost;
    __shared__ float s[2][6][16];                        // of rows that follow each other, in turn
    const uint32_t per_row = waves * 64, step = gridDim.x * rows_per_wg;
    const uint32_t mine = __builtin_amdgcn_readfirstlane(threadIdx.x / per_row);
    uint32_t c[P];
    float w_pre[P][N], w_y[P][N], sum_pre[P][N] = {}, sum_y[P][N] = {};
#pragma unroll
    for (int p = 0; p < P; ++p) c[p] = (p * per_row + threadIdx.x % per_row) * N;
    Row next;
    next.load(a, blockIdx.x * rows_per_wg + mine, c);
#pragma unroll
    for (int p = 0; p < P; ++p) {
        weights_at<N>(a, a.w_pre, c[p], w_pre[p]);
        if (FACTORS) column_factors<N>(a, c[p], w_y[p]);
    }
    const float inv_h = 1.0f / float(a.H);
    uint32_t turn = 0;
    for (uint32_t base = blockIdx.x * rows_per_wg; base < a.T; base += step, turn ^= 1) {   // as often for the whole workgroup
        const uint32_t t = base + mine;
        const Row row = next;
        next.load(a, t + step, c);
        float v[6] = {};
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float r = row.r[p][j], dw = row.dn[p][j] * w_pre[p][j];
                v[0] += r * r;
                v[1] += dw * r;
                if (MODE == kAdd || MODE == kPost) {
                    const float y = row.y[p][j], q = FACTORS ? y * w_y[p][j] : y;
                    if (D_OUT) v[2] += row.d_out[p][j] * q;
                    v[3] += dw * q;
                    v[4] += r * q;
                    if (MODE == kPost) v[5] += y * y;
                }
            }
        if constexpr (MODE == kAdd || MODE == kPost) {
            row_sums<6>(v, s[turn], waves);
        } else {
            float two[2] = {v[0], v[1]};
            row_sums<2>(two, s[turn], waves);
            v[0] = two[0];
            v[1] = two[1];
        }
        const bool here = t < a.T;                       // a row that is not there adds 0, also where eps is 0
        const float rstd = here ? rstd_of(a, v[0]) : 0.0f, mean = v[1] * rstd * inv_h;
        const float rstd_y = MODE != kPost ? 1.0f : here ? rstd_of(a, v[5]) : 0.0f;
        float scale = a.scale;
        if (MODE != kAlone && a.gate_token) scale = here ? scale * gate_value(a, scalar_at(a.gate, min(t, a.T - 1))) : 0.0f;
        const float dot = (v[2] + rstd * (v[3] - rstd * mean * v[4])) * rstd_y;             // sum dr w_post g_channel hy
        const float mean_y = MODE == kPost ? scale * dot * inv_h : 0.0f;                     // mean(dy' w_post hy)
        float dr[P][N], dy[P][N];
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float h = row.r[p][j] * rstd;
                dr[p][j] = (D_OUT ? row.d_out[p][j] : 0.0f) + rstd * (row.dn[p][j] * w_pre[p][j] - h * mean);
                sum_pre[p][j] += row.dn[p][j] * h;
                if (MODE != kAlone) {
                    const float hy = MODE == kPost ? row.y[p][j] * rstd_y : row.y[p][j];
                    dy[p][j] = scale * dr[p][j];
                    if (FACTORS) {
                        sum_y[p][j] += dy[p][j] * hy;
                        dy[p][j] *= w_y[p][j];
                    }
                    if (MODE == kPost) dy[p][j] = rstd_y * (dy[p][j] - hy * mean_y);
                }
            }
        next.arrive();
        const uint32_t columns = here ? a.H : 0;
        const row_t r_out = row_at(static_cast<R*>(a.d_residual), t, a.d_residual_stride, columns);
        const row_t y_out = row_at(static_cast<Y*>(a.d_y), t, a.d_y_stride, columns);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            store<R, N, kStream>(r_out, c[p], dr[p]);
            if (MODE != kAlone) store<Y, N, kStream>(y_out, c[p], dy[p]);
        }
        if ((MODE == kAdd || MODE == kPost) && a.gate_token) {
            const float v_gate = scalar_at(a.gate, min(t, a.T - 1));
            if (c[0] == 0 && here) a.d_gate[t] = a.scale * dot * gate_slope(a, v_gate);
        }
    }
    // the sums of the rows side by side in a workgroup become one, by way of LDS and in their order
    __shared__ float s_sum[2][WAVES == 8 ? 2048 : 1];    // [row][column]: 4 rows of up to 512, or 2 of up to 1024
    if (WAVES == 8 && rows_per_wg > 1) {
        if (mine > 0) {
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    s_sum[0][mine * per_row * 8 + c[p] + j] = sum_pre[p][j];
                    if (FACTORS) s_sum[1][mine * per_row * 8 + c[p] + j] = sum_y[p][j];
                }
        }
        __syncthreads();
        if (mine > 0) return;
        for (uint32_t i = 1; i < rows_per_wg; ++i)
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    sum_pre[p][j] += s_sum[0][i * per_row * 8 + c[p] + j];
                    if (FACTORS) sum_y[p][j] += s_sum[1][i * per_row * 8 + c[p] + j];
                }
    }
    const row_t to_pre = row_at(partial_row(a, 0, blockIdx.x), 0, 0, a.H), to_y = row_at(partial_row(a, 1, blockIdx.x), 0, 0, a.H);
#pragma unroll
    for (int p = 0; p < P; ++p) {
        store<float, N, kCached>(to_pre, c[p], sum_pre[p]);
        if (FACTORS) store<float, N, kCached>(to_y, c[p], sum_y[p]);
    }
}

// Any width and alignment, as norm_any_kernel; the sums over the tokens are kept in the workgroup's partial rows.
template <typename Y, typename R>
__global__ __launch_bounds__(1024) void norm_grad_any_kernel(NormArgs a) {
    __shared__ float s_a[3][16], s_b[1][16];
    const uint32_t waves = blockDim.x / 64;
    const float inv_h = 1.0f / float(a.H);
    const bool factors = a.w_post || a.gate_channel;
    float* sum_pre = partial_row(a, 0, blockIdx.x);
    float* sum_y = partial_row(a, 1, blockIdx.x);
    for (uint32_t c = threadIdx.x; c < a.H; c += blockDim.x) {
        sum_pre[c] = 0.0f;
        if (factors) sum_y[c] = 0.0f;
    }
    auto factor_at = [&](uint32_t c) { return (a.w_post ? weight_at(a, a.w_post, c) : 1.0f) * (a.gate_channel ? gate_value(a, a.gate[c]) : 1.0f); };
    for (uint32_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        const Y* y = static_cast<const Y*>(a.y) + t * a.y_stride;
        const R* r = static_cast<const R*>(a.residual) + t * a.residual_stride;
        const R* d_out = static_cast<const R*>(a.d_residual_out) + t * a.d_residual_out_stride;
        const bf16_t* dn = reinterpret_cast<const bf16_t*>(a.d_normed) + t * a.d_normed_stride;
        float v[3] = {0.0f, 0.0f, 0.0f};
        for (uint32_t c = threadIdx.x; c < a.H; c += blockDim.x) {
            const float x = to_float(r[c]), q = a.y ? to_float(y[c]) : 0.0f;
            v[0] += x * x;
            v[1] += to_float(dn[c]) * weight_at(a, a.w_pre, c) * x;
            v[2] += q * q;
        }
        row_sums<3>(v, s_a, waves);
        const float rstd = rstd_of(a, v[0]), mean = v[1] * rstd * inv_h;
        const float rstd_y = a.w_post ? rstd_of(a, v[2]) : 1.0f;
        const float scale = a.gate_token ? a.scale * gate_value(a, a.gate[t]) : a.scale;
        auto dr_at = [&](uint32_t c) {
            const float h = to_float(r[c]) * rstd;
            return (a.d_residual_out ? to_float(d_out[c]) : 0.0f) + rstd * (to_float(dn[c]) * weight_at(a, a.w_pre, c) - h * mean);
        };
        float dot[1] = {0.0f};
        if (a.gate_token || a.w_post) {
            for (uint32_t c = threadIdx.x; c < a.H; c += blockDim.x) dot[0] += dr_at(c) * to_float(y[c]) * rstd_y * factor_at(c);
            row_sums<1>(dot, s_b, waves);
        }
        const float mean_y = a.w_post ? scale * dot[0] * inv_h : 0.0f;
        for (uint32_t c = threadIdx.x; c < a.H; c += blockDim.x) {
            const float dr = dr_at(c);
            sum_pre[c] += to_float(dn[c]) * to_float(r[c]) * rstd;
            if (a.y) {
                const float hy = to_float(y[c]) * rstd_y;
                float dy = scale * dr;
                if (factors) {
                    sum_y[c] += dy * hy;
                    dy *= factor_at(c);
                }
                if (a.w_post) dy = rstd_y * (dy - hy * mean_y);
                from_float(static_cast<Y*>(a.d_y) + t * a.d_y_stride + c, dy);
            }
            from_float(static_cast<R*>(a.d_residual) + t * a.d_residual_stride + c, dr);
        }
        if (a.gate_token && threadIdx.x == 0) a.d_gate[t] = a.scale * dot[0] * gate_slope(a, a.gate[t]);
        __syncthreads();
    }
}

// A workgroup adds up 16 columns: 64 groups of threads take every 64th partial sum, then their sums are added in order (256 partial
// sums of 4096 columns, two kinds: 4.8 us, the launch included).
__global__ __launch_bounds__(256) void column_sum_kernel(NormArgs a) {
    __shared__ float s[64][17];
    const uint32_t c = blockIdx.x * 16, lane = threadIdx.x & 3, group = threadIdx.x >> 2, c4 = c + lane * 4;
    float v[4] = {};
    const bool whole = a.H % 4 == 0;
    if (c4 < a.H) {
#pragma unroll 4
        for (uint32_t p = group; p < a.n_partials; p += 64) {
            const float* row = partial_row(a, blockIdx.y, p) + c4;
            if (whole) {
                const float4 q = *reinterpret_cast<const float4*>(row);
                v[0] += q.x; v[1] += q.y; v[2] += q.z; v[3] += q.w;
            } else {
                for (uint32_t j = 0; j < 4 && c4 + j < a.H; ++j) v[j] += row[j];
            }
        }
    }
    for (int j = 0; j < 4; ++j) s[group][lane * 4 + j] = v[j];
    __syncthreads();
    // 16 threads of a wavefront's quarter share a column: every 16th group's sum, then across the lanes
    const uint32_t col = threadIdx.x >> 4, part = threadIdx.x & 15;
    const float sum = group_sum<16>(s[part][col] + s[part + 16][col] + s[part + 32][col] + s[part + 48][col]);
    const uint32_t to = c + col;
    if (part != 0 || to >= a.H) return;
    if (blockIdx.y == 0) {
        a.d_w_pre[to] = sum;
        return;
    }
    const float g = a.gate_channel ? gate_value(a, a.gate[to]) : 1.0f;
    if (a.w_post) a.d_w_post[to] = g * sum;
    if (a.gate_channel) a.d_gate[to] = (a.w_post ? weight_at(a, a.w_post, to) : 1.0f) * sum * gate_slope(a, a.gate[to]);
}

uint32_t any_threads(uint32_t H) { return H >= 1024 ? 1024 : (H + 63) / 64 * 64; }

// Wavefronts that a CU's workgroups are to have together.  Few, with the next row's loads under way, read and write in longer
// runs than many (8192 x 5120 to 163840 x 256, all kinds of call): forward with 8 / 12 / 16 to a CU 5.8-6.2 / 5.8-6.2 /
// 5.4-6.1 TB/s where FP32 rows take part, 5.0-5.9 / 5.6-6.1 / 5.4-6.0 where all are BF16; gradient with 4 / 8 / 16 to a CU 5.6-6.1 /
// 5.3-6.0 / 4.8-5.8 and 4.6-5.8 / 5.1-5.8 / 4.6-5.7.  Rows of up to 512 columns need 8 for the gradient (4.0, 5.4 with 8).
constexpr uint32_t kMostGradWaves = 8;
template <typename Y, typename R>
uint32_t forward_waves() { return sizeof(Y) == 2 && sizeof(R) == 2 ? 12 : 8; }
template <typename Y, typename R>
uint32_t grad_waves(uint32_t H) { return (sizeof(Y) == 2 && sizeof(R) == 2) || H <= 512 ? kMostGradWaves : 4; }

// Workgroups that walk through the rows: what the 256 CUs get, or one row (one group of short rows) to each if there are fewer.
uint32_t walkers(const RowShape& s, uint32_t T, uint32_t wave_slots) {
    const uint32_t in_wg = s.waves * s.rows_per_wg, most = 256 * (wave_slots > in_wg ? wave_slots / in_wg : 1);
    const uint32_t need = (T + s.rows_per_wg - 1) / s.rows_per_wg;
    return need < most ? need : most;
}

Mode mode_of(const NormArgs& a) { return !a.y ? kAlone : a.w_post ? kPost : a.gate_channel ? kScaled : kAdd; }

template <typename Y, typename R, Mode MODE>
void go_rows(const NormArgs& a, hipStream_t stream) {
    const RowShape s = row_shape(a.H);
    hipLaunchKernelGGL((norm_kernel<Y, R, MODE>), dim3(walkers(s, a.T, forward_waves<Y, R>())), dim3(s.threads()), 0, stream, a, s.waves, s.rows_per_wg);
}

template <typename Y, typename R>
hipError_t go(const NormArgs& a, bool vec, hipStream_t stream) {
    if (!vec || a.H > kRowColumns) {
        hipLaunchKernelGGL((norm_any_kernel<Y, R>), dim3(a.T), dim3(any_threads(a.H)), 0, stream, a);
    } else {
        switch (mode_of(a)) {
            case kAlone: go_rows<R, R, kAlone>(a, stream); break;
            case kAdd: go_rows<Y, R, kAdd>(a, stream); break;
            case kScaled: go_rows<Y, R, kScaled>(a, stream); break;
            case kPost: go_rows<Y, R, kPost>(a, stream); break;
        }
    }
    return hipGetLastError();
}

template <typename Y, typename R, Mode MODE, bool D_OUT>
void go_grad_rows(const NormArgs& a, const RowShape& s, hipStream_t stream) {
    if (s.waves <= 8) hipLaunchKernelGGL((norm_grad_kernel<Y, R, MODE, D_OUT, 8>), dim3(a.n_partials), dim3(s.threads()), 0, stream, a, s.waves, s.rows_per_wg);
    else hipLaunchKernelGGL((norm_grad_kernel<Y, R, MODE, D_OUT, 16>), dim3(a.n_partials), dim3(s.threads()), 0, stream, a, s.waves, s.rows_per_wg);
}

template <typename Y, typename R, Mode MODE>
void go_grad_rows(NormArgs& a, hipStream_t stream) {
    const RowShape s = row_shape(a.H);
    a.n_partials = walkers(s, a.T, grad_waves<Y, R>(a.H));
    if (a.d_residual_out) go_grad_rows<Y, R, MODE, true>(a, s, stream);
    else go_grad_rows<Y, R, MODE, false>(a, s, stream);
}

template <typename Y, typename R>
hipError_t go_grad(NormArgs a, bool vec, hipStream_t stream) {
    if (a.T == 0) {
        a.n_partials = 0;
    } else if (!vec || a.H > kRowColumns) {
        a.n_partials = a.T < 256 ? a.T : 256;
        hipLaunchKernelGGL((norm_grad_any_kernel<Y, R>), dim3(a.n_partials), dim3(any_threads(a.H)), 0, stream, a);
    } else {
        switch (mode_of(a)) {
            case kAlone: go_grad_rows<R, R, kAlone>(a, stream); break;
            case kAdd: go_grad_rows<Y, R, kAdd>(a, stream); break;
            case kScaled: go_grad_rows<Y, R, kScaled>(a, stream); break;
            case kPost: go_grad_rows<Y, R, kPost>(a, stream); break;
        }
    }
    const uint32_t n_sums = a.w_post || a.gate_channel ? 2 : 1;          // also of no tokens, where y's address says nothing
    hipLaunchKernelGGL(column_sum_kernel, dim3((a.H + 15) / 16, n_sums), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

uint32_t norm_grad_partials(uint32_t T, uint32_t H) {
    const RowShape s = row_shape(H);
    const uint32_t rows = walkers(s, T, kMostGradWaves), any = T < 256 ? T : 256;
    return H <= kRowColumns && rows > any ? rows : any;
}

hipError_t launch_block_norm(const NormArgs& a, bool y_f32, bool residual_f32, bool vec, hipStream_t stream) {
    if (y_f32) return residual_f32 ? go<float, float>(a, vec, stream) : go<float, bf16_t>(a, vec, stream);
    return residual_f32 ? go<bf16_t, float>(a, vec, stream) : go<bf16_t, bf16_t>(a, vec, stream);
}

hipError_t launch_block_norm_grad(const NormArgs& a, bool y_f32, bool residual_f32, bool vec, hipStream_t stream) {
    if (y_f32) return residual_f32 ? go_grad<float, float>(a, vec, stream) : go_grad<float, bf16_t>(a, vec, stream);
    return residual_f32 ? go_grad<bf16_t, float>(a, vec, stream) : go_grad<bf16_t, bf16_t>(a, vec, stream);
}

}  // namespace fluxmoe
