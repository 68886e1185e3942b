// The norms around a block and what lies between them, for a row y of the block's output and the residual stream's row x:
//   y' = y * rstd(y) * w_post       (y itself where there is no norm behind the block)
//   r  = x + scale * g * y'         (g: 1, one number for the token, or one for each channel; raw or through a sigmoid)
//   n  = r * rstd(r) * w_pre        rstd(v) = 1 / sqrt(mean(v^2) + eps)
// and the gradients of x, y, g, w_pre and w_post.  All in FP32 between one read of the inputs and one write of the outputs; n
// is taken from r before r is rounded.
//
// A row is a few hundred wide additions and two reductions: bound by memory.  A lane holds eight neighbouring columns in
// registers from load to store, a row is spread over as many wavefronts as that takes (up to 16: 8192 columns), and a
// workgroup has several rows where a row is short.
#include "block_device.h"
#include "block_ops.h"

namespace fluxmoe {
namespace {

constexpr uint32_t kRowColumns = 8192;       // what 16 wavefronts hold in registers

// N sums over the `waves` wavefronts of a row, in a fixed order.  `s`: LDS of its own for each call in a row's course.
template <int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*s)[N], uint32_t waves) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = group_sum<64>(v[i]);
    if (waves == 1) return;
    const uint32_t wave = threadIdx.x >> 6, first = wave / waves * waves;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) s[wave][i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.0f;
    for (uint32_t w = 0; w < waves; ++w)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += s[first + w][i];
}

__device__ __forceinline__ float weight_at(const NormArgs& a, const void* w, uint32_t c) {
    const float v = a.weight_f32 ? static_cast<const float*>(w)[c] : to_float(static_cast<const bf16_t*>(w)[c]);
    return a.zero_centred ? v + 1.0f : v;
}
__device__ __forceinline__ void weight_at8(const NormArgs& a, const void* w, uint32_t c, float (&f)[8]) {
    const float one = a.zero_centred ? 1.0f : 0.0f;
    if (a.weight_f32) {
        Pack8<float> p;
        p.load(static_cast<const float*>(w) + c);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = p[j] + one;
    } else {
        Pack8<bf16_t> p;
        p.load(static_cast<const bf16_t*>(w) + c);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = p[j] + one;
    }
}
__device__ __forceinline__ float gate_value(const NormArgs& a, float v) { return a.gate_sigmoid ? sigmoid(v) : v; }
__device__ __forceinline__ float rstd_of(const NormArgs& a, float squares) { return rsqrtf(squares / float(a.H) + a.eps); }

// ================================================================ forward
template <typename Y, typename R>
__global__ __launch_bounds__(1024) void norm_kernel(NormArgs a, uint32_t waves, uint32_t rows_per_wg) {
    __shared__ float s_y[16][1], s_r[16][1];
    const uint32_t per_row = waves * 64;
    const uint32_t t = __builtin_amdgcn_readfirstlane(blockIdx.x * rows_per_wg + threadIdx.x / per_row);
    const uint32_t c = threadIdx.x % per_row * 8;
    const bool on = t < a.T && c < a.H;
    Pack8<Y> py;
    Pack8<R> px;
    py.zero();
    px.zero();
    float w_pre[8], w_post[8], g[8];
    if (on) {
        px.load_stream(static_cast<const R*>(a.residual) + t * a.residual_stride + c);
        if (a.y) py.load_stream(static_cast<const Y*>(a.y) + t * a.y_stride + c);
        weight_at8(a, a.w_pre, c, w_pre);
        if (a.w_post) weight_at8(a, a.w_post, c, w_post);
        if (a.gate_channel) {
            Pack8<float> p;
            p.load(a.gate + c);
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = gate_value(a, p[j]);
        }
    }
    float r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = px[j];
    if (a.y) {
        float scale = a.scale;
        if (a.gate_token) scale *= gate_value(a, a.gate[t < a.T ? t : 0]);
        if (a.w_post) {
            float sq[1] = {0.0f};
#pragma unroll
            for (int j = 0; j < 8; ++j) sq[0] += py[j] * py[j];
            row_sums<1>(sq, s_y, waves);
            scale *= rstd_of(a, sq[0]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float v = py[j] * scale;
            if (a.w_post) v *= w_post[j];
            if (a.gate_channel) v *= g[j];
            r[j] = on ? r[j] + v : 0.0f;
        }
        if (on && a.residual_out) store8_stream(static_cast<R*>(a.residual_out) + t * a.residual_out_stride + c, r);
    }
    float sq[1] = {0.0f};
#pragma unroll
    for (int j = 0; j < 8; ++j) sq[0] += r[j] * r[j];
    row_sums<1>(sq, s_r, waves);
    const float rstd = rstd_of(a, sq[0]);
    if (!on) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] *= rstd * w_pre[j];
    store8(reinterpret_cast<bf16_t*>(a.normed) + t * a.normed_stride + c, r);
}

// Any width and alignment: a column at a time, the row read again for each reduction.  Slower where rows outgrow the caches.
template <typename Y, typename R>
__global__ __launch_bounds__(1024) void norm_any_kernel(NormArgs a) {
    __shared__ float s_y[16][1], s_r[16][1];
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
// A workgroup takes every grid-th row and keeps its columns' sums over the tokens in registers; column_sum_kernel adds up the
// workgroups' sums in a fixed order.
struct GradSums {
    float w_pre[8], w_post[8], gate[8];
};

template <typename Y, typename R>
struct GradRow {
    Pack8<R> r, d_out;
    Pack8<bf16_t> dn;
    Pack8<Y> y;
    __device__ __forceinline__ void load(const NormArgs& a, uint32_t t, uint32_t c, bool on) {
        if (on) {
            r.load_stream(static_cast<const R*>(a.residual) + t * a.residual_stride + c);
            dn.load_stream(reinterpret_cast<const bf16_t*>(a.d_normed) + t * a.d_normed_stride + c);
            if (a.d_residual_out) d_out.load_stream(static_cast<const R*>(a.d_residual_out) + t * a.d_residual_out_stride + c);
            else d_out.zero();
            if (a.y) y.load_stream(static_cast<const Y*>(a.y) + t * a.y_stride + c);
            else y.zero();
        } else {
            r.zero();
            dn.zero();
            d_out.zero();
            y.zero();
        }
    }
};

__device__ __forceinline__ float* partial_row(const NormArgs& a, uint32_t sum, uint32_t part) {
    return a.partials + (uint64_t(sum) * a.n_partials + part) * a.H;
}

template <typename Y, typename R>
__global__ __launch_bounds__(1024) void norm_grad_kernel(NormArgs a, uint32_t waves, uint32_t rows_per_wg) {
    __shared__ float s_a[16][3], s_b[16][2];
    const uint32_t per_row = waves * 64;
    const uint32_t mine = __builtin_amdgcn_readfirstlane(threadIdx.x / per_row);
    const uint32_t c = threadIdx.x % per_row * 8;
    const bool in = c < a.H;
    float w_pre[8] = {}, w_post[8] = {}, g[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] = 1.0f;
    if (in) {
        weight_at8(a, a.w_pre, c, w_pre);
        if (a.w_post) weight_at8(a, a.w_post, c, w_post);
        if (a.gate_channel) {
            Pack8<float> p;
            p.load(a.gate + c);
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = gate_value(a, p[j]);
        }
    }
    GradSums sums = {};
    const float inv_h = 1.0f / float(a.H);
    const uint32_t step = gridDim.x * rows_per_wg;
    GradRow<Y, R> next;
    next.load(a, blockIdx.x * rows_per_wg + mine, c, in && blockIdx.x * rows_per_wg + mine < a.T);
    for (uint32_t base = blockIdx.x * rows_per_wg; base < a.T; base += step) {      // the same count for the whole workgroup
        const uint32_t t = base + mine;
        const bool on = in && t < a.T;
        const GradRow<Y, R> row = next;
        if (base + step < a.T) next.load(a, t + step, c, in && t + step < a.T);
        float v[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[0] += row.r[j] * row.r[j];
            v[1] += row.dn[j] * w_pre[j] * row.r[j];
            v[2] += row.y[j] * row.y[j];
        }
        row_sums<3>(v, s_a, waves);
        const float rstd = rstd_of(a, v[0]), mean = v[1] * rstd * inv_h;
        float dr[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float h = row.r[j] * rstd;
            dr[j] = row.d_out[j] + rstd * (row.dn[j] * w_pre[j] - h * mean);
            sums.w_pre[j] += row.dn[j] * h;
        }
        if (on) store8_stream(static_cast<R*>(a.d_residual) + t * a.d_residual_stride + c, dr);
        if (a.y) {
            const float rstd_y = a.w_post ? rstd_of(a, v[2]) : 1.0f;
            const float token = a.gate_token ? a.gate[t < a.T ? t : 0] : 1.0f;
            const float g_token = a.gate_token ? gate_value(a, token) : 1.0f;
            const float scale = a.scale * g_token;
            float u[2] = {0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float h = row.y[j] * rstd_y, inner = a.w_post ? h * w_post[j] : h;
                u[0] += dr[j] * inner;
                u[1] += dr[j] * inner * g[j];
                sums.gate[j] += dr[j] * inner;
                sums.w_post[j] += scale * g[j] * dr[j] * h;
            }
            if (a.gate_token || a.w_post) row_sums<2>(u, s_b, waves);
            const float mean_y = a.w_post ? scale * u[1] * inv_h : 0.0f;        // mean(dy' w_post h)
            float dy[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                dy[j] = scale * g[j] * dr[j];
                if (a.w_post) dy[j] = rstd_y * (dy[j] * w_post[j] - row.y[j] * rstd_y * mean_y);
            }
            if (on) store8_stream(static_cast<Y*>(a.d_y) + t * a.d_y_stride + c, dy);
            if (a.gate_token && t < a.T && c == 0)
                a.d_gate[t] = a.scale * u[0] * (a.gate_sigmoid ? g_token * (1.0f - g_token) : 1.0f);
        }
        if (waves > 1) __syncthreads();                  // the next row writes s_a and s_b again
    }
    if (!in) return;
    const uint32_t part = blockIdx.x * rows_per_wg + mine;
    uint32_t n = 0;
    store8(partial_row(a, n++, part) + c, sums.w_pre);
    if (a.w_post) store8(partial_row(a, n++, part) + c, sums.w_post);
    if (a.gate_channel) store8(partial_row(a, n++, part) + c, sums.gate);
}

// Any width and alignment, as norm_any_kernel; the sums over the tokens are kept in the workgroup's partial rows.
template <typename Y, typename R>
__global__ __launch_bounds__(1024) void norm_grad_any_kernel(NormArgs a) {
    __shared__ float s_a[16][3], s_b[16][2];
    const uint32_t waves = blockDim.x / 64;
    const float inv_h = 1.0f / float(a.H);
    float* sum_pre = partial_row(a, 0, blockIdx.x);
    float* sum_post = partial_row(a, 1, blockIdx.x);
    float* sum_gate = partial_row(a, a.w_post ? 2 : 1, blockIdx.x);
    for (uint32_t c = threadIdx.x; c < a.H; c += blockDim.x) {
        sum_pre[c] = 0.0f;
        if (a.w_post) sum_post[c] = 0.0f;
        if (a.gate_channel) sum_gate[c] = 0.0f;
    }
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
        const float g_token = a.gate_token ? gate_value(a, a.gate[t]) : 1.0f, scale = a.scale * g_token;
        auto dr_at = [&](uint32_t c) {
            const float h = to_float(r[c]) * rstd;
            return (a.d_residual_out ? to_float(d_out[c]) : 0.0f) + rstd * (to_float(dn[c]) * weight_at(a, a.w_pre, c) - h * mean);
        };
        float u[2] = {0.0f, 0.0f};
        if (a.gate_token || a.w_post) {
            for (uint32_t c = threadIdx.x; c < a.H; c += blockDim.x) {
                const float inner = to_float(y[c]) * rstd_y * (a.w_post ? weight_at(a, a.w_post, c) : 1.0f);
                const float p = dr_at(c) * inner;
                u[0] += p;
                u[1] += p * (a.gate_channel ? gate_value(a, a.gate[c]) : 1.0f);
            }
            row_sums<2>(u, s_b, waves);
        }
        const float mean_y = a.w_post ? scale * u[1] * inv_h : 0.0f;
        for (uint32_t c = threadIdx.x; c < a.H; c += blockDim.x) {
            const float dr = dr_at(c);
            sum_pre[c] += to_float(dn[c]) * to_float(r[c]) * rstd;
            if (a.y) {
                const float h = to_float(y[c]) * rstd_y, w = a.w_post ? weight_at(a, a.w_post, c) : 1.0f;
                const float g = a.gate_channel ? gate_value(a, a.gate[c]) : 1.0f;
                float dy = scale * g * dr;
                if (a.w_post) {
                    sum_post[c] += dy * h;
                    dy = rstd_y * (dy * w - h * mean_y);
                }
                if (a.gate_channel) sum_gate[c] += dr * h * w;
                from_float(static_cast<Y*>(a.d_y) + t * a.d_y_stride + c, dy);
            }
            from_float(static_cast<R*>(a.d_residual) + t * a.d_residual_stride + c, dr);
        }
        if (a.gate_token && threadIdx.x == 0) a.d_gate[t] = a.scale * u[0] * (a.gate_sigmoid ? g_token * (1.0f - g_token) : 1.0f);
        __syncthreads();
    }
}

// A workgroup adds up 32 columns: 32 groups of threads take every 32nd partial sum, then their sums are added in order.
__global__ __launch_bounds__(256) void column_sum_kernel(NormArgs a) {
    __shared__ float s[32][33];
    const uint32_t c = blockIdx.x * 32, lane = threadIdx.x & 7, group = threadIdx.x >> 3;
    float v[4] = {};
    const uint32_t c4 = c + lane * 4;
    const bool whole = a.H % 4 == 0;
    if (c4 < a.H)
        for (uint32_t p = group; p < a.n_partials; p += 32) {
            const float* row = partial_row(a, blockIdx.y, p) + c4;
            if (whole) {
                const float4 q = *reinterpret_cast<const float4*>(row);
                v[0] += q.x; v[1] += q.y; v[2] += q.z; v[3] += q.w;
            } else {
                for (uint32_t j = 0; j < 4 && c4 + j < a.H; ++j) v[j] += row[j];
            }
        }
    for (int j = 0; j < 4; ++j) s[group][lane * 4 + j] = v[j];
    __syncthreads();
    if (threadIdx.x >= 32 || c + threadIdx.x >= a.H) return;
    float sum = 0.0f;
    for (int i = 0; i < 32; ++i) sum += s[i][threadIdx.x];
    const uint32_t col = c + threadIdx.x;
    if (blockIdx.y == 0) {
        a.d_w_pre[col] = sum;
    } else if (a.w_post && blockIdx.y == 1) {
        a.d_w_post[col] = sum;
    } else {
        const float g = a.gate_sigmoid ? sigmoid(a.gate[col]) : 0.0f;
        a.d_gate[col] = a.scale * sum * (a.gate_sigmoid ? g * (1.0f - g) : 1.0f);
    }
}

uint32_t any_threads(uint32_t H) { return H >= 1024 ? 1024 : (H + 63) / 64 * 64; }

// Workgroups of the gradient: 16 wavefronts to each of the 256 CUs, which is what 128 registers a lane leave room for.
uint32_t grad_workgroups(const RowShape& s, uint32_t T) {
    const uint32_t in_wg = s.waves * s.rows_per_wg, most = 256 * (in_wg >= 16 ? 1 : 16 / in_wg);
    const uint32_t need = (T + s.rows_per_wg - 1) / s.rows_per_wg;
    return need < most ? need : most;
}

template <typename Y, typename R>
hipError_t go(const NormArgs& a, bool vec, hipStream_t stream) {
    if (vec && a.H <= kRowColumns) {
        const RowShape s = row_shape(a.H);
        hipLaunchKernelGGL((norm_kernel<Y, R>), dim3((a.T + s.rows_per_wg - 1) / s.rows_per_wg), dim3(s.threads()), 0, stream, a, s.waves, s.rows_per_wg);
    } else {
        hipLaunchKernelGGL((norm_any_kernel<Y, R>), dim3(a.T), dim3(any_threads(a.H)), 0, stream, a);
    }
    return hipGetLastError();
}

template <typename Y, typename R>
hipError_t go_grad(NormArgs a, bool vec, hipStream_t stream) {
    if (a.T == 0) {
        a.n_partials = 0;
    } else if (vec && a.H <= kRowColumns) {
        const RowShape s = row_shape(a.H);
        const uint32_t wgs = grad_workgroups(s, a.T);
        a.n_partials = wgs * s.rows_per_wg;
        hipLaunchKernelGGL((norm_grad_kernel<Y, R>), dim3(wgs), dim3(s.threads()), 0, stream, a, s.waves, s.rows_per_wg);
    } else {
        a.n_partials = a.T < 256 ? a.T : 256;
        hipLaunchKernelGGL((norm_grad_any_kernel<Y, R>), dim3(a.n_partials), dim3(any_threads(a.H)), 0, stream, a);
    }
    const uint32_t n_sums = 1 + (a.w_post ? 1 : 0) + (a.gate_channel ? 1 : 0);
    hipLaunchKernelGGL(column_sum_kernel, dim3((a.H + 31) / 32, n_sums), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

uint32_t norm_grad_partials(uint32_t T, uint32_t H) {
    const RowShape s = row_shape(H);
    const uint32_t rows = grad_workgroups(s, T) * s.rows_per_wg, any = T < 256 ? T : 256;
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
