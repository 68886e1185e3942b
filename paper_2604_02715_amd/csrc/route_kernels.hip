// Router: the K best of E scores for each token, their gates, and the gradient of the gates.
//
// A row of logits lies in LPR lanes of eight neighbouring experts each (more than 512 experts: 16 to 64 to a lane), so that a
// wavefront holds 64 / LPR rows.  Scores are compared as integers whose order is that of the floats.  A round takes one
// expert: each lane knows its best, the lanes' largest is found in log2(LPR) steps, a ballot names the lowest lane that has
// it (its experts come before those of the others, so equal scores go to the lowest expert), and that lane alone takes the
// expert out and looks for its next best.
#include <cmath>

#include "block_device.h"
#include "block_ops.h"

namespace fluxmoe {
namespace {

constexpr uint32_t kThreads = 256;

// Larger floats have larger keys, -0 and +0 the same one; 0 is that of an expert never to be chosen (minus infinity, NaN).
__device__ __forceinline__ uint32_t order_key(float v) {
    v += 0.0f;
    const uint32_t b = __float_as_uint(v);
    const uint32_t k = b ^ (uint32_t(int32_t(b) >> 31) | 0x80000000u);
    return v > -INFINITY ? k : 0u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k); }

// e^(v - top) where top is the largest of the row; 1 at the top itself, also where that is infinite
__device__ __forceinline__ float softmax_term(float v, float top) { return v == top ? 1.0f : expf(v - top); }

// The lane's NV logits from expert `first` on; past the row's end `pad`.
template <typename L, int NV>
__device__ __forceinline__ void load_logits(const L* row, uint32_t first, uint32_t E, bool vec, float pad, float (&l)[NV]) {
#pragma unroll
    for (int c = 0; c < NV; c += 8) {
        if (vec && first + c + 8 <= E) {
            Pack8<L> p;
            p.load(row + first + c);
#pragma unroll
            for (int j = 0; j < 8; ++j) l[c + j] = p[j];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) l[c + j] = first + c + j < E ? to_float(row[first + c + j]) : pad;
        }
    }
}

template <int NV>
__device__ __forceinline__ void lane_best(const uint32_t (&key)[NV], uint32_t& best, uint32_t& at) {
    best = key[0];
    at = 0;
#pragma unroll
    for (int j = 1; j < NV; ++j)
        if (key[j] > best) { best = key[j]; at = j; }
}

template <typename L, int LPR, int NV, bool SIGMOID>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a) {
    __shared__ int32_t s_id[kThreads];           // a row's K results lie at its first lane's number and behind it (K <= LPR)
    __shared__ uint32_t s_key[kThreads];
    const uint32_t tid = threadIdx.x, sub = tid & (LPR - 1), base = tid - sub;
    const uint32_t row = blockIdx.x * (kThreads / LPR) + tid / LPR;
    const bool valid = row < a.T;
    const uint32_t first = sub * NV;
    const L* logits = static_cast<const L*>(a.logits) + uint64_t(valid ? row : 0) * a.row_stride;

    uint32_t key[NV];
    {
        float l[NV];
        load_logits<L, NV>(logits, first, valid ? a.E : 0, a.vec != 0, -INFINITY, l);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float v = l[j];
            if constexpr (SIGMOID) {
                const float s = sigmoid(v) + (a.bias && first + j < a.E ? a.bias[first + j] : 0.0f);
                v = v > -INFINITY ? s : -INFINITY;
            }
            key[j] = order_key(v);
        }
    }
    s_id[tid] = -1;
    s_key[tid] = 0;
    wave_fence();

    uint32_t best, at;
    lane_best<NV>(key, best, at);
    float total = 0.0f;
    for (uint32_t k = 0; k < a.K; ++k) {
        const uint32_t most = group_max<LPR>(best);
        if (!SIGMOID && k == 0 && !a.renormalize) {      // the whole row's softmax
            const float top = key_value(most);
#pragma unroll
            for (int j = 0; j < NV; ++j) total += key[j] ? softmax_term(key_value(key[j]), top) : 0.0f;
            total = group_sum<LPR>(total);
        }
        const uint64_t have = __ballot(best == most && most != 0);
        const uint64_t mine = LPR == 64 ? have : (have >> (tid & 63 & ~(LPR - 1))) & ((1ull << (LPR & 63)) - 1);
        if (mine && sub == uint32_t(__builtin_ctzll(mine))) {
            s_id[base + k] = int32_t(first + at);
            s_key[base + k] = most;
#pragma unroll
            for (int j = 0; j < NV; ++j) key[j] = uint32_t(j) == at ? 0u : key[j];
            lane_best<NV>(key, best, at);
        }
    }
    wave_fence();

    const int32_t id = s_id[tid];
    const bool chosen = sub < a.K && id >= 0;
    float p = 0.0f;
    if (chosen) {
        if constexpr (SIGMOID) p = sigmoid(to_float(logits[id]));
        else p = softmax_term(key_value(s_key[tid]), key_value(s_key[base]));
    }
    if (a.renormalize) {
        total = group_sum<LPR>(p);
        if (total == 0.0f) total = 1.0f;                 // nothing to choose from, or sigmoids below the smallest float
    }
    if (SIGMOID && !a.renormalize) total = 1.0f;
    if (valid && sub < a.K) {
        a.ids[uint64_t(row) * a.K + sub] = id;
        a.gates[uint64_t(row) * a.K + sub] = chosen ? p / total * a.scale : 0.0f;
    }
}

// With c the chosen scores (a softmax's numerators: its sum cancels where the gates are divided by theirs), C their sum and
// d = scale * d_gates:
//   renormalised:  d_c = (d - sum(d c) / C) / C, then times c (softmax) or c (1 - c) (sigmoid)
//   sigmoid:       d c (1 - c)
//   softmax:       p_i (d_i - sum_j d_j p_j) for every expert i of the row, chosen or not
// The K values of a row are spread over its experts in LDS; every lane then writes its experts.
template <typename L, int LPR, int NV, bool SIGMOID>
__global__ __launch_bounds__(kThreads) void route_grad_kernel(RouteArgs a) {
    __shared__ __align__(16) float s_row[kThreads * NV];  // LPR * NV >= E places for a row
    const uint32_t tid = threadIdx.x, sub = tid & (LPR - 1), base = tid - sub;
    const uint32_t row = blockIdx.x * (kThreads / LPR) + tid / LPR;
    const bool valid = row < a.T;
    const uint32_t first = sub * NV;
    const L* logits = static_cast<const L*>(a.logits) + uint64_t(valid ? row : 0) * a.row_stride;
    const bool dense = !SIGMOID && !a.renormalize;

    int32_t id = -1;
    float d = 0.0f;
    if (valid && sub < a.K) {
        id = a.ids[uint64_t(row) * a.K + sub];
        d = a.d_gates[uint64_t(row) * a.K + sub] * a.scale;
    }
    const bool chosen = uint32_t(id) < a.E;
    const float l_chosen = chosen ? to_float(logits[id]) : -INFINITY;
#pragma unroll
    for (int j = 0; j < NV; j += 4) *reinterpret_cast<float4*>(&s_row[tid * NV + j]) = make_float4(0, 0, 0, 0);
    wave_fence();

    float out[NV];
    if (dense) {
        float l[NV], top = -INFINITY, total = 0.0f;
        load_logits<L, NV>(logits, first, valid ? a.E : 0, a.vec != 0, -INFINITY, l);
#pragma unroll
        for (int j = 0; j < NV; ++j) top = fmaxf(top, l[j]);
        top = group_max<LPR>(top);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            l[j] = l[j] > -INFINITY ? softmax_term(l[j], top) : 0.0f;
            total += l[j];
        }
        total = group_sum<LPR>(total);
        const float inv = total > 0.0f ? 1.0f / total : 0.0f;
        const float p_chosen = chosen && l_chosen > -INFINITY ? softmax_term(l_chosen, top) * inv : 0.0f;
        const float mean = group_sum<LPR>(chosen ? d * p_chosen : 0.0f);
        if (chosen) s_row[base * NV + id] = d;
        wave_fence();
#pragma unroll
        for (int j = 0; j < NV; ++j) out[j] = l[j] * inv * (s_row[tid * NV + j] - mean);
    } else {
        float c = 0.0f, slope;
        if constexpr (SIGMOID) {
            const float e = expf(-l_chosen);
            c = chosen ? 1.0f / (1.0f + e) : 0.0f;
            slope = l_chosen > 0.0f ? c * (e * c) : c * (1.0f - c);     // 1 - c without its cancellation near 1
        } else {
            const float top = group_max<LPR>(l_chosen);
            c = chosen && l_chosen > -INFINITY ? softmax_term(l_chosen, top) : 0.0f;
            slope = c;
        }
        if (a.renormalize) {
            float total = group_sum<LPR>(c);
            if (total == 0.0f) total = 1.0f;
            const float mean = group_sum<LPR>(chosen ? d * (c / total) : 0.0f);
            d = (d - mean) / total;
        }
        if (chosen) s_row[base * NV + id] = d * slope;
        wave_fence();
#pragma unroll
        for (int j = 0; j < NV; ++j) out[j] = s_row[tid * NV + j];
    }
    if (!valid) return;
    L* dst = static_cast<L*>(a.d_logits) + uint64_t(row) * a.d_stride;
#pragma unroll
    for (int c = 0; c < NV; c += 8) {
        if (a.d_vec && first + c + 8 <= a.E) {
            const float o[8] = {out[c], out[c + 1], out[c + 2], out[c + 3], out[c + 4], out[c + 5], out[c + 6], out[c + 7]};
            store8(dst + first + c, o);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (first + c + j < a.E) from_float(dst + first + c + j, out[c + j]);
        }
    }
}

template <typename L, bool SIGMOID, int LPR, int NV>
hipError_t go(const RouteArgs& a, bool grad, hipStream_t stream) {
    const uint32_t rows = kThreads / LPR, grid = (a.T + rows - 1) / rows;
    if (grad) hipLaunchKernelGGL((route_grad_kernel<L, LPR, NV, SIGMOID>), dim3(grid), dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((route_kernel<L, LPR, NV, SIGMOID>), dim3(grid), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

// As few lanes to a row as hold its experts at eight each, and one for every chosen expert.
template <typename L, bool SIGMOID>
hipError_t pick(const RouteArgs& a, bool grad, hipStream_t stream) {
    if (a.E <= 16 && a.K <= 2) return go<L, SIGMOID, 2, 8>(a, grad, stream);
    if (a.E <= 64 && a.K <= 8) return go<L, SIGMOID, 8, 8>(a, grad, stream);
    if (a.E <= 256 && a.K <= 32) return go<L, SIGMOID, 32, 8>(a, grad, stream);
    if (a.E <= 512) return go<L, SIGMOID, 64, 8>(a, grad, stream);
    if (a.E <= 1024) return go<L, SIGMOID, 64, 16>(a, grad, stream);
    if (a.E <= 2048) return go<L, SIGMOID, 64, 32>(a, grad, stream);
    return go<L, SIGMOID, 64, 64>(a, grad, stream);
}

hipError_t launch(const RouteArgs& a, bool f32, bool sigmoid, bool grad, hipStream_t stream) {
    if (f32) return sigmoid ? pick<float, true>(a, grad, stream) : pick<float, false>(a, grad, stream);
    return sigmoid ? pick<bf16_t, true>(a, grad, stream) : pick<bf16_t, false>(a, grad, stream);
}

}  // namespace

hipError_t launch_route(const RouteArgs& a, bool f32, bool sigmoid, hipStream_t stream) { return launch(a, f32, sigmoid, false, stream); }
hipError_t launch_route_grad(const RouteArgs& a, bool f32, bool sigmoid, hipStream_t stream) { return launch(a, f32, sigmoid, true, stream); }

}  // namespace fluxmoe
