// Router: the K best of E scores for each token, their gates, and the gradient of the gates.
//
// A row of logits lies in LPR lanes of eight neighbouring experts each (more than 512 experts: 16 to 64 to a lane), so that a
// wavefront holds 64 / LPR rows.  Scores are compared as integers whose order is that of the floats.  A round takes one
// expert: each lane knows its best, the lanes' largest is found in log2(LPR) steps, a ballot names the lowest lane that has
// it (its experts come before those of the others, so equal scores go to the lowest expert), and that lane alone takes the
// expert out and looks for its next best.
// The K rounds follow each other: bound by their length (1 x 512 top-10 4 us, the launch's 2.1 included; 16381 x 160 by sigmoids
// 8.6 us in route_many_kernel, which takes 7 from 2048 rows on, for bytes of 1), and by instructions beyond that, where there are more rows
// than the CUs hold at once (32768 x 160 11.9).  The gradient is bound by memory (8192 x 512 FP32, every logit, 7.9 us; bytes 5.2).
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

__device__ __forceinline__ void load8(const bf16_t* p, float* f) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = __uint_as_float((j & 1) ? (w[j / 2] & 0xFFFF0000u) : (w[j / 2] << 16));
}
__device__ __forceinline__ void load8(const float* p, float* f) {
#pragma unroll
    for (int j = 0; j < 8; j += 4) {
        const float4 v = *reinterpret_cast<const float4*>(p + j);
        f[j] = v.x;
        f[j + 1] = v.y;
        f[j + 2] = v.z;
        f[j + 3] = v.w;
    }
}
// past the caches (16384 x 512 FP32 gradients 11.6 us, through them 15.8)
__device__ __forceinline__ void store8(bf16_t* p, const float* f) {
    store_stream16(p, make_uint4(pack_bf16_rne(f[0], f[1]), pack_bf16_rne(f[2], f[3]), pack_bf16_rne(f[4], f[5]), pack_bf16_rne(f[6], f[7])));
}
__device__ __forceinline__ void store8(float* p, const float* f) {
    store_stream16(p, make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])));
    store_stream16(p + 4, make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])));
}

// Eight logits from expert `first` on; minus infinity past the row's end.
template <typename L>
__device__ __forceinline__ void load_logits(const L* row, uint32_t first, uint32_t E, bool vec, float* l) {
    if (vec && first + 8 <= E) {
        load8(row + first, l);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) l[j] = first + j < E ? to_float(row[first + j]) : -INFINITY;
    }
}

// Keys of eight experts from `first` on.
template <bool SIGMOID>
__device__ __forceinline__ void keys_of(const RouteArgs& a, uint32_t first, const float* l, uint32_t* key) {
    if constexpr (SIGMOID) {
        Pack<float, 8> bias;                             // 0 where there is none
        bias.template load<kCached>(row_at(a.bias, 0, 0, a.bias ? a.E : 0), first);
        float v[8], score[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = l[j] > -INFINITY ? l[j] : 0.0f;
        sigmoid8(v, score);
#pragma unroll
        for (int j = 0; j < 8; ++j) key[j] = l[j] > -INFINITY ? order_key(score[j] + bias[j]) : 0u;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) key[j] = order_key(l[j]);
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

// Takes the experts of the groups that are not kept out of a row's keys.  Each of a row's groups belongs to as many lanes as there are
// for it (a power of two); they share its keys out, and the two largest of each part meet in the steps of a reduction.  A group is kept
// if fewer than top_groups groups come before it, which every lane counts for its own.  s_row: the row's keys, one word apart after
// each group so that lanes of different groups read different banks; s_group: its groups' scores.
template <int LPR, int NV>
__device__ __forceinline__ void keep_groups(const RouteArgs& a, uint32_t sub, uint32_t (&key)[NV], uint32_t* s_row, uint32_t* s_group) {
    const uint32_t size = a.E / a.groups, first = sub * NV;
    uint32_t g = first / size, at = first - g * size;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (first + j < a.E) s_row[first + j + g] = key[j];
        if (++at == size) { at = 0; ++g; }
    }
    wave_fence();
    uint32_t lanes = LPR;                                // to a group
    while (lanes * a.groups > LPR) lanes /= 2;
    const uint32_t group = sub / lanes;
    uint32_t one = 0, two = 0;
    if (group < a.groups)
        for (uint32_t i = sub & (lanes - 1); i < size; i += lanes) {
            const uint32_t k = s_row[group * (size + 1) + i];
            two = max(two, min(one, k));
            one = max(one, k);
        }
    for (uint32_t d = 1; d < lanes; d *= 2) {
        const uint32_t o = __shfl_xor(one, d), t = __shfl_xor(two, d);
        two = max(max(two, t), min(one, o));
        one = max(one, o);
    }
    // the sum is rounded as written; a score that sank to minus infinity is still one
    const uint32_t score = a.group_top2 && two ? max(order_key(key_value(one) + key_value(two)), 1u) : one;
    if (group < a.groups && (sub & (lanes - 1)) == 0) s_group[group] = score;
    wave_fence();
    uint32_t ahead = 0;
    for (uint32_t o = 0; o < a.groups; ++o) {
        const uint32_t k = s_group[o];
        ahead += k > score || (k == score && o < group);
    }
    const uint64_t kept = __ballot(group < a.groups && score != 0 && ahead < a.top_groups) >> (threadIdx.x & 63 & ~(LPR - 1));
    g = first / size;
    at = first - g * size;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (g >= a.groups || !((kept >> (g * lanes)) & 1)) key[j] = 0;
        if (++at == size) { at = 0; ++g; }
    }
}

template <typename L, int LPR, int NV, bool SIGMOID, bool GROUPED>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a) {
    __shared__ uint32_t s_keys[GROUPED ? kThreads / LPR : 1][GROUPED ? LPR * NV + kRouteMaxGroups : 1];
    __shared__ uint32_t s_groups[GROUPED ? kThreads / LPR : 1][GROUPED ? kRouteMaxGroups : 1];
    __shared__ int32_t s_id[kThreads];           // a row's K results lie at its first lane's number and behind it (K <= LPR)
    __shared__ uint32_t s_key[kThreads];
    const uint32_t tid = threadIdx.x, sub = tid & (LPR - 1), base = tid - sub;
    const uint32_t row = blockIdx.x * (kThreads / LPR) + tid / LPR;
    const bool valid = row < a.T;
    const uint32_t first = sub * NV;
    const L* logits = static_cast<const L*>(a.logits) + uint64_t(valid ? row : 0) * a.row_stride;

    uint32_t key[NV];
#pragma unroll
    for (int c = 0; c < NV; c += 8) {
        float l[8];
        load_logits(logits, first + c, valid ? a.E : 0, a.vec != 0, l);
        keys_of<SIGMOID>(a, first + c, l, &key[c]);
    }
    s_id[tid] = -1;
    s_key[tid] = 0;
    wave_fence();

    uint32_t best, at, top_key = 0;
    lane_best<NV>(key, best, at);
    float total = 0.0f;
    if constexpr (GROUPED) {
        if (!SIGMOID && !a.renormalize) {                // the whole row's softmax, whichever groups are kept
            top_key = group_max<LPR>(best);
            const float top = key_value(top_key);
#pragma unroll
            for (int j = 0; j < NV; ++j) total += key[j] ? softmax_term(key_value(key[j]), top) : 0.0f;
            total = group_sum<LPR>(total);
        }
        keep_groups<LPR, NV>(a, sub, key, s_keys[tid / LPR], s_groups[tid / LPR]);
        lane_best<NV>(key, best, at);
    }
    for (uint32_t k = 0; k < a.K; ++k) {
        const uint32_t most = group_max<LPR>(best);
        if (!GROUPED && !SIGMOID && k == 0 && !a.renormalize) {      // the whole row's softmax
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
        else p = softmax_term(key_value(s_key[tid]), key_value(GROUPED && !a.renormalize ? top_key : s_key[base]));
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

// The same for many rows, with fewer lanes to a row and so fewer instructions in all, if in longer rounds: 8 or 16 lanes, up to four
// chunks of eight experts to each.  The keys lie in LDS (each lane's own), the chunks' largest ones in registers; when a lane's best is
// taken, only that chunk is read again.  Of equal keys the largest complement of an expert's number wins.
template <typename L, int LPR, int CHUNKS, bool SIGMOID>
__global__ __launch_bounds__(kThreads) void route_many_kernel(RouteArgs a) {
    __shared__ uint4 s_key[CHUNKS][2][kThreads];
    const uint32_t tid = threadIdx.x, sub = tid & (LPR - 1);
    const uint32_t row = blockIdx.x * (kThreads / LPR) + tid / LPR;
    const bool valid = row < a.T;
    const L* logits = static_cast<const L*>(a.logits) + uint64_t(valid ? row : 0) * a.row_stride;
    auto first_of = [&](uint32_t ch) { return (ch * LPR + sub) * 8; };

    uint32_t key[CHUNKS][8];
#pragma unroll
    for (int ch = 0; ch < CHUNKS; ++ch) {
        float l[8];
        load_logits(logits, first_of(ch), valid ? a.E : 0, a.vec != 0, l);
        keys_of<SIGMOID>(a, first_of(ch), l, key[ch]);
        s_key[ch][0][tid] = make_uint4(key[ch][0], key[ch][1], key[ch][2], key[ch][3]);
        s_key[ch][1][tid] = make_uint4(key[ch][4], key[ch][5], key[ch][6], key[ch][7]);
    }
    uint32_t most[CHUNKS], rank[CHUNKS], best, best_rank;        // rank: the complement of the expert
    auto best_of_lane = [&]() {
        best = most[0];
        best_rank = rank[0];
#pragma unroll
        for (int ch = 1; ch < CHUNKS; ++ch)
            if (most[ch] > best) { best = most[ch]; best_rank = rank[ch]; }
    };
#pragma unroll
    for (int ch = 0; ch < CHUNKS; ++ch) {
        uint32_t at;
        lane_best<8>(key[ch], most[ch], at);
        rank[ch] = ~(first_of(ch) + at);
    }
    best_of_lane();
    float total = 0.0f;
    if (!SIGMOID && !a.renormalize) {                            // the whole row's softmax
        const float top = key_value(group_max<LPR>(best));
#pragma unroll
        for (int ch = 0; ch < CHUNKS; ++ch)
#pragma unroll
            for (int j = 0; j < 8; ++j) total += key[ch][j] ? softmax_term(key_value(key[ch][j]), top) : 0.0f;
        total = group_sum<LPR>(total);
    }
    uint32_t top_key = 0, got_key[2] = {0, 0};
    int32_t got_id[2] = {-1, -1};                                // lane i keeps the i-th and the LPR + i-th choice
    for (uint32_t k = 0; k < a.K; ++k) {
        const uint32_t won = group_max<LPR>(best);
        const uint32_t won_rank = group_max<LPR>(best == won ? best_rank : 0u);
        if (k == 0) top_key = won;
        const bool keep = sub == (k & (LPR - 1)) && won != 0;
        const uint32_t id = ~won_rank;
        if (k < LPR) {
            if (keep) { got_id[0] = int32_t(id); got_key[0] = won; }
        } else {
            if (keep) { got_id[1] = int32_t(id); got_key[1] = won; }
        }
        if (best_rank == won_rank && won != 0) {                 // this lane's best was taken
            const uint32_t ch = id / (8 * LPR), j = id & 7;
            reinterpret_cast<uint32_t*>(&s_key[ch][j >> 2][tid])[j & 3] = 0;
            const uint4 lo = s_key[ch][0][tid], hi = s_key[ch][1][tid];
            const uint32_t left[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            uint32_t m, at;
            lane_best<8>(left, m, at);
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
                if (uint32_t(c) == ch) { most[c] = m; rank[c] = ~(first_of(c) + at); }
            best_of_lane();
        }
    }
    float p[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (got_id[i] >= 0) {
            if constexpr (SIGMOID) p[i] = sigmoid(to_float(logits[got_id[i]]));
            else p[i] = softmax_term(key_value(got_key[i]), key_value(top_key));
        }
    if (a.renormalize) {
        total = group_sum<LPR>(p[0] + p[1]);
        if (total == 0.0f) total = 1.0f;
    }
    if (SIGMOID && !a.renormalize) total = 1.0f;
    if (!valid) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t k = sub + i * LPR;
        if (k >= a.K) break;
        a.ids[uint64_t(row) * a.K + k] = got_id[i];
        a.gates[uint64_t(row) * a.K + k] = got_id[i] >= 0 ? p[i] / total * a.scale : 0.0f;
    }
}

// With c the chosen scores (a softmax's numerators: its sum cancels where the gates are divided by theirs), C their sum and
// d = scale * d_gates:
//   renormalised:  (d - sum(d c) / C) times c / C (softmax) or c (1 - c) / C (sigmoid)
//   sigmoid:       d c (1 - c)
//   softmax:       p_i (d_i - sum_j d_j p_j) for every expert i of the row, chosen or not
// The K values of a row are spread over its experts in LDS; the lanes then write the row, eight experts at a time.
template <typename L, int LPR, int CHUNKS, bool SIGMOID>
__global__ __launch_bounds__(kThreads) void route_grad_kernel(RouteArgs a) {
    __shared__ __align__(16) float s_row[kThreads / LPR][LPR * CHUNKS * 8];
    const uint32_t tid = threadIdx.x, sub = tid & (LPR - 1);
    const uint32_t row = blockIdx.x * (kThreads / LPR) + tid / LPR;
    const bool valid = row < a.T;
    const L* logits = static_cast<const L*>(a.logits) + uint64_t(valid ? row : 0) * a.row_stride;
    const bool dense = !SIGMOID && !a.renormalize;
    float* spread = s_row[tid / LPR];
    auto first_of = [&](uint32_t ch) { return (ch * LPR + sub) * 8; };

    int32_t id = -1;
    float d = 0.0f;
    if (valid && sub < a.K) {
        id = a.ids[uint64_t(row) * a.K + sub];
        d = a.d_gates[uint64_t(row) * a.K + sub] * a.scale;
    }
    const bool chosen = uint32_t(id) < a.E;
    const float l_chosen = chosen ? to_float(logits[id]) : -INFINITY;
#pragma unroll
    for (int ch = 0; ch < CHUNKS; ++ch) {
        float4* p = reinterpret_cast<float4*>(spread + first_of(ch));
        p[0] = p[1] = make_float4(0, 0, 0, 0);
    }
    wave_fence();

    float l[CHUNKS][8], inv = 0.0f, mean = 0.0f;
    if (dense) {
        float top = -INFINITY, total = 0.0f;
#pragma unroll
        for (int ch = 0; ch < CHUNKS; ++ch) {
            load_logits(logits, first_of(ch), valid ? a.E : 0, a.vec != 0, l[ch]);
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, l[ch][j]);
        }
        top = group_max<LPR>(top);
#pragma unroll
        for (int ch = 0; ch < CHUNKS; ++ch)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                l[ch][j] = l[ch][j] > -INFINITY ? softmax_term(l[ch][j], top) : 0.0f;
                total += l[ch][j];
            }
        total = group_sum<LPR>(total);
        inv = total > 0.0f ? 1.0f / total : 0.0f;
        const float p_chosen = chosen && l_chosen > -INFINITY ? softmax_term(l_chosen, top) * inv : 0.0f;
        mean = group_sum<LPR>(chosen ? d * p_chosen : 0.0f);
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
            mean = group_sum<LPR>(chosen ? d * (c / total) : 0.0f);
            d -= mean;
            slope /= total;                              // at most 1, where 1 / total of sigmoids below the normal numbers is infinite
        }
        d *= slope;
    }
    if (chosen) spread[id] = d;
    wave_fence();
    if (!valid) return;
    L* dst = static_cast<L*>(a.d_logits) + uint64_t(row) * a.d_stride;
#pragma unroll
    for (int ch = 0; ch < CHUNKS; ++ch) {
        const uint32_t e = first_of(ch);
        float out[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            out[j] = spread[e + j];
            if (dense) out[j] = l[ch][j] * inv * (out[j] - mean);
        }
        if (a.d_vec && e + 8 <= a.E) {
            store8(dst + e, out);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (e + j < a.E) from_float(dst + e + j, out[j]);
        }
    }
}

uint32_t workgroups(const RouteArgs& a, uint32_t lanes) {
    const uint32_t rows = kThreads / lanes;
    return (a.T + rows - 1) / rows;
}
template <typename L, bool SIGMOID, int LPR, int NV, bool GROUPED = false>
void go(const RouteArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL((route_kernel<L, LPR, NV, SIGMOID, GROUPED>), dim3(workgroups(a, LPR)), dim3(kThreads), 0, stream, a);
}
template <typename L, bool SIGMOID, int LPR, int CHUNKS>
void go_many(const RouteArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL((route_many_kernel<L, LPR, CHUNKS, SIGMOID>), dim3(workgroups(a, LPR)), dim3(kThreads), 0, stream, a);
}
template <typename L, bool SIGMOID, int LPR, int CHUNKS>
void go_grad(const RouteArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL((route_grad_kernel<L, LPR, CHUNKS, SIGMOID>), dim3(workgroups(a, LPR)), dim3(kThreads), 0, stream, a);
}

// The rows beyond which route_many_kernel is the faster one.  Its rounds are longer, but its wavefronts hold several times as many rows,
// so that it goes on at a chain's length (160 experts, top-8 by sigmoids: 6.9 us from 2048 to 8192 rows, 7.8 at 16384) where
// route_kernel takes longer with the rows (4.5 at 2048, 6.4 at 6144, 7.6 at 6145, 12.2 at 16384).  Its time over route_kernel's, top-8 by
// sigmoids (BF16) / by softmax (FP32); 16 choices cross earlier, two later:
//   experts  4097 rows    6144         6145         8192         8193         12288
//       128  0.95 / 1.03  0.91 / 0.95  0.81 / 0.86  0.77 / 0.82  0.75 / 0.77  0.64 / 0.66
//       160  1.13 / 1.22  1.07 / 1.13  0.94 / 1.04  0.90 / 0.98  0.91 / 0.92  0.77 / 0.77
//       193  1.45 / 1.35  1.35 / 1.24  1.19 / 1.16  1.11 / 1.10  1.10 / 1.06  0.93 / 1.05
//       256  1.33 / 1.33  1.22 / 1.27  1.10 / 1.14  1.03 / 1.09  1.09 / 1.01  0.90 / 0.84
//       384  1.07 / 1.00  0.88 / 0.84  0.85 / 0.79  0.73 / 0.70  0.87 / 0.75  0.68 / 0.62
//       512  1.10 / 1.02  0.92 / 0.84  0.87 / 0.81  0.76 / 0.70  0.91 / 0.77  0.70 / 0.63
//   160, 16  1.01         0.96         0.84         0.80         0.81         0.68
//   256, 16  1.18         1.11         0.97         0.92         0.96         0.79
//   160, 2   1.21         1.12         1.11         1.03         1.05         0.90
//   256, 2   1.42         1.27         1.28         1.14         1.22         0.99
// Up to 128 experts and from 257 on they are level about 4096 rows.
uint32_t many_rows(uint32_t E) { return E <= 128 || E > 256 ? 4096 : E <= 192 ? 6144 : 8192; }

// The same with a lane for every group, too.
template <typename L, bool SIGMOID>
void pick_grouped(const RouteArgs& a, hipStream_t stream) {
    if (a.E <= 64 && a.K <= 8 && a.groups <= 8) go<L, SIGMOID, 8, 8, true>(a, stream);
    else if (a.E <= 256 && a.K <= 32 && a.groups <= 32) go<L, SIGMOID, 32, 8, true>(a, stream);
    else if (a.E <= 512) go<L, SIGMOID, 64, 8, true>(a, stream);
    else if (a.E <= 1024) go<L, SIGMOID, 64, 16, true>(a, stream);
    else if (a.E <= 2048) go<L, SIGMOID, 64, 32, true>(a, stream);
    else go<L, SIGMOID, 64, 64, true>(a, stream);
}

// As few lanes to a row as hold its experts at eight each, and one for every chosen expert.
template <typename L, bool SIGMOID>
void pick(const RouteArgs& a, hipStream_t stream) {
    if (a.T > many_rows(a.E) && a.E > 64 && a.E <= 512 && a.K <= 16) {
        if (a.E <= 128) go_many<L, SIGMOID, 8, 2>(a, stream);
        else if (a.E <= 192) go_many<L, SIGMOID, 8, 3>(a, stream);
        else if (a.E <= 256) go_many<L, SIGMOID, 8, 4>(a, stream);
        else go_many<L, SIGMOID, 16, 4>(a, stream);
        return;
    }
    if (a.E <= 16 && a.K <= 2) go<L, SIGMOID, 2, 8>(a, stream);
    else if (a.E <= 64 && a.K <= 8) go<L, SIGMOID, 8, 8>(a, stream);
    else if (a.E <= 256 && a.K <= 32) go<L, SIGMOID, 32, 8>(a, stream);
    else if (a.E <= 512) go<L, SIGMOID, 64, 8>(a, stream);
    else if (a.E <= 1024) go<L, SIGMOID, 64, 16>(a, stream);
    else if (a.E <= 2048) go<L, SIGMOID, 64, 32>(a, stream);
    else go<L, SIGMOID, 64, 64>(a, stream);
}

template <typename L, bool SIGMOID>
void pick_grad(const RouteArgs& a, hipStream_t stream) {
    if (a.E <= 16 && a.K <= 2) go_grad<L, SIGMOID, 2, 1>(a, stream);
    else if (a.E <= 64 && a.K <= 8) go_grad<L, SIGMOID, 8, 1>(a, stream);
    else if (a.E <= 256 && a.K <= 32) go_grad<L, SIGMOID, 32, 1>(a, stream);
    else if (a.E <= 512) go_grad<L, SIGMOID, 64, 1>(a, stream);
    else if (a.E <= 1024) go_grad<L, SIGMOID, 64, 2>(a, stream);
    else if (a.E <= 2048) go_grad<L, SIGMOID, 64, 4>(a, stream);
    else go_grad<L, SIGMOID, 64, 8>(a, stream);
}

template <typename L, bool SIGMOID>
hipError_t pick(const RouteArgs& a, bool grad, hipStream_t stream) {
    if (grad) pick_grad<L, SIGMOID>(a, stream);
    else if (a.groups > 1) pick_grouped<L, SIGMOID>(a, stream);
    else pick<L, SIGMOID>(a, stream);
    return hipGetLastError();
}

hipError_t launch(const RouteArgs& a, bool f32, bool sigmoid, bool grad, hipStream_t stream) {
    if (f32) return sigmoid ? pick<float, true>(a, grad, stream) : pick<float, false>(a, grad, stream);
    return sigmoid ? pick<bf16_t, true>(a, grad, stream) : pick<bf16_t, false>(a, grad, stream);
}

}  // namespace

hipError_t launch_route(const RouteArgs& a, bool f32, bool sigmoid, hipStream_t stream) { return launch(a, f32, sigmoid, false, stream); }
hipError_t launch_route_grad(const RouteArgs& a, bool f32, bool sigmoid, hipStream_t stream) { return launch(a, f32, sigmoid, true, stream); }

}  // namespace fluxmoe
