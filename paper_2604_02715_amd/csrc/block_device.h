// Device code shared by the operators around the routed experts.
#pragma once

#include <hip/hip_runtime.h>

#include "decode_args.h"
#include "ffn_device.h"

namespace fluxmoe {

// ---------------------------------------------------------------- reductions over neighbouring lanes
// The other half's value for halves of 1, 2, 4 or 8 lanes (the mirrored forms serve where all lanes of a half already
// hold the same value).
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
    return uint32_t(__builtin_amdgcn_update_dpp(0, int(v), CTRL, 0xF, 0xF, false));
}
constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E, kDppHalfMirror = 0x141, kDppMirror = 0x140;

// op over the LANES lanes of each aligned group (a power of two); every lane gets the result.  The order of the operands is
// fixed, so a sum has the same bits every time.
template <int LANES, typename T, typename Op>
__device__ __forceinline__ T group_reduce(T v, Op op) {
    static_assert(sizeof(T) == 4, "32-bit values");
    auto with = [&](uint32_t o) { v = op(v, __builtin_bit_cast(T, o)); };
    if constexpr (LANES >= 2) with(dpp<kDppXor1>(__builtin_bit_cast(uint32_t, v)));
    if constexpr (LANES >= 4) with(dpp<kDppXor2>(__builtin_bit_cast(uint32_t, v)));
    if constexpr (LANES >= 8) with(dpp<kDppHalfMirror>(__builtin_bit_cast(uint32_t, v)));
    if constexpr (LANES >= 16) with(dpp<kDppMirror>(__builtin_bit_cast(uint32_t, v)));
    if constexpr (LANES >= 32) {
        const uint32_t b = __builtin_bit_cast(uint32_t, v);
        const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
        v = op(__builtin_bit_cast(T, uint32_t(r[0])), __builtin_bit_cast(T, uint32_t(r[1])));
    }
    if constexpr (LANES >= 64) {
        const uint32_t b = __builtin_bit_cast(uint32_t, v);
        const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
        v = op(__builtin_bit_cast(T, uint32_t(r[0])), __builtin_bit_cast(T, uint32_t(r[1])));
    }
    return v;
}
template <int LANES>
__device__ __forceinline__ float group_sum(float v) {
    return group_reduce<LANES>(v, [](float a, float b) { return a + b; });
}
template <int LANES>
__device__ __forceinline__ float group_max(float v) {
    return group_reduce<LANES>(v, [](float a, float b) { return fmaxf(a, b); });
}
template <int LANES>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
    return group_reduce<LANES>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

// What other lanes of the wavefront wrote to LDS before is read behind it.
__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// ---------------------------------------------------------------- BF16 and FP32 elements
struct bf16_t { uint16_t bits; };

__device__ __forceinline__ float to_float(bf16_t v) { return __uint_as_float(uint32_t(v.bits) << 16); }
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ void from_float(bf16_t* p, float v) { p->bits = uint16_t(pack_bf16_rne(v, v)); }
__device__ __forceinline__ void from_float(float* p, float v) { *p = v; }

// Eight consecutive elements in registers, as loaded: 16 bytes of BF16, 32 of FP32.
template <typename T>
struct Pack8;
template <>
struct Pack8<bf16_t> {
    uint4 v;
    __device__ __forceinline__ void load(const bf16_t* p) { v = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void load_stream(const bf16_t* p) { v = load_stream16(p); }
    __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ float operator[](int i) const {
        const uint32_t w = i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w;
        return __uint_as_float((i & 1) ? (w & 0xFFFF0000u) : (w << 16));
    }
};
template <>
struct Pack8<float> {
    uint4 lo, hi;
    __device__ __forceinline__ void load(const float* p) {
        lo = *reinterpret_cast<const uint4*>(p);
        hi = *reinterpret_cast<const uint4*>(p + 4);
    }
    __device__ __forceinline__ void load_stream(const float* p) {
        lo = load_stream16(p);
        hi = load_stream16(p + 4);
    }
    __device__ __forceinline__ void zero() { lo = hi = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ float operator[](int i) const {
        const uint4& q = i < 4 ? lo : hi;
        const uint32_t w = (i & 3) == 0 ? q.x : (i & 3) == 1 ? q.y : (i & 3) == 2 ? q.z : q.w;
        return __uint_as_float(w);
    }
};

__device__ __forceinline__ uint4 pack8_bf16(const float (&f)[8]) {
    return make_uint4(pack_bf16_rne(f[0], f[1]), pack_bf16_rne(f[2], f[3]), pack_bf16_rne(f[4], f[5]), pack_bf16_rne(f[6], f[7]));
}
__device__ __forceinline__ void store8(bf16_t* p, const float (&f)[8]) { *reinterpret_cast<uint4*>(p) = pack8_bf16(f); }
__device__ __forceinline__ void store8(float* p, const float (&f)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ void store8_stream(bf16_t* p, const float (&f)[8]) { store_stream16(p, pack8_bf16(f)); }
__device__ __forceinline__ void store8_stream(float* p, const float (&f)[8]) {
    store_stream16(p, make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])));
    store_stream16(p + 4, make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])));
}

// 1 / (1 + e^-v), each step rounded as written (the choice of experts goes by these bits)
__device__ __forceinline__ float sigmoid(float v) { return 1.0f / (1.0f + expf(-v)); }

// Row kernels: `waves` wavefronts to a row of eight elements per lane, and so many rows that a workgroup has four wavefronts
// where a row needs fewer.
struct RowShape {
    uint32_t waves, rows_per_wg;
    __host__ __device__ uint32_t threads() const { return 64 * waves * rows_per_wg; }
};
__host__ __device__ inline RowShape row_shape(uint32_t H) {
    const uint32_t w = (H + 511) / 512;
    RowShape s;
    s.waves = w < 1 ? 1 : w > 16 ? 16 : w;
    s.rows_per_wg = s.waves >= 3 ? 1 : 4 / s.waves;
    return s;
}

}  // namespace fluxmoe
