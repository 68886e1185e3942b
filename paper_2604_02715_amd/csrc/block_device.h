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

// A row in memory, for the wavefront as a whole: reads past its columns give 0 and writes there do nothing, and a row of no
// columns takes the place of one that is not there.  So the kernels below have no branches around their loads and stores, and a
// wait for a load counts exactly what was issued behind it.
typedef __amdgpu_buffer_rsrc_t row_t;
template <typename T>
__device__ __forceinline__ row_t row_at(const T* base, uint64_t row, uint64_t stride, uint32_t columns) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(base + row * stride), 0, int(columns * sizeof(T)), 0x00020000);
}
constexpr int kCached = 0, kStream = 2;      // cache policies: the usual one; touched once (non-temporal)

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// N consecutive elements in registers, as loaded.  arrive() is the place where a load has to be complete: ahead of stores, as a
// later wait for it would be one for them, too (loads and stores count down one counter, in the order of their issue).
template <typename T, int N>
struct Pack;
template <>
struct Pack<bf16_t, 8> {
    u32x4 v;
    template <int POLICY>
    __device__ __forceinline__ void load(row_t row, uint32_t c) { v = __builtin_amdgcn_raw_buffer_load_b128(row, c * 2, 0, POLICY); }
    __device__ __forceinline__ void arrive() { asm volatile("" : "+v"(v)); }
    __device__ __forceinline__ float operator[](int i) const { return __uint_as_float((i & 1) ? (v[i / 2] & 0xFFFF0000u) : (v[i / 2] << 16)); }
};
template <>
struct Pack<bf16_t, 4> {
    u32x2 v;
    template <int POLICY>
    __device__ __forceinline__ void load(row_t row, uint32_t c) { v = __builtin_amdgcn_raw_buffer_load_b64(row, c * 2, 0, POLICY); }
    __device__ __forceinline__ void arrive() { asm volatile("" : "+v"(v)); }
    __device__ __forceinline__ float operator[](int i) const { return __uint_as_float((i & 1) ? (v[i / 2] & 0xFFFF0000u) : (v[i / 2] << 16)); }
};
template <>
struct Pack<float, 4> {
    u32x4 v;
    template <int POLICY>
    __device__ __forceinline__ void load(row_t row, uint32_t c) { v = __builtin_amdgcn_raw_buffer_load_b128(row, c * 4, 0, POLICY); }
    __device__ __forceinline__ void arrive() { asm volatile("" : "+v"(v)); }
    __device__ __forceinline__ float operator[](int i) const { return __uint_as_float(v[i]); }
};
template <>
struct Pack<float, 8> {
    Pack<float, 4> lo, hi;
    template <int POLICY>
    __device__ __forceinline__ void load(row_t row, uint32_t c) {
        lo.load<POLICY>(row, c);
        hi.load<POLICY>(row, c + 4);
    }
    __device__ __forceinline__ void arrive() { lo.arrive(); hi.arrive(); }
    __device__ __forceinline__ float operator[](int i) const { return i < 4 ? lo[i] : hi[i - 4]; }
};

// N values rounded to the row's type and written from column c on.
template <typename T, int N, int POLICY>
__device__ __forceinline__ void store(row_t row, uint32_t c, const float* f) {
    static_assert(N % 4 == 0, "pieces of four columns");
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const u32x4 v = {__float_as_uint(f[i]), __float_as_uint(f[i + 1]), __float_as_uint(f[i + 2]), __float_as_uint(f[i + 3])};
            __builtin_amdgcn_raw_buffer_store_b128(v, row, (c + i) * 4, 0, POLICY);
        }
    } else if constexpr (N == 8) {
        const u32x4 v = {pack_bf16_rne(f[0], f[1]), pack_bf16_rne(f[2], f[3]), pack_bf16_rne(f[4], f[5]), pack_bf16_rne(f[6], f[7])};
        __builtin_amdgcn_raw_buffer_store_b128(v, row, c * 2, 0, POLICY);
    } else {
        const u32x2 v = {pack_bf16_rne(f[0], f[1]), pack_bf16_rne(f[2], f[3])};
        __builtin_amdgcn_raw_buffer_store_b64(v, row, c * 2, 0, POLICY);
    }
}

// An element that the whole wavefront reads and nothing in the launch writes: through the scalar cache, so that the wait for it
// is not a wait for the vector loads and stores that are under way.
template <typename T>
__device__ __forceinline__ T scalar_at(const T* p, uint64_t i) {
    return ((const __attribute__((address_space(4))) T*)(uintptr_t)p)[i];
}

// What a lane loads at once of rows of types A and B: eight columns where both are BF16, four where one is FP32, so that a lane's
// load has at most 16 bytes and a wavefront's no gaps between lanes (FP32 rows added up by token: pieces of four 62 us, of eight 68;
// BF16 to FP32 34 / 35; BF16 to BF16 42 / 34).
template <typename A, typename B>
constexpr int kPiece = sizeof(A) == 2 && sizeof(B) == 2 ? 8 : 4;

// 1 / (1 + e^-v), each step rounded as written (the choice of experts goes by these bits).
__device__ __forceinline__ float sigmoid(float v) { return 1.0f / (1.0f + expf(-v)); }

// The same of eight values.  The quotient by one Newton step on the hardware's reciprocal (Markstein 1990): equal to the division for
// every significand of the divisor, which the tests go through; where one leaves the normal numbers, the division itself.
__device__ __forceinline__ void sigmoid8(const float* v, float* s) {
    float d[8], most = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        d[j] = 1.0f + expf(-v[j]);
        most = fmaxf(most, d[j]);
        const float r = __builtin_amdgcn_rcpf(d[j]);
        s[j] = fmaf(fmaf(-d[j], r, 1.0f), r, r);
    }
    if (most > 0x1p100f) {
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] = 1.0f / d[j];
    }
}

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
