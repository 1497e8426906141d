// Rows of K and V as they are stored in pages, and as callers' tensors hold them: shared by the kernels that move them (ls_cache.hip, ls_rotate.hip).
//
// A row has d values of one position and KV head.  e4m3 pages hold code = x * 2^(127 - E), rounded to nearest even, with one byte E a row: the least power of
// two by which the row's largest finite value fits under 448, the largest of e4m3.  A power of two, and not max / 448: the products are exact, so that the
// only rounding is that of the code, a stored value times its power is a bf16, and the attention over it needs no scaled products; what it costs is at most one of the
// fifteen binades of e4m3 below a row's largest value.  e2m1 pages hold two codes a byte and a byte E for each 32 values, likewise; values up to 7 become the largest code, 6: from there on they
// are as far from it as those between 4 and 6 may be from theirs, and the next power of two would take half of their codes from the 31 others.
#pragma once
#include <type_traits>
#include "ls_device.h"
#include "ls_internal.h"

namespace ls {

// Workgroups of a launch.  A dimension of a grid has less than 2^32 threads: of one that has more, HIP runs what is left of the number modulo 2^32, and says nothing.
constexpr int64_t MOVE_GROUPS = 1 << 23;

constexpr int stored_bytes(int type, int d) { return type == CACHE_BF16 ? 2 * d : type == CACHE_E4M3 ? d : d / 2; }         // of a row's values
constexpr int stored_exps(int type, int d) { return type == CACHE_BF16 ? 0 : type == CACHE_E4M3 ? 1 : d / 32; }             // and its exponents

// Largest over the LPR (2, 4, 8 or 16) neighbouring lanes of a row
template <int LPR>
__device__ __forceinline__ float row_largest(float x) {
    auto with = [](float v, auto ctrl) {
        return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, 0xF, 0xF, false)));
    };
    x = with(x, std::integral_constant<int, 0xB1>{});      // quad_perm 1,0,3,2
    if (LPR >= 4) x = with(x, std::integral_constant<int, 0x4E>{});                          // quad_perm 2,3,0,1
    if (LPR >= 8) x = with(x, std::integral_constant<int, 0x141>{});                         // row_half_mirror
    if (LPR == 16) x = with(x, std::integral_constant<int, 0x140>{});                        // row_mirror
    return x;
}
// The exponent byte of a row whose largest finite value is x >= 0: 448 is 1.75 * 2^8
__device__ __forceinline__ uint32_t row_exponent(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const int e = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return e > 10 ? (uint32_t)e : 10u;                     // (below, the smallest code would be no normal bf16)
}
// .. of 32 values in e2m1: 7 is 1.75 * 2^2
__device__ __forceinline__ uint32_t group_exponent(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const int e = (int)(u >> 23) - 2 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return e > 2 ? (uint32_t)e : 2u;
}
__device__ __forceinline__ float power_of(uint32_t E) { return __builtin_bit_cast(float, E << 23); }        // 2^(E - 127)

// Eight neighbouring values of a row, as they come and as floats
template <typename T> struct Eight;
template <> struct Eight<bf16_t> {
    bf16x8 v;
    __device__ void load(const unsigned char* p) { v = *reinterpret_cast<const bf16x8*>(p); }
    __device__ void store(unsigned char* p) const { *reinterpret_cast<bf16x8*>(p) = v; }
    __device__ float at(int i) const { return (float)v[i]; }
    __device__ void set(int i, float x) { v[i] = (__bf16)x; }
};
template <> struct Eight<float> {
    f32x4 v[2];
    __device__ void load(const unsigned char* p) { v[0] = reinterpret_cast<const f32x4*>(p)[0]; v[1] = reinterpret_cast<const f32x4*>(p)[1]; }
    __device__ void store(unsigned char* p) const { reinterpret_cast<f32x4*>(p)[0] = v[0]; reinterpret_cast<f32x4*>(p)[1] = v[1]; }
    __device__ float at(int i) const { return v[i / 4][i % 4]; }
    __device__ void set(int i, float x) { v[i / 4][i % 4] = x; }
};

// N neighbouring values x of a row of D, its lane's of D / N neighbouring lanes (`part`: which), into the pages: row r of the pool `pages`, exponents `exps`
template <int TYPE, int D, int N, typename T>
__device__ __forceinline__ void store_part(const Eight<T> (&x)[N / 8], unsigned char* pages, uint8_t* exps, int64_t r, int part) {
    unsigned char* const dst = pages + r * stored_bytes(TYPE, D) + part * stored_bytes(TYPE, N);
    if constexpr (TYPE == CACHE_BF16) {
#pragma unroll
        for (int c = 0; c < N / 8; ++c) {
            Eight<bf16_t> y;
#pragma unroll
            for (int e = 0; e < 8; ++e) y.set(e, x[c].at(e));
            y.store(dst + 16 * c);
        }
    } else if constexpr (TYPE == CACHE_E4M3) {
        float m = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) { const float y = fabsf(x[e / 8].at(e % 8)); m = fmaxf(m, y < INFINITY ? y : 0.f); }
        const uint32_t E = row_exponent(row_largest<D / N>(m));
        const float f = power_of(254u - E);
#pragma unroll
        for (int c = 0; c < N / 8; ++c) {
            uint32_t w[2] = {0u, 0u};
#pragma unroll
            for (int e = 0; e < 8; e += 4) {
                int u = __builtin_amdgcn_cvt_pk_fp8_f32(x[c].at(e) * f, x[c].at(e + 1) * f, 0, false);
                w[e / 4] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[c].at(e + 2) * f, x[c].at(e + 3) * f, u, true);
            }
            *reinterpret_cast<uint2*>(dst + 8 * c) = make_uint2(w[0], w[1]);
        }
        if (part == 0) exps[r] = (uint8_t)E;
    } else {
        float m = 0.f;                                     // (infinite where a value is none)
#pragma unroll
        for (int e = 0; e < N; ++e) { const float y = fabsf(x[e / 8].at(e % 8)); m = fmaxf(m, y < INFINITY ? y : INFINITY); }
        m = row_largest<32 / N>(m);
        const bool fine = m < INFINITY;
        const uint32_t E = fine ? group_exponent(m) : 255u;
        const float f = power_of(254u - E);
#pragma unroll
        for (int c = 0; c < N / 8; ++c) {
            const Eight<T>& y = x[c];
            uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, y.at(0) * f, y.at(1) * f, 1.0f, 0);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y.at(2) * f, y.at(3) * f, 1.0f, 1);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y.at(4) * f, y.at(5) * f, 1.0f, 2);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y.at(6) * f, y.at(7) * f, 1.0f, 3);
            *reinterpret_cast<uint32_t*>(dst + 4 * c) = fine ? w : 0u;
        }
        if (part % (32 / N) == 0) exps[r * (D / 32) + part / (32 / N)] = (uint8_t)E;
    }
}

}  // namespace ls
