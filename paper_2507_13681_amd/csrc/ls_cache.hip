// Rows of K and V into the pages of a cache and back (ls_cache_write, ls_cache_read).
//
// A row has d values of one position and KV head.  e4m3 pages hold code = x * 2^(127 - E), rounded to nearest even, with one byte E a row: the least power of
// two by which the row's largest finite value fits under 448, the largest of e4m3.  A power of two, and not max / 448: the products are exact, so that the
// only rounding is that of the code, a stored value times its power is a bf16, and the attention over it needs no scaled products; what it costs is at most one of the
// fifteen binades of e4m3 below a row's largest value.
//
// Bound by memory: each row is read and written once, and of each position the table's entry.  8 KV heads of 128, e4m3, us: 32768 bf16 rows written 43 (4.7 TB/s, read and written), four caches of
// 16384 read back 79 (5.1 TB/s; a copy of 1 GiB reaches 5.15); one row of each of four sequences written 4.6, where an empty launch is 2.6.
#include <type_traits>
#include "ls_device.h"
#include "ls_internal.h"

namespace ls {

constexpr int MOVE_THREADS = 256;
// The chip's last-level cache.  A call whose tensors have more (all their rows: what `count` leaves of them only the device knows) reads pages past it: they would only displace the rows that it writes, which are wanted next.  Rows read back, together with a call that reads those,
// us: four caches of 16384 e4m3 246 -> 233, bf16 268 -> 249; of less data, which the next call may still find there, 16384 rows to fp32 94 for 87 where the same pages are read again.
// Rows that a call writes, or reads from the caller's tensor, never pass it by: 32768 rows read back would take 32 instead of 42 us, and with a call that reads them 131 instead of 123.
constexpr int64_t ON_CHIP = 256 << 20;
// Workgroups of a launch.  A dimension of a grid has less than 2^32 threads: of one that has more, HIP runs what is left of the number modulo 2^32, and says nothing.
constexpr int64_t MOVE_GROUPS = 1 << 23;

// Largest over the LPR (8 or 16) neighbouring lanes of a row
template <int LPR>
__device__ __forceinline__ float row_largest(float x) {
    auto with = [](float v, auto ctrl) {
        return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, 0xF, 0xF, false)));
    };
    x = with(x, std::integral_constant<int, 0xB1>{});      // quad_perm 1,0,3,2
    x = with(x, std::integral_constant<int, 0x4E>{});      // quad_perm 2,3,0,1
    x = with(x, std::integral_constant<int, 0x141>{});     // row_half_mirror
    if (LPR == 16) x = with(x, std::integral_constant<int, 0x140>{});                        // row_mirror
    return x;
}
// The exponent byte of a row whose largest finite value is x >= 0: 448 is 1.75 * 2^8
__device__ __forceinline__ uint32_t row_exponent(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const int e = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return e > 10 ? (uint32_t)e : 10u;                     // (below, the smallest code would be no normal bf16)
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

// Loads by f(load) of what is wanted once (`once`, wave-uniform) or again.  The empty statements keep the two sides apart: joined, all would be ordinary loads.
template <typename F>
__device__ __forceinline__ void load_by(bool once, F f) {
    if (once) { asm volatile(""); f([](auto* p) { return __builtin_nontemporal_load(p); }); asm volatile(""); }
    else f([](auto* p) { return *p; });
}

// grid (blocks of rows, groups of KV heads).  A workgroup has 256 / (d / 8) neighbouring rows, and of a row d / 8 lanes eight values each: whose sequence each
// row is of, and the place that the table gives it, are found once for all its heads and for K and V.
template <bool WRITE, typename T, bool E4M3, int D>
__global__ __launch_bounds__(MOVE_THREADS) void move_kernel(MoveArgs a) {
    constexpr int LPR = D / 8, ROWS = MOVE_THREADS / LPR, SRC = Elem<T>::bytes, DST = E4M3 ? 1 : 2;
    __shared__ int seq_s[ROWS], stop_s;
    const int tid = threadIdx.x, slot = tid / LPR, part = tid % LPR;
    const int64_t row0 = (a.group0 + blockIdx.x) * ROWS;
    const bool first = row0 == 0 && blockIdx.y == 0;
    int b = -1, i = 0;
    int64_t at = row0 + slot;                              // the row, and that of the tensor it is
    if (a.starts) {
        // Each sequence lays claim to its rows among these, up to the first one whose starts are none.
        if (tid < ROWS) seq_s[tid] = -1;
        if (tid == 0) stop_s = a.B;
        __syncthreads();
        for (int s = tid; s < a.B; s += MOVE_THREADS)
            if (!starts_ok(a.starts[s], a.starts[s + 1], a.n_hat)) atomicMin(&stop_s, s);
        __syncthreads();
        const int stop = stop_s;
        for (int s = tid; s < stop; s += MOVE_THREADS) {
            const int64_t x = a.starts[s], y = a.starts[s + 1];
            const int64_t lo = x > row0 ? x : row0, hi = y < row0 + ROWS ? y : row0 + ROWS;
            for (int64_t r = lo; r < hi; ++r) seq_s[r - row0] = s;
        }
        if (stop < a.B && first && tid == 0) atomicOr(a.status, STAT_STARTS);
        __syncthreads();
        b = seq_s[slot];
        if (b >= 0) i = (int)(at - a.starts[b]);
    } else if (at < (int64_t)a.B * a.n_hat) {
        b = (int)(at / a.n_hat);
        i = (int)(at - (int64_t)b * a.n_hat);
        at = i;
        if (a.count && i >= a.count[b]) b = -1;
    }
    int page = -1;
    int64_t p = 0;
    if (b >= 0) {
        p = (a.pos ? (int64_t)a.pos[b] : 0) + i;
        page = page_of(a.cache, b, p);
        if (page < 0 && part == 0 && blockIdx.y == 0) atomicOr(a.status, STAT_PAGE_RANGE);
    }
    if (page < 0) return;
    const int h0 = blockIdx.y * a.heads, h1 = h0 + a.heads < a.cache.Hkv ? h0 + a.heads : a.cache.Hkv;
    const int64_t seq = a.starts ? 0 : b;
    const int64_t place = ((int64_t)page * a.cache.Hkv << a.cache.page_log) + (p & ((1 << a.cache.page_log) - 1));       // of head 0, in rows
    unsigned char* const rows[2] = {a.k.data + (seq * a.k.seq + at * a.k.row + 8 * part) * SRC, a.v.data + (seq * a.v.seq + at * a.v.row + 8 * part) * SRC};
    const int64_t step[2] = {a.k.head * SRC, a.v.head * SRC};
    unsigned char* const pool[2] = {a.cache.k, a.cache.v};
    uint8_t* const exps[2] = {a.cache.kx, a.cache.vx};
    auto put = [&](const Eight<T>& x, int h, int t) {      // into the cache
        const int64_t r = place + ((int64_t)h << a.cache.page_log);
        unsigned char* dst = pool[t] + r * (D * DST) + 8 * part * DST;
        if constexpr (E4M3) {
            float m = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) { const float y = fabsf(x.at(e)); m = fmaxf(m, y < INFINITY ? y : 0.f); }
            const uint32_t E = row_exponent(row_largest<LPR>(m));
            const float f = power_of(254u - E);
            uint32_t w[2] = {0u, 0u};
#pragma unroll
            for (int e = 0; e < 8; e += 4) {
                int u = __builtin_amdgcn_cvt_pk_fp8_f32(x.at(e) * f, x.at(e + 1) * f, 0, false);
                w[e / 4] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x.at(e + 2) * f, x.at(e + 3) * f, u, true);
            }
            *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
            if (part == 0) exps[t][r] = (uint8_t)E;
        } else {
            Eight<bf16_t> y;
#pragma unroll
            for (int e = 0; e < 8; ++e) y.set(e, x.at(e));
            y.store(dst);
        }
    };
    if constexpr (WRITE) {
        int h = h0;
        for (; h + 2 <= h1; h += 2) {                      // four rows in flight
            Eight<T> x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j].load(rows[j & 1] + (h + j / 2) * step[j & 1]);
#pragma unroll
            for (int j = 0; j < 4; ++j) put(x[j], h + j / 2, j & 1);
        }
        for (; h < h1; ++h)
#pragma unroll
            for (int t = 0; t < 2; ++t) { Eight<T> x; x.load(rows[t] + h * step[t]); put(x, h, t); }
    } else {
        auto get = [&](auto load, int h, int t, uint2& w, Eight<bf16_t>& x, uint32_t& E) {
            const int64_t r = place + ((int64_t)h << a.cache.page_log);
            const unsigned char* src = pool[t] + r * (D * DST) + 8 * part * DST;
            if constexpr (E4M3) {
                typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
                const u32x2 y = load(reinterpret_cast<const u32x2*>(src));
                w = make_uint2(y.x, y.y);
                E = exps[t][r];
            } else {
                x.v = load(reinterpret_cast<const bf16x8*>(src));
            }
        };
        auto give = [&](int h, int t, const uint2& w, const Eight<bf16_t>& x, uint32_t E) {
            Eight<T> y;
            if constexpr (E4M3) {
                const float f = power_of(E);               // (of which a conversion looks at the exponent alone: 2^-127 for 0, and NaN comes of 255)
                const uint32_t u[2] = {w.x, w.y};
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    if constexpr (std::is_same<T, float>::value) {               // (by way of bf16 codes of the bytes 0 to 2 would lose bits)
                        typedef __attribute__((ext_vector_type(2))) float f32x2;
                        const f32x2 z = (e & 2) ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(u[e / 4], f, true) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(u[e / 4], f, false);
                        y.set(e, z.x); y.set(e + 1, z.y);
                    } else {
                        typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
                        const bf16x2 z = (e & 2) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[e / 4], f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[e / 4], f, false);
                        y.set(e, (float)z.x); y.set(e + 1, (float)z.y);
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) y.set(e, x.at(e));
            }
            y.store(rows[t] + h * step[t]);
        };
        int h = h0;
        for (; h + 2 <= h1; h += 2) {
            uint2 w[4]; Eight<bf16_t> x[4]; uint32_t E[4];
            load_by(a.once, [&](auto load) {
#pragma unroll
            for (int j = 0; j < 4; ++j) get(load, h + j / 2, j & 1, w[j], x[j], E[j]);
            });
#pragma unroll
            for (int j = 0; j < 4; ++j) give(h + j / 2, j & 1, w[j], x[j], E[j]);
        }
        for (; h < h1; ++h)
#pragma unroll
            for (int t = 0; t < 2; ++t) { uint2 w; Eight<bf16_t> x; uint32_t E; load_by(a.once, [&](auto load) { get(load, h, t, w, x, E); }); give(h, t, w, x, E); }
    }
}

template <bool WRITE, typename T, bool E4M3, int D>
static hipError_t run_move_t(MoveArgs a, hipStream_t st) {
    constexpr int ROWS = MOVE_THREADS / (D / 8), BYTES = Elem<T>::bytes + (E4M3 ? 1 : 2);
    const int64_t rows = (a.starts ? 1 : (int64_t)a.B) * a.n_hat;
    const int64_t blocks = (rows + ROWS - 1) / ROWS;
    // All heads of a row in one workgroup where there are rows enough: what a row is and where it goes is found once for them.  Two heads of them otherwise, for more workgroups.  All heads / two, us:
    // four caches of 16384 (their pages through the caches), packed 81 / 86, padded 81 / 79, 16384 rows of 32 heads of 64 49 / 51, four single rows 5.5 / 4.7, 3400 rows of fp32 5.8 / 5.4.
    a.heads = a.cache.Hkv;
    while (a.heads > 2 && blocks * ((a.cache.Hkv + a.heads - 1) / a.heads) < 2048) a.heads = (a.heads + 1) / 2;
    a.once = rows * a.cache.Hkv * (2 * D * BYTES) > ON_CHIP;
    for (a.group0 = 0; a.group0 < blocks; a.group0 += MOVE_GROUPS) {
        const int64_t here = blocks - a.group0 < MOVE_GROUPS ? blocks - a.group0 : MOVE_GROUPS;
        hipLaunchKernelGGL((move_kernel<WRITE, T, E4M3, D>), dim3((uint32_t)here, (a.cache.Hkv + a.heads - 1) / a.heads), dim3(MOVE_THREADS), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <bool WRITE, typename T>
static hipError_t run_move_d(const MoveArgs& a, int type, int d, hipStream_t st) {
    if (type) return d == 128 ? run_move_t<WRITE, T, true, 128>(a, st) : run_move_t<WRITE, T, true, 64>(a, st);
    return d == 128 ? run_move_t<WRITE, T, false, 128>(a, st) : run_move_t<WRITE, T, false, 64>(a, st);
}
hipError_t run_move(const MoveArgs& a, bool write, int dtype, int type, int d, hipStream_t st) {
    if (write) return dtype == 0 ? run_move_d<true, bf16_t>(a, type, d, st) : run_move_d<true, float>(a, type, d, st);
    return dtype == 0 ? run_move_d<false, bf16_t>(a, type, d, st) : run_move_d<false, float>(a, type, d, st);
}

}  // namespace ls
