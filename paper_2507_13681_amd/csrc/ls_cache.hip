// Rows of K and V into the pages of a cache and back (ls_cache_write, ls_cache_read).
//
// Bound by memory: each row is read and written once, and of each position the table's entry.  8 KV heads of 128, e4m3, us: 32768 bf16 rows written 43 (4.7 TB/s, read and written), four caches of
// 16384 read back 79 (5.1 TB/s; a copy of 1 GiB reaches 5.15); one row of each of four sequences written 4.6, where an empty launch is 2.6.
// e2m1: 10923 rows written 17.2, or 13.1 where they are on the chip, or 22 (kernel) behind a call that wrote 134 MB (57 MB: 11 at a copy's rate), 32768 read back 37.6 (kernel 33, 5.1 TB/s).
#include "ls_rows.h"

namespace ls {

constexpr int MOVE_THREADS = 256;
// The chip's last-level cache.  A call whose tensors have more (all their rows: what `count` leaves of them only the device knows) reads pages past it: they would only displace the rows that it writes, which are wanted next.  Rows read back, together with a call that reads those,
// us: four caches of 16384 e4m3 246 -> 233, bf16 268 -> 249; of less data, which the next call may still find there, 16384 rows to fp32 94 for 87 where the same pages are read again.
// Rows that a call writes, or reads from the caller's tensor, never pass it by: 32768 rows read back would take 32 instead of 42 us, and with a call that reads them 131 instead of 123.
constexpr int64_t ON_CHIP = 256 << 20;

// Loads by f(load) of what is wanted once (`once`, wave-uniform) or again.  The empty statements keep the two sides apart: joined, all would be ordinary loads.
template <typename F>
__device__ __forceinline__ void load_by(bool once, F f) {
    if (once) { asm volatile(""); f([](auto* p) { return __builtin_nontemporal_load(p); }); asm volatile(""); }
    else f([](auto* p) { return *p; });
}

// grid (blocks of rows, groups of KV heads).  A workgroup has 256 / (d / 8) neighbouring rows, and of a row d / 8 lanes eight values each: whose sequence each
// row is of, and the place that the table gives it, are found once for all its heads and for K and V.
template <bool WRITE, typename T, int TYPE, int D>
__global__ __launch_bounds__(MOVE_THREADS) void move_kernel(MoveArgs a) {
    constexpr int LPR = D / 8, ROWS = MOVE_THREADS / LPR, SRC = Elem<T>::bytes;
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
    if (b < 0) return;
    const int h0 = blockIdx.y * a.heads, h1 = h0 + a.heads < a.cache.Hkv ? h0 + a.heads : a.cache.Hkv;
    const int64_t seq = a.starts ? 0 : b;
    unsigned char* const rows[2] = {a.k.data + (seq * a.k.seq + at * a.k.row + 8 * part) * SRC, a.v.data + (seq * a.v.seq + at * a.v.row + 8 * part) * SRC};
    const int64_t step[2] = {a.k.head * SRC, a.v.head * SRC};
    // Rows that are written go by here four at a time; the first of them into bf16 pages are asked for before it is known where they go.  (Us, with / without: 10923 rows of 8 heads of 128 18.1 / 18.7, 24 sequences of 0 to 512 padded
    // 9.5 / 10.1; codes have more to do behind their loads and gain nothing: e4m3 15.0 / 14.7, 11.1 / 10.6, e2m1 13.5 / 13.4, 10.0 / 9.7.)  Rows that are none are not read: a padded batch is mostly those.
    constexpr bool AHEAD = WRITE && TYPE == CACHE_BF16;
    Eight<T> ahead[4];
    auto ask = [&](int h) {
#pragma unroll
        for (int j = 0; j < 4; ++j) ahead[j].load(rows[j & 1] + (h + j / 2) * step[j & 1]);
    };
    if (AHEAD && h0 + 2 <= h1) ask(h0);
    const int64_t p = (a.pos ? (int64_t)a.pos[b] : 0) + i;
    const int page = page_of(a.cache, b, p);
    if (page < 0 && part == 0 && blockIdx.y == 0) atomicOr(a.status, STAT_PAGE_RANGE);
    if (page < 0) return;
    const int64_t place = ((int64_t)page * a.cache.Hkv << a.cache.page_log) + (p & ((1 << a.cache.page_log) - 1));       // of head 0, in rows
    unsigned char* const pool[2] = {a.cache.k, a.cache.v};
    uint8_t* const exps[2] = {a.cache.kx, a.cache.vx};
    auto put = [&](const Eight<T>& x, int h, int t) {      // into the cache
        const Eight<T> one[1] = {x};
        store_part<TYPE, D, 8>(one, pool[t], exps[t], place + ((int64_t)h << a.cache.page_log), part);
    };
    if constexpr (WRITE) {
        int h = h0;
        for (; h + 2 <= h1; h += 2) {                      // four rows in flight
            if (!AHEAD || h != h0) ask(h);
#pragma unroll
            for (int j = 0; j < 4; ++j) put(ahead[j], h + j / 2, j & 1);
        }
        for (; h < h1; ++h)
#pragma unroll
            for (int t = 0; t < 2; ++t) { Eight<T> x; x.load(rows[t] + h * step[t]); put(x, h, t); }
    } else {
        auto get = [&](auto load, int h, int t, uint2& w, Eight<bf16_t>& x, uint32_t& E) {
            const int64_t r = place + ((int64_t)h << a.cache.page_log);
            const unsigned char* src = pool[t] + r * stored_bytes(TYPE, D) + part * stored_bytes(TYPE, 8);
            if constexpr (TYPE == CACHE_E2M1) {
                w.x = load(reinterpret_cast<const uint32_t*>(src));
                E = exps[t][r * (D / 32) + part / 4];
            } else if constexpr (TYPE == CACHE_E4M3) {
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
            if constexpr (TYPE == CACHE_E2M1) {
                const float f = power_of(E);
                auto two = [&](auto i) {                   // byte i's
                    constexpr int I = decltype(i)::value;
                    if constexpr (std::is_same<T, float>::value) {
                        const auto z = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w.x, f, I);
                        y.set(2 * I, z[0]); y.set(2 * I + 1, z[1]);
                    } else {
                        const auto z = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w.x, f, I);
                        y.set(2 * I, (float)z[0]); y.set(2 * I + 1, (float)z[1]);
                    }
                };
                two(std::integral_constant<int, 0>{}); two(std::integral_constant<int, 1>{}); two(std::integral_constant<int, 2>{}); two(std::integral_constant<int, 3>{});
            } else if constexpr (TYPE == CACHE_E4M3) {
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

template <bool WRITE, typename T, int TYPE, int D>
static hipError_t run_move_t(MoveArgs a, hipStream_t st) {
    constexpr int ROWS = MOVE_THREADS / (D / 8), BYTES = D * Elem<T>::bytes + stored_bytes(TYPE, D);
    const int64_t rows = (a.starts ? 1 : (int64_t)a.B) * a.n_hat;
    const int64_t blocks = (rows + ROWS - 1) / ROWS;
    // All heads of a row in one workgroup where there are rows enough: what a row is and where it goes is found once for them.  Two heads of them otherwise, for more workgroups.  All heads / two, us:
    // four caches of 16384 (their pages through the caches), packed 81 / 86, padded 81 / 79, 16384 rows of 32 heads of 64 49 / 51, four single rows 5.5 / 4.7, 3400 rows of fp32 5.8 / 5.4.
    a.heads = a.cache.Hkv;
    while (a.heads > 2 && blocks * ((a.cache.Hkv + a.heads - 1) / a.heads) < 2048) a.heads = (a.heads + 1) / 2;
    a.once = rows * a.cache.Hkv * (2 * BYTES) > ON_CHIP;
    for (a.group0 = 0; a.group0 < blocks; a.group0 += MOVE_GROUPS) {
        const int64_t here = blocks - a.group0 < MOVE_GROUPS ? blocks - a.group0 : MOVE_GROUPS;
        hipLaunchKernelGGL((move_kernel<WRITE, T, TYPE, D>), dim3((uint32_t)here, (a.cache.Hkv + a.heads - 1) / a.heads), dim3(MOVE_THREADS), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <bool WRITE, typename T>
static hipError_t run_move_d(const MoveArgs& a, int type, int d, hipStream_t st) {
    if (type == CACHE_E2M1) return d == 128 ? run_move_t<WRITE, T, CACHE_E2M1, 128>(a, st) : run_move_t<WRITE, T, CACHE_E2M1, 64>(a, st);
    if (type == CACHE_E4M3) return d == 128 ? run_move_t<WRITE, T, CACHE_E4M3, 128>(a, st) : run_move_t<WRITE, T, CACHE_E4M3, 64>(a, st);
    return d == 128 ? run_move_t<WRITE, T, CACHE_BF16, 128>(a, st) : run_move_t<WRITE, T, CACHE_BF16, 64>(a, st);
}
hipError_t run_move(const MoveArgs& a, bool write, int dtype, int type, int d, hipStream_t st) {
    if (write) return dtype == 0 ? run_move_d<true, bf16_t>(a, type, d, st) : run_move_d<true, float>(a, type, d, st);
    return dtype == 0 ? run_move_d<false, bf16_t>(a, type, d, st) : run_move_d<false, float>(a, type, d, st);
}

}  // namespace ls
