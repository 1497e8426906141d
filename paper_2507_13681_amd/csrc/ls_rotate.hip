// Norms of queries and keys head by head, and the rotation by their positions, in one pass (ls_norm_rotate):
//     y = x / sqrt(mean(x^2) + eps) * w,     (a, b) -> (a cos t - b sin t, b cos t + a sin t)  for the pairs of the first `dims` values,  t = position * freq[pair],
// into rows, and K (with V as it is) into the pages of a cache by their slots.
//
// Bound by memory: each row is read and written once.  A row of a head is d / 16 neighbouring lanes', eight values here and eight there: of those that are rotated the chunks of eight values c and
// c + dims / 16, so that both values of a pair are in one lane whichever way pairs are counted.
// Angles.  A position times a frequency is formed in 64 bits and brought into a quarter turn there (t - k pi / 2 with pi / 2 in two parts): in 32 bits the angle of position 260000 would be off by up to
// 2^-7.  Sine and cosine of what is left, at most pi / 4, are their series up to t^9 and t^10, whose next terms are below 2^-29.  The angles of a workgroup's rows are formed once, one or a few a
// thread, and handed out through LDS: a workgroup has whole rows as far as it can (32 and 8 heads of 128: 4 rows of 40), since each row's 64 sines and cosines are as many instructions as the row itself.
// 32 and 8 heads of 128, us: 32768 rows 128 (671 MB, 5.2 TB/s, a copy's rate; angles formed by each group of lanes for its heads of a row, 138), 23897 rows into rows and pages 122 (5.2 TB/s), e4m3 129, e2m1 128 (4.5 and 4.4 TB/s, 114 and 110 at a copy's rate); a row of each of four sequences into
// pages 4.2 (kernel 3.8; recorded into a graph 2.9), where an empty launch is 2.6.
// Pages.  What a row becomes is rounded to the rows' type and then stored as ls_cache_write stores it, so that both ways give the same pages; 8 and 4 bits want
// neighbouring values in a lane, which LDS brings together (a row's lanes are one wave's: no barrier).
#include "ls_rows.h"

namespace ls {

constexpr int ROTATE_THREADS = 256;
constexpr int NO_PAGES = -1;
constexpr int rotate_rows(int d) { return 4096 / d; }      // of a workgroup, at most
constexpr int ROTATE_FEW = 1280;

// Sum over the L (4 or 8) neighbouring lanes of a row, in every lane
template <int L>
__device__ __forceinline__ float row_sum(float x) {
    auto with = [](float v, auto ctrl) {
        return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, 0xF, 0xF, false));
    };
    x = with(x, std::integral_constant<int, 0xB1>{});      // quad_perm 1,0,3,2
    x = with(x, std::integral_constant<int, 0x4E>{});      // quad_perm 2,3,0,1
    if (L == 8) x = with(x, std::integral_constant<int, 0x141>{});                           // row_half_mirror
    return x;
}

__device__ __forceinline__ void sine_cosine(double t, float& sine, float& cosine) {
    const double k = __builtin_rint(t * 0.63661977236758134308);               // quarter turns
    const float x = (float)__builtin_fma(-k, 6.123233995736766036e-17, __builtin_fma(-k, 1.5707963267948965580, t));
    const int quarter = (int)__builtin_fma(-4.0, __builtin_rint(k * 0.25), k);  // -2 .. 2
    const float y = x * x;
    float s = __builtin_fmaf(y, 1.f / 362880.f, -1.f / 5040.f), c = __builtin_fmaf(y, -1.f / 3628800.f, 1.f / 40320.f);
    s = __builtin_fmaf(y, s, 1.f / 120.f);
    c = __builtin_fmaf(y, c, -1.f / 720.f);
    s = __builtin_fmaf(y, s, -1.f / 6.f);
    c = __builtin_fmaf(y, c, 1.f / 24.f);
    c = __builtin_fmaf(y, c, -0.5f);
    s = __builtin_fmaf(y * x, s, x);
    c = __builtin_fmaf(y, c, 1.f);
    sine = quarter & 1 ? c : s;
    cosine = quarter & 1 ? s : c;
    if (quarter & 2) sine = -sine;
    if ((quarter + 1) & 2) cosine = -cosine;
}

// A workgroup has `each` neighbouring rows and of those a.chunk heads, an item each: a row of a head, which a group of lanes takes.
template <typename T, int TYPE, int D, bool NEIGHBOURS>
__global__ __launch_bounds__(ROTATE_THREADS) void rotate_kernel(RotateArgs a) {
    constexpr int L = D / 16, GROUPS = ROTATE_THREADS / L, SIZE = Elem<T>::bytes, MOST = rotate_rows(D);
    constexpr bool GATHER = TYPE == CACHE_E4M3 || TYPE == CACHE_E2M1;
    __shared__ __align__(16) unsigned char gather_s[GATHER ? GROUPS * D * SIZE : 16];
    __shared__ __align__(16) float cosine_s[MOST * D / 2], sine_s[MOST * D / 2], weight_s[2][D];
    __shared__ int4 row_s[MOST];                           // sequence, number in it, page, place in the page
    const int tid = threadIdx.x, group = tid / L, p = tid % L;
    const uint32_t rows = (uint32_t)a.B * (uint32_t)a.n_hat, row0 = (uint32_t)(a.group0 + blockIdx.x) * (uint32_t)a.each;
    const int each = rows - row0 < (uint32_t)a.each ? (int)(rows - row0) : a.each;
    const int h0 = blockIdx.y * a.chunk, chunk = a.heads - h0 < a.chunk ? a.heads - h0 : a.chunk, items = each * chunk;
    // x / n for x of less than 2^13, off by nothing: the half is more than what the reciprocal may be off by
    auto over = [](int x, float per) { return (int)(((float)x + 0.5f) * per); };
    const float per_chunk = __builtin_amdgcn_rcpf((float)chunk), per_half = __builtin_amdgcn_rcpf((float)(a.dims / 2));
    // ---- what this lane has of a row
    const int turned = a.dims / 16, half = a.dims / 2;
    const bool turns = p < turned;
    const int c0 = turns ? p : 2 * p, c1 = turns ? p + turned : 2 * p + 1;
    auto address = [&](const RowArgs& r, int b, int i, int h) { return r.data + ((int64_t)b * r.seq + (int64_t)i * r.row + (int64_t)h * r.head) * SIZE; };
    Eight<T> x[2], next[2];
    auto load = [&](int b, int i, int h, Eight<T> (&to)[2]) {
        const bool is_v = TYPE != NO_PAGES && h >= a.Hq + a.Hkv;
        const unsigned char* r = h < a.Hq ? address(a.q, b, i, h) : is_v ? address(a.v, b, i, h - a.Hq - a.Hkv) : address(a.k, b, i, h - a.Hq);
        to[0].load(r + (is_v ? 2 * p : c0) * (8 * SIZE));
        to[1].load(r + (is_v ? 2 * p + 1 : c1) * (8 * SIZE));
    };
    auto sequence_of = [&](uint32_t row) { return a.B == 1 ? 0u : row / (uint32_t)a.n_hat; };
    // ---- of the rows: angles, weights, where they are and go.  All of it is asked for first, then the rows, and then one waits.
    int64_t slot = -1;
    if (TYPE != NO_PAGES && tid < each) slot = a.slots[row0 + tid];
    const float wq = a.q_weight && tid < D ? a.q_weight[tid] : 0.f, wk = a.k_weight && tid < D ? a.k_weight[tid] : 0.f;
    const int angles = each * half;
    int position = 0;
    float freq = 0.f;
    auto ask_angle = [&](int e) {
        const int at = over(e, per_half);
        const uint32_t row = row0 + at;
        position = a.positions ? a.positions[row] : (int)(row - sequence_of(row) * (uint32_t)a.n_hat);
        freq = a.freq[e - at * half];
    };
    if (tid < angles) ask_angle(tid);
    int k = group, r = over(k, per_chunk), h = h0 + k - r * chunk;
    if (k < items) {
        const uint32_t b = sequence_of(row0 + r);
        load((int)b, (int)(row0 + r - b * (uint32_t)a.n_hat), h, x);
    }
    for (int e = tid; e < angles; e += ROTATE_THREADS) {
        if (e != tid) ask_angle(e);
        sine_cosine((double)position * (double)freq, sine_s[e], cosine_s[e]);
    }
    if (tid < D) { weight_s[0][tid] = wq; weight_s[1][tid] = wk; }
    if (tid < each) {
        const uint32_t row = row0 + tid, b = sequence_of(row);
        int4 w = make_int4((int)b, (int)(row - b * (uint32_t)a.n_hat), -1, 0);
        if constexpr (TYPE != NO_PAGES) {
            const int64_t at = slot >> a.cache.page_log;
            if (slot >= 0 && at < (int64_t)a.cache.pages) { w.z = (int)at; w.w = (int)(slot & ((1 << a.cache.page_log) - 1)); }
            else if (slot >= 0 && blockIdx.y == 0) atomicOr(a.status, STAT_PAGE_RANGE);
        }
        row_s[tid] = w;
    }
    __syncthreads();
    for (; k < items; k += GROUPS) {
        const bool more = k + GROUPS < items;
        const int r1 = more ? over(k + GROUPS, per_chunk) : 0, h1 = h0 + k + GROUPS - r1 * chunk;
        if (more) {
            const int4 w = row_s[r1];
            load(w.x, w.y, h1, next);
        }
        const int4 at = row_s[r];
        const bool is_q = h < a.Hq;
        if (TYPE == NO_PAGES || h < a.Hq + a.Hkv) {
            float y[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] = x[e / 8].at(e % 8);
            if (is_q ? a.q_weight : a.k_weight) {
                const float* w = weight_s[is_q ? 0 : 1];
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 16; ++e) sum = __builtin_fmaf(y[e], y[e], sum);
                sum = row_sum<L>(sum);
                if (sum < 0x1p100f && (sum > 0x1p-60f || a.eps > 0x1p-40f)) {
                    const float f = __builtin_amdgcn_rsqf(__builtin_fmaf(sum, 1.f / D, a.eps));
#pragma unroll
                    for (int e = 0; e < 16; ++e) y[e] = y[e] * f * w[8 * (e < 8 ? c0 : c1) + e % 8];
                } else {                                   // squares that fp32 cannot hold
                    double s = 0.0;
#pragma unroll
                    for (int e = 0; e < 16; ++e) s = __builtin_fma((double)y[e], (double)y[e], s);
#pragma unroll
                    for (int o = 1; o < L; o *= 2) s += __shfl_xor(s, o, 64);
                    const double f = 1.0 / sqrt(s * (1.0 / D) + (double)a.eps);
#pragma unroll
                    for (int e = 0; e < 16; ++e) y[e] = (float)((double)y[e] * f * (double)w[8 * (e < 8 ? c0 : c1) + e % 8]);
                }
            }
            if (turns) {
                const float *cosine = cosine_s + r * half, *sine = sine_s + r * half;
#pragma unroll
                for (int e = 0; e < 8; ++e) {              // a pair
                    const int u = NEIGHBOURS ? 8 * (e / 4) + 2 * (e % 4) : e, v = NEIGHBOURS ? u + 1 : e + 8, n = NEIGHBOURS ? 4 * (e < 4 ? c0 : c1) + e % 4 : 8 * p + e;
                    const float c = cosine[n], s = sine[n], z = __builtin_fmaf(y[u], c, -(y[v] * s));
                    y[v] = __builtin_fmaf(y[v], c, y[u] * s);
                    y[u] = z;
                }
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e / 8].set(e % 8, y[e]);
            if (is_q || a.k_out.data) {
                unsigned char* to = is_q ? address(a.q_out, at.x, at.y, h) : address(a.k_out, at.x, at.y, h - a.Hq);
                x[0].store(to + c0 * (8 * SIZE));
                x[1].store(to + c1 * (8 * SIZE));
            }
        }
        if constexpr (TYPE != NO_PAGES) {
            if (!is_q && at.z >= 0) {
                const bool is_v = h >= a.Hq + a.Hkv;
                const int j = h - a.Hq - (is_v ? a.Hkv : 0);
                const int64_t row = (((int64_t)at.z * a.cache.Hkv + j) << a.cache.page_log) + at.w;
                unsigned char* pool = is_v ? a.cache.v : a.cache.k;
                uint8_t* exps = is_v ? a.cache.vx : a.cache.kx;
                if constexpr (GATHER) {
                    if (!is_v) {
                        unsigned char* mine = gather_s + group * D * SIZE;
                        __builtin_amdgcn_wave_barrier();   // (the reads of the item before come first)
                        x[0].store(mine + c0 * (8 * SIZE));
                        x[1].store(mine + c1 * (8 * SIZE));
                        __builtin_amdgcn_wave_barrier();
                        x[0].load(mine + 2 * p * (8 * SIZE));
                        x[1].load(mine + (2 * p + 1) * (8 * SIZE));
                    }
                    store_part<TYPE, D, 16>(x, pool, exps, row, p);
                } else {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        Eight<bf16_t> z;
#pragma unroll
                        for (int e = 0; e < 8; ++e) z.set(e, x[c].at(e));
                        z.store(pool + row * (2 * D) + (is_v ? 2 * p + c : c ? c1 : c0) * 16);
                    }
                }
            }
        }
        if (more) { x[0] = next[0]; x[1] = next[1]; r = r1; h = h1; }
    }
}

template <typename T, int TYPE, int D>
static hipError_t run_rotate_t(RotateArgs a, hipStream_t st) {
    constexpr int GROUPS = ROTATE_THREADS / (D / 16);
    const int64_t rows = (int64_t)a.B * a.n_hat;
    a.heads = a.Hq + (TYPE == NO_PAGES ? 1 : 2) * a.Hkv;
    // Three to six items a group where there are rows enough, as many as leave the fewest groups idle in the end; else one.  (32 and 8 heads of 128, us, one / more: into rows 500 rows 5.1 / 7.5,
    // 1000 7.8 / 9.4, 2500 13.9 / 12.2, 8000 48.9 / 38.4; into rows and pages 500 5.4 / 6.9, 800 7.9 / 8.1, 1000 8.8 / 8.6, 1500 10.9 / 9.7, 8000 56.2 / 47.4.)
    const bool few = rows * a.heads <= (int64_t)ROTATE_FEW * GROUPS;
    const int most = few ? GROUPS : 6 * GROUPS;
    a.chunk = a.heads < most ? a.heads : most;
    a.each = 1;
    float best = 0.f;
    for (int e = 1; e <= rotate_rows(D) && e * a.chunk <= most; ++e) {
        const int items = e * a.chunk, rounds = (items + GROUPS - 1) / GROUPS;
        const float use = (float)items / (float)(rounds * GROUPS) * (!few && rounds < 3 ? 0.5f : 1.f);
        if (use > best) { best = use; a.each = e; }
    }
    const int64_t blocks = (rows + a.each - 1) / a.each;
    for (a.group0 = 0; a.group0 < blocks; a.group0 += MOVE_GROUPS) {
        const int64_t here = blocks - a.group0 < MOVE_GROUPS ? blocks - a.group0 : MOVE_GROUPS;
        const dim3 grid((uint32_t)here, (a.heads + a.chunk - 1) / a.chunk);
        if (a.neighbours) hipLaunchKernelGGL((rotate_kernel<T, TYPE, D, true>), grid, dim3(ROTATE_THREADS), 0, st, a);
        else hipLaunchKernelGGL((rotate_kernel<T, TYPE, D, false>), grid, dim3(ROTATE_THREADS), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <typename T, int TYPE>
static hipError_t run_rotate_d(const RotateArgs& a, int d, hipStream_t st) { return d == 128 ? run_rotate_t<T, TYPE, 128>(a, st) : run_rotate_t<T, TYPE, 64>(a, st); }
template <typename T>
static hipError_t run_rotate_p(const RotateArgs& a, int type, int d, hipStream_t st) {
    if (type == CACHE_E2M1) return run_rotate_d<T, CACHE_E2M1>(a, d, st);
    if (type == CACHE_E4M3) return run_rotate_d<T, CACHE_E4M3>(a, d, st);
    return type == CACHE_BF16 ? run_rotate_d<T, CACHE_BF16>(a, d, st) : run_rotate_d<T, NO_PAGES>(a, d, st);
}
hipError_t run_rotate(const RotateArgs& a, int dtype, int type, int d, hipStream_t st) {
    return dtype == 0 ? run_rotate_p<bf16_t>(a, type, d, st) : run_rotate_p<float>(a, type, d, st);
}

}  // namespace ls
