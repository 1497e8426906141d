// One new token of each sequence over its pages (ls_paged_attend):
//     out = softmax(scale * q K^T) V   over the first len[b] positions of sequence b's cache.
//
// The step reads every K and V row once and does 4 d FLOP per (query head, key): it is bound by HBM bandwidth, at small sizes by latency.
// The query heads of a KV head are the columns of 16x16x32 products (NH blocks of 16), so that the rows are read once for all of them.
//   Work.  What there is to do follows from the lengths, which only the device knows: every wave (of e2m1 pages one of a workgroup) adds them up, cuts each KV head's 32-key tiles into parts of about
//   equal length (PagedLength) and finds the part that its workgroup has, so a batch of one long and many short sequences fills the chip as one of equals does.
//   A part.  The waves of a workgroup take its tiles in turn.  S^T = K Q^T with K fragments straight from global memory, online softmax per head in a lane,
//   P -> bf16, O^T += V^T P^T with the V^T fragments read transposed from a wave-private, swizzled LDS copy of the 32 V rows that a global -> LDS transfer filled.
//   e4m3: K codes become bf16 with their row's power of two in one instruction for two of them, exactly; V codes come through the 8-bit transpose read and
//   become bf16 as they are, and their rows' powers go into the probabilities, exactly too.
//   The waves' partial results are merged through LDS; where a head is in parts, the workgroup that finishes it last merges those, or, of many parts and query heads, a launch more does.
// One token, 8 KV heads of 128, caches not on the chip, us: one sequence with 32 query heads, 300 keys e4m3 7.1 (an empty launch is 2.6), 519 bf16 8.7, 131072 bf16 96.7 (5.6 TB/s), e4m3 54.9 (4.9 TB/s);
// 64 query heads, four e4m3 caches of 16384 31.1 (4.3 TB/s).  About 5 us of each pass before the first rows arrive and while results are put together (135, 212 and 537 MB take that more than at 5.1, 4.1 and 5.8 TB/s).
// Pages.  A page holds a multiple of 16 positions, so that each half of a tile lies in one: lane l of a wave keeps the page of half l of its next 64, and a
// tile's two are lane reads.  What lies behind the length in the last page is read with it, and left out by selects; a half in no page at all is read from page 0 and left out.
#include "ls_paged.h"

namespace ls {

// Parts of heads put together by a launch of its own: grid (B * Hq), a lane for two neighbouring values of a query head and every fourth part.
template <int D>
__global__ __launch_bounds__(2 * D) void paged_join_kernel(PagedArgs a) {
    constexpr int PS = D + 4, LANES = D / 2, SUBS = 4;
    __shared__ float2 red[SUBS][LANES + 1];                    // of each subset: values, and behind them its normaliser
    __shared__ float top[SUBS];
    const int tid = threadIdx.x, sub = tid / LANES, dd = 2 * (tid % LANES);
    const int b = blockIdx.x / a.Hq, hq = blockIdx.x % a.Hq, kvh = hq / a.G;
    PagedUnits w;
    if (!w.find_head(a, b, kvh, tid & 63) || w.cuts == 1) return;
    const float* src = a.part + ((int64_t)w.base * a.G + hq % a.G) * PS;
    const int64_t step = (int64_t)a.G * PS;
    float m = -INFINITY, o0 = 0.f, o1 = 0.f, l = 0.f;
    for (int s0 = sub; s0 < w.cuts; s0 += SUBS * PG_BATCH) {
        float2 x[PG_BATCH], ml[PG_BATCH];
#pragma unroll
        for (int e = 0; e < PG_BATCH; ++e) {
            const int s = s0 + e * SUBS < w.cuts ? s0 + e * SUBS : s0;
            x[e] = *reinterpret_cast<const float2*>(src + s * step + dd);
            ml[e] = *reinterpret_cast<const float2*>(src + s * step + D);
        }
        float m_new = m;
#pragma unroll
        for (int e = 0; e < PG_BATCH; ++e) m_new = fmaxf(m_new, ml[e].x);
        const float corr = m > -INFINITY ? fast_exp2((m - m_new) * a.scale_log2e) : 0.f;
        m = m_new; o0 *= corr; o1 *= corr; l *= corr;
#pragma unroll
        for (int e = 0; e < PG_BATCH; ++e) {
            const bool is = s0 + e * SUBS < w.cuts;            // (behind them part s0 once more: its infinities times 0 would be NaN)
            const float wgt = ml[e].x > -INFINITY ? fast_exp2((ml[e].x - m) * a.scale_log2e) : 0.f;
            o0 += is ? x[e].x * wgt : 0.f; o1 += is ? x[e].y * wgt : 0.f; l += is ? ml[e].y * wgt : 0.f;
        }
    }
    red[sub][tid % LANES] = make_float2(o0, o1);
    if (dd == 0) { red[sub][LANES] = make_float2(l, 0.f); top[sub] = m; }
    __syncthreads();
    if (sub > 0) return;
    for (int u = 1; u < SUBS; ++u) m = fmaxf(m, top[u]);
    o0 = o1 = l = 0.f;
    for (int u = 0; u < SUBS; ++u) {
        const float wgt = top[u] > -INFINITY ? fast_exp2((top[u] - m) * a.scale_log2e) : 0.f;
        const float2 x = red[u][tid % LANES];
        o0 += x.x * wgt; o1 += x.y * wgt; l += red[u][LANES].x * wgt;
    }
    const float inv = l != 0.f ? 1.f / l : 0.f;
    reinterpret_cast<uint32_t*>(reinterpret_cast<bf16_t*>(a.out) + (int64_t)blockIdx.x * D)[dd / 2] = (uint32_t)f2bf(o0 * inv) | ((uint32_t)f2bf(o1 * inv) << 16);
    if (a.lse && dd == 0) a.lse[blockIdx.x] = l != 0.f ? (m * a.scale_log2e + log2f(l)) * 0.69314718055994531f : -INFINITY;
}

// The same for e2m1 pages, by what paged_kernel left of the heads (their parts need not be found again, which is most of a workgroup's time), WIDTH values of a query head a workgroup.  Of few rows a workgroup for a
// whole one is the longest: one KV head of 128, 28129 positions, us by workgroups of 32 values / by paged_join_kernel: 32 query heads 14.5 / 16.3, 8 10.5 / 12.7; 65000, 32: 16.1 / 19.9.  Of many rows the workgroups
// are too many: 8 sequences of 9000, 64 query heads of 64, by 32 values 15.5, by 64 14.0.
constexpr int PAGED_JOIN_FEW = 256;
template <int D, int WIDTH>
__global__ __launch_bounds__(256) void paged4_join_kernel(PagedArgs a) {
    constexpr int PS = D + 4, LANES = WIDTH / 2, SUBS = 256 / LANES, SHARES = D / WIDTH;
    __shared__ float2 red[SUBS][LANES + 1];                    // of each subset: values, and behind them its normaliser
    __shared__ float top[SUBS];
    const int tid = threadIdx.x, sub = tid / LANES, at = tid % LANES, share = blockIdx.x % SHARES, row = blockIdx.x / SHARES;
    const int b = row / a.Hq, hq = row - b * a.Hq, kvh = hq / a.G, dd = WIDTH * share + 2 * at;
    const int2 parts = a.heads[b * a.Hkv + kvh];
    if (parts.y == 1) return;
    const float* src = a.part + ((int64_t)parts.x * a.G + hq % a.G) * PS;
    const int64_t step = (int64_t)a.G * PS;
    float m = -INFINITY, o0 = 0.f, o1 = 0.f, l = 0.f;
    for (int s0 = sub; s0 < parts.y; s0 += SUBS * PG_BATCH) {
        float2 x[PG_BATCH], ml[PG_BATCH];
#pragma unroll
        for (int e = 0; e < PG_BATCH; ++e) {
            const int s = s0 + e * SUBS < parts.y ? s0 + e * SUBS : s0;
            x[e] = *reinterpret_cast<const float2*>(src + s * step + dd);
            ml[e] = *reinterpret_cast<const float2*>(src + s * step + D);
        }
        float m_new = m;
#pragma unroll
        for (int e = 0; e < PG_BATCH; ++e) m_new = fmaxf(m_new, ml[e].x);
        const float corr = m > -INFINITY ? fast_exp2((m - m_new) * a.scale_log2e) : 0.f;
        m = m_new; o0 *= corr; o1 *= corr; l *= corr;
#pragma unroll
        for (int e = 0; e < PG_BATCH; ++e) {
            const bool is = s0 + e * SUBS < parts.y;           // (behind them part s0 once more: its infinities times 0 would be NaN)
            const float wgt = ml[e].x > -INFINITY ? fast_exp2((ml[e].x - m) * a.scale_log2e) : 0.f;
            o0 += is ? x[e].x * wgt : 0.f; o1 += is ? x[e].y * wgt : 0.f; l += is ? ml[e].y * wgt : 0.f;
        }
    }
    red[sub][at] = make_float2(o0, o1);
    if (at == 0) { red[sub][LANES] = make_float2(l, 0.f); top[sub] = m; }
    __syncthreads();
    if (sub > 0) return;
    for (int u = 1; u < SUBS; ++u) m = fmaxf(m, top[u]);
    o0 = o1 = l = 0.f;
    for (int u = 0; u < SUBS; ++u) {
        const float wgt = top[u] > -INFINITY ? fast_exp2((top[u] - m) * a.scale_log2e) : 0.f;
        const float2 x = red[u][at];
        o0 += x.x * wgt; o1 += x.y * wgt; l += red[u][LANES].x * wgt;
    }
    reinterpret_cast<uint32_t*>(reinterpret_cast<bf16_t*>(a.out) + (int64_t)row * D)[dd / 2] = (uint32_t)f2bf(l != 0.f ? o0 / l : 0.f) | ((uint32_t)f2bf(l != 0.f ? o1 / l : 0.f) << 16);
    if (a.lse && dd == 0) a.lse[row] = l != 0.f ? (m * a.scale_log2e + log2f(l)) * 0.69314718055994531f : -INFINITY;
}

void launch_paged_join(const PagedArgs& a, int d, hipStream_t st) {
    if (a.four) {
        const int rows = a.B * a.Hq;
        if (rows > PAGED_JOIN_FEW && d == 128) hipLaunchKernelGGL((paged4_join_kernel<128, 128>), dim3(rows), dim3(256), 0, st, a);
        else if (rows > PAGED_JOIN_FEW) hipLaunchKernelGGL((paged4_join_kernel<64, 64>), dim3(rows), dim3(256), 0, st, a);
        else if (d == 128) hipLaunchKernelGGL((paged4_join_kernel<128, 32>), dim3(rows * 4), dim3(256), 0, st, a);
        else hipLaunchKernelGGL((paged4_join_kernel<64, 32>), dim3(rows * 2), dim3(256), 0, st, a);
    } else if (d == 128) hipLaunchKernelGGL((paged_join_kernel<128>), dim3(a.B * a.Hq), dim3(2 * 128), 0, st, a);
    else hipLaunchKernelGGL((paged_join_kernel<64>), dim3(a.B * a.Hq), dim3(2 * 64), 0, st, a);
}

// A head's tiles are at most all there are, and a part no shorter than these by the slots: t / paged_length(..) <= slots / Hkv, whatever t is.
int paged_most_cuts(int B, int Hkv, int64_t most, bool four) {
    const int64_t heads = (int64_t)B * Hkv, tiles = (most + PAGED_TILE - 1) / PAGED_TILE, by_work = (paged_slots(heads) + Hkv - 1) / Hkv;
    const int least = paged_at_once(heads) ? paged_shortest(four) : PAGED_SHORTEST_MANY;
    const int64_t by_tiles = paged_cuts((int)tiles, least, paged_whole(heads, least, 1, four));
    return (int)(by_work < by_tiles ? by_work : by_tiles);
}
int paged_units(int B, int Hkv, int64_t most, bool four) {
    // no more than the slots, or beside those the head that each part begins; and no more than all heads of the longest would be
    const int64_t heads = (int64_t)B * Hkv, full = heads * paged_most_cuts(B, Hkv, most, four), slots = paged_slots(heads) + (paged_at_once(heads) ? 0 : heads);
    return (int)(full < slots ? full : slots);
}

bool paged_joins(int B, int Hkv, int G, int64_t most, bool four) { return paged_most_cuts(B, Hkv, most, four) * G <= PAGED_JOIN; }

hipError_t init_paged_kernels() {
    hipError_t e;
    if ((e = init_paged_t<128, CACHE_BF16>()) != hipSuccess || (e = init_paged_t<128, CACHE_E4M3>()) != hipSuccess || (e = init_paged_t<64, CACHE_BF16>()) != hipSuccess) return e;
    if ((e = init_paged_t<64, CACHE_E4M3>()) != hipSuccess) return e;
    return init_paged4_kernels();
}
hipError_t run_paged(const PagedArgs& a, int type, int d, int units, hipStream_t st) {
    if (type == CACHE_E2M1) return run_paged4(a, d, units, st);
    if (type == CACHE_E4M3) return d == 128 ? run_paged_d<128, CACHE_E4M3>(a, units, st) : run_paged_d<64, CACHE_E4M3>(a, units, st);
    return d == 128 ? run_paged_d<128, CACHE_BF16>(a, units, st) : run_paged_d<64, CACHE_BF16>(a, units, st);
}

}  // namespace ls
