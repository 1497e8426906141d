// Sequences of a paged cache that grow and shrink (ls_cache_resize): pages from and to a ring of free ones, block tables, and of the rows that a step adds their
// packed starts, positions and slots.
//
// Everything follows from prefix sums over the sequences: of the rows that they add, of the pages that they need and of those that they give back.  A workgroup has 1024 sequences at a time, one a
// thread, and every workgroup of a launch adds up all of them by itself (8 bytes a sequence, from the caches) rather than wait for another to do it; pages and rows are shared out among the
// workgroups evenly, however unevenly the sequences have them, and which sequence one is of is found by bisecting the sums in LDS.
// Nobody waits for anybody: pages that are taken are read where those that are given back in the same call are not written, table entries that are read (of positions that were there) are none of those
// that are written, and where lengths or the ring's state are updated in place by more than one workgroup, a launch of one more does that behind the others.
// Bound by its launch and a chain of dependent loads (lengths, then pages, then rows).
#include "ls_rows.h"

namespace ls {

constexpr int RESIZE_THREADS = 1024;

// Sum over the lanes to the left and this one, of values of less than 2^32
__device__ __forceinline__ int64_t lanes_upto64(uint32_t x) {
    return (int64_t)lanes_upto(x & 0xFFFFu) + ((int64_t)lanes_upto(x >> 16) << 16);
}

__global__ __launch_bounds__(RESIZE_THREADS) void resize_kernel(ResizeArgs a) {
    __shared__ int64_t waves_s[3][16];
    __shared__ int rows_s[RESIZE_THREADS], take_s[RESIZE_THREADS], give_s[RESIZE_THREADS];    // sums up to and with each of the sequences; MANY: of no account
    __shared__ int old_s[RESIZE_THREADS], from_s[RESIZE_THREADS];      // positions that it had, -1: it does not grow; and its first page that comes or goes
    __shared__ int fits_s[16], taken_s[16];
    constexpr int MANY = 0x7FFFFFFF;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const bool first = blockIdx.x == 0;
    const int64_t room = (int64_t)a.max_pages << a.page_log, most = room < MANY ? room : MANY;
    auto pages_of = [&](int64_t n) { return (int)((n + (1 << a.page_log) - 1) >> a.page_log); };
    int head = a.state[0], count = a.state[1], odd = 0, bad = 0;
    if (head < 0 || head >= a.pages || count < 0 || count > a.pages) { odd = STAT_PAGE_RANGE; head = count = 0; }
    auto ring = [&](int64_t i) { return (int)(i < a.pages ? i : i < 2 * (int64_t)a.pages ? i - a.pages : i - 2 * (int64_t)a.pages); };        // i < 3 pages
    const int spare = a.pages - count;                         // places of the ring that hold nothing
    const int64_t step = (int64_t)gridDim.x * RESIZE_THREADS, me = (int64_t)blockIdx.x * RESIZE_THREADS + tid;
    int64_t rows0 = 0, need0 = 0, give0 = 0;                   // sums over the sequences so far
    int fits0 = 0, taken0 = 0;                                 // rows of those that have room, pages of those that got some
    for (int b0 = 0; b0 < a.B; b0 += RESIZE_THREADS) {
        const int here = a.B - b0 < RESIZE_THREADS ? a.B - b0 : RESIZE_THREADS, b = b0 + tid;
        const int old = tid < here ? a.len[b] : 0, add = tid < here ? a.add[b] : 0;
        const bool ok = old >= 0 && old <= most, shrinks = ok && add < 0;
        const int64_t sum = (int64_t)old + add, now = sum < 0 ? 0 : sum;
        // ---- sums
        const int64_t r = lanes_upto64(add > 0 ? (uint32_t)add : 0u), g = lanes_upto64(shrinks ? (uint32_t)(pages_of(old) - pages_of(now)) : 0u);
        if (lane == 63) { waves_s[0][wv] = r; waves_s[1][wv] = g; }
        __syncthreads();
        const int64_t give1 = give0;
        int64_t rows_to = rows0 + r, give_to = give0 + g;
        for (int w = 0; w < 16; ++w) {
            if (w < wv) { rows_to += waves_s[0][w]; give_to += waves_s[1][w]; }
            rows0 += waves_s[0][w]; give0 += waves_s[1][w];
        }
        const bool fits = rows_to <= a.n_rows, wants = ok && add > 0 && fits && now <= most;
        const int need = wants ? pages_of(now) - pages_of(old) : 0;
        const int64_t d = lanes_upto64((uint32_t)need);
        if (lane == 63) waves_s[2][wv] = d;
        __syncthreads();
        int64_t need_to = need0 + d;
        for (int w = 0; w < 16; ++w) {
            if (w < wv) need_to += waves_s[2][w];
            need0 += waves_s[2][w];
        }
        const bool grows = wants && (need == 0 || need_to <= count);
        if (!ok || (add > 0 && fits && now > most)) odd |= STAT_PAGE_RANGE;
        if (add > 0 && !fits) odd |= STAT_STARTS;
        if (wants && !grows) odd |= STAT_PAGES_OUT;
        // ---- how far rows and pages go: the sums rise, so that those which are of account are the first ones
        const uint64_t fit = __ballot(fits), got = __ballot(need > 0 && grows);
        if (fit ? lane == 63 - __builtin_clzll(fit) : lane == 0) fits_s[wv] = fit ? (int)rows_to : 0;
        if (got ? lane == 63 - __builtin_clzll(got) : lane == 0) taken_s[wv] = got ? (int)need_to : 0;
        rows_s[tid] = fits ? (int)rows_to : MANY;
        take_s[tid] = need_to <= count ? (int)need_to : MANY;
        give_s[tid] = give_to < MANY ? (int)give_to : MANY;
        old_s[tid] = grows ? old : -1;
        from_s[tid] = pages_of(shrinks ? now : old);
        __syncthreads();
        const int fits1 = fits0, taken1 = taken0;
        for (int w = 0; w < 16; ++w) {
            fits0 = fits_s[w] > fits0 ? fits_s[w] : fits0;
            taken0 = taken_s[w] > taken0 ? taken_s[w] : taken0;
        }
        if (a.finish && first && tid < here) {
            if (a.starts) a.starts[b + 1] = fits ? (int)rows_to : fits0;
            a.new_len[b] = grows || shrinks ? (int)now : old;
        }
        if (a.bulk) {
            // ---- the pages and rows of these sequences: whose one is, and its number there
            auto find = [&](const int* to, int before, int x, int& i) {
                int lo = 0, hi = here - 1;
                while (lo < hi) {
                    const int mid = (lo + hi) >> 1;
                    if (to[mid] > x) hi = mid;
                    else lo = mid + 1;
                }
                i = x - (lo ? to[lo - 1] : before);
                return lo;
            };
            int i;
            const int64_t back = give0 < spare ? give0 : spare;
            for (int64_t x = give1 + me; x < back; x += step) {
                const int t = find(give_s, (int)give1, (int)x, i);
                a.free[ring((int64_t)head + count + x)] = a.table[(int64_t)(b0 + t) * a.max_pages + from_s[t] + i];
            }
            for (int64_t x = taken1 + me; x < taken0; x += step) {
                const int t = find(take_s, taken1, (int)x, i);
                a.table[(int64_t)(b0 + t) * a.max_pages + from_s[t] + i] = a.free[ring(head + x)];
            }
            if (a.positions || a.slots) {
                for (int64_t x = fits1 + me; x < fits0; x += step) {
                    const int t = find(rows_s, fits1, (int)x, i), had = old_s[t], p = had < 0 ? 0 : had + i;
                    if (a.positions) a.positions[x] = p;
                    if (!a.slots) continue;
                    int64_t slot = -1;
                    if (had >= 0) {
                        const int at = p >> a.page_log, have = from_s[t];
                        const int page = at < have ? a.table[(int64_t)(b0 + t) * a.max_pages + at] : a.free[ring((int64_t)head + (t ? take_s[t - 1] : taken1) + at - have)];
                        if ((uint32_t)page < (uint32_t)a.pages) slot = ((int64_t)page << a.page_log) + (p & ((1 << a.page_log) - 1));
                        else bad = STAT_PAGE_RANGE;
                    }
                    a.slots[x] = slot;
                }
            }
        }
        __syncthreads();
    }
    if (a.bulk)                                                // rows of no sequence
        for (int64_t x = fits0 + me; x < a.n_rows; x += step) {
            if (a.positions) a.positions[x] = 0;
            if (a.slots) a.slots[x] = -1;
        }
    if (give0 > spare) odd |= STAT_PAGE_RANGE;
    if (a.finish && first) {
        if (tid == 0) {
            if (a.starts) a.starts[0] = 0;
            const int given = give0 < spare ? (int)give0 : spare;
            a.new_state[0] = ring((int64_t)head + taken0);
            a.new_state[1] = count - taken0 + given;
        }
        bad |= odd;
    }
    if (bad) atomicOr(a.status, bad);
}

hipError_t run_resize(ResizeArgs a, hipStream_t st) {
    const int64_t groups = (a.n_rows + 4 * RESIZE_THREADS - 1) / (4 * RESIZE_THREADS);
    const int grid = groups < 256 ? (int)groups : 256;
    const bool in_place = a.new_len == a.len || a.new_state == a.state;
    a.bulk = 1;
    a.finish = grid == 1 || !in_place;
    hipLaunchKernelGGL(resize_kernel, dim3(grid), dim3(RESIZE_THREADS), 0, st, a);
    if (!a.finish) {
        a.bulk = 0; a.finish = 1;
        hipLaunchKernelGGL(resize_kernel, dim3(1), dim3(RESIZE_THREADS), 0, st, a);
    }
    return hipGetLastError();
}

}  // namespace ls
