// Sequences of a paged cache that grow and shrink (ls_cache_resize): pages from and to a ring of free ones, block tables, and of the rows that a step adds their
// packed starts, positions and slots.
//
// Everything follows from prefix sums over the sequences: of the rows that they add, of the pages that they need and of those that they give back.  A workgroup has 1024 sequences at a time, one a
// thread, and every workgroup of a launch adds up all of them by itself (8 bytes a sequence, from the caches) rather than wait for another to do it; pages and rows are shared out among the
// workgroups evenly, however unevenly the sequences have them, and which sequence one is of is found by bisecting the sums in LDS.  How many workgroups there are goes by the rows that a call has room
// for, which is what the host knows: a step of up to 1024 rows has one (in place 8192), whatever comes back, and moves 1000 pages in a us.  (Contexts that end in a step of few rows, us: 24 of 512 pages 11.6, 64 of 512 27, 512 of
// 2048 1032.)
// Nobody waits for anybody: pages that are taken are read where those that are given back in the same call are not written, table entries that are read (of positions that were there) are none of those
// that are written, and where lengths or the ring's state are updated in place by more than one workgroup, a launch of one more does that behind the others.
// Bound by its launch and a chain of dependent loads (lengths, then pages, then rows), and of many sequences by the sums.  A decode step in place, us: 4 sequences 3.9, 256 4.6, 1024 5.6, 4096 17, 65535 (of one KV head) 292 (they
// come 1024 at a time); without starts, of 4 to 4096, 3.8, 3.8, 4.6, 13.4; sixteen sequences that grow by 23900 rows in all 4.7; 512 by 1.04 million rows 10.7 (13 MB: 2.5 of them).
#include "ls_rows.h"

namespace ls {

// Sum over the lanes to the left and this one, of values of less than 2^32
__device__ __forceinline__ int64_t lanes_upto64(uint32_t x) {
    if (__ballot(x >> 26 != 0u) == 0ull) return (int64_t)lanes_upto(x);
    return (int64_t)lanes_upto(x & 0xFFFFu) + ((int64_t)lanes_upto(x >> 16) << 16);
}
// .. in a row of 16 lanes
__device__ __forceinline__ uint32_t row_upto(uint32_t x) {
    int32_t s = (int32_t)x;
    s += __builtin_amdgcn_update_dpp(0, s, 0x111, 0xF, 0xF, false);       // row_shr:1, 2, 4, 8
    s += __builtin_amdgcn_update_dpp(0, s, 0x112, 0xF, 0xF, false);
    s += __builtin_amdgcn_update_dpp(0, s, 0x114, 0xF, 0xF, false);
    s += __builtin_amdgcn_update_dpp(0, s, 0x118, 0xF, 0xF, false);
    return (uint32_t)s;
}

constexpr int RESIZE_WAVES = 16, RESIZE_THREADS = 64 * RESIZE_WAVES, RESIZE_ALONE = 8 * RESIZE_THREADS;

template <bool PACKED>
__global__ __launch_bounds__(RESIZE_THREADS, 8) void resize_kernel(ResizeArgs a) {
    constexpr int WAVES = RESIZE_WAVES, THREADS = RESIZE_THREADS, MANY = 0x7FFFFFFF;
    enum { GIVE, TAKE, ROWS };
    __shared__ int64_t waves_s[3][WAVES], given_s;
    __shared__ int upto_s[3][THREADS];                         // sums up to and with each of the sequences: of pages that come back, pages that go, rows; MANY: of no account
    __shared__ int old_s[THREADS], from_s[THREADS];            // positions that it had, -1: it does not grow; and its first page that comes or goes
    __shared__ int fits_s, taken_s;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const bool first = blockIdx.x == 0;
    const int64_t room = (int64_t)a.max_pages << a.page_log, most = room < MANY ? room : MANY;
    auto pages_of = [&](int64_t n) { return (int)((n + (1 << a.page_log) - 1) >> a.page_log); };
    int head = a.state[0], count = a.state[1], odd = 0, bad = 0;
    if (head < 0 || head >= a.pages || count < 0 || count > a.pages) { odd = STAT_PAGE_RANGE; head = count = 0; }
    auto ring = [&](int from, int i) {                         // entry i of those from `from` on (both less than `pages`)
        const uint32_t at = (uint32_t)from + (uint32_t)i;
        return at < (uint32_t)a.pages ? at : at - (uint32_t)a.pages;
    };
    const int spare = a.pages - count;                         // entries of the ring that hold nothing, ..
    const int tail = spare ? (int)ring(head, count) : head;    // .. from this one on
    const int64_t step = (int64_t)gridDim.x * THREADS, me = (int64_t)blockIdx.x * THREADS + tid;
    int turn = blockIdx.x;                                     // (of few pages and rows another workgroup's each time)
    // the sum up to and with this lane's sequence, of which `mine` are this wave's, and that of all
    auto join = [&](int which, int64_t mine, int64_t& all) {
        const int64_t w = waves_s[which][lane % WAVES];        // (less than 2^38)
        int64_t before, sum;
        if (__ballot(w >> 28 != 0) == 0ull) {
            const uint32_t s = row_upto((uint32_t)w);
            before = wv ? (uint32_t)__builtin_amdgcn_readlane((int)s, wv - 1) : 0u;              // (up to 2^32: lanes are read as int, which would be negative here)
            sum = (uint32_t)__builtin_amdgcn_readlane((int)s, WAVES - 1);
        } else {
            const uint32_t lo = row_upto((uint32_t)w & 0xFFFFFFu), hi = row_upto((uint32_t)(w >> 24));
            auto at = [&](int l) { return (int64_t)__builtin_amdgcn_readlane((int)lo, l) + ((int64_t)__builtin_amdgcn_readlane((int)hi, l) << 24); };
            before = wv ? at(wv - 1) : 0;
            sum = at(WAVES - 1);
        }
        const int64_t upto = all + before + mine;
        all += sum;
        return upto;
    };
    int64_t rows0 = 0, need0 = 0, give0 = 0;                   // sums over the sequences so far
    int fits0 = 0, taken0 = 0;                                 // rows of those that have room, pages of those that got some
    int len1 = tid < a.B ? a.len[tid] : 0, add1 = tid < a.B ? a.add[tid] : 0;
    for (int b0 = 0; b0 < a.B; b0 += THREADS) {
        const int here = a.B - b0 < THREADS ? a.B - b0 : THREADS, b = b0 + tid, old = len1, add = add1;
        len1 = b + THREADS < a.B ? a.len[b + THREADS] : 0;     // (asked for ahead; nobody but this thread writes them)
        add1 = b + THREADS < a.B ? a.add[b + THREADS] : 0;
        const bool live = 64 * wv < here;                      // waves without a sequence leave the instructions to the others
        const bool ok = old >= 0 && old <= most, shrinks = ok && add < 0;
        const int64_t sum = (int64_t)old + add, now = sum < 0 ? 0 : sum, give1 = give0;
        const int fits1 = fits0, taken1 = taken0;
        // ---- sums
        int64_t r = 0, g = 0, d = 0, rows_to = 0, give_to = 0;
        if (live) {
            r = lanes_upto64(add > 0 ? (uint32_t)add : 0u);
            g = lanes_upto64(shrinks ? (uint32_t)(pages_of(old) - pages_of(now)) : 0u);
        }
        if (tid == 0) fits_s = taken_s = 0;
        if (lane == 63) { waves_s[ROWS][wv] = r; waves_s[GIVE][wv] = g; }
        __syncthreads();
        if (live) {
            rows_to = join(ROWS, r, rows0);
            give_to = join(GIVE, g, give0);
            if (tid == 0) given_s = give0;
        }
        const bool fits = PACKED ? rows_to <= a.n_rows : add <= a.n_rows, wants = ok && add > 0 && fits && now <= most;
        const int need = wants ? pages_of(now) - pages_of(old) : 0;
        if (live) d = lanes_upto64((uint32_t)need);
        if (lane == 63) waves_s[TAKE][wv] = d;
        __syncthreads();
        bool grows = false;
        if (live) {
            const int64_t need_to = join(TAKE, d, need0);
            grows = wants && (need == 0 || need_to <= count);
            if (!ok || (add > 0 && fits && now > most)) odd |= STAT_PAGE_RANGE;
            if (add > 0 && !fits) odd |= STAT_STARTS;
            if (wants && !grows) odd |= STAT_PAGES_OUT;
            // how far rows and pages go: the sums rise, so that those which are of account are the first ones
            const uint64_t fit = __ballot(PACKED && fits), got = __ballot(need > 0 && grows);
            if (fit && lane == 63 - __builtin_clzll(fit)) atomicMax(&fits_s, (int)rows_to);
            if (got && lane == 63 - __builtin_clzll(got)) atomicMax(&taken_s, (int)need_to);
            upto_s[TAKE][tid] = need_to <= count ? (int)need_to : MANY;
            old_s[tid] = grows ? old : -1;
            from_s[tid] = pages_of(shrinks ? now : old);
        } else {
            upto_s[TAKE][tid] = MANY;
        }
        upto_s[ROWS][tid] = !PACKED ? (grows ? add : 0) : live && fits ? (int)rows_to : MANY;            // (padded: how many are its own)
        upto_s[GIVE][tid] = live && give_to < MANY ? (int)give_to : MANY;
        __syncthreads();
        fits0 = fits_s > fits0 ? fits_s : fits0;
        taken0 = taken_s > taken0 ? taken_s : taken0;
        give0 = given_s;
        if (a.finish && first && tid < here) {
            if (PACKED) a.starts[b + 1] = fits ? (int)rows_to : fits0;
            a.new_len[b] = grows || shrinks ? (int)now : old;
        }
        if (a.bulk) {
            // ---- the pages and rows of these sequences, one behind the other: whose one is, its number there, and the page number that it is about, which lies in
            // the ring or in the table
            const int64_t gives = (give0 < spare ? give0 : spare) - give1, n_give = gives > 0 ? gives : 0, n_take = taken0 - taken1;
            const int64_t items = n_give + n_take + (!a.positions && !a.slots ? 0 : PACKED ? fits0 - fits1 : here * a.n_rows);
            int top = 1;
            while (top < here) top *= 2;
            for (int64_t y = (int64_t)turn * THREADS + tid; y < items; y += step) {
                const int kind = y < n_give ? GIVE : y < n_give + n_take ? TAKE : ROWS, before = kind == GIVE ? (int)give1 : kind == TAKE ? taken1 : PACKED ? fits1 : 0;
                const int x = (int)(before + y - (kind == GIVE ? 0 : kind == TAKE ? n_give : n_give + n_take));
                const int* upto = upto_s[kind];
                int t = 0;
                if (!PACKED && kind == ROWS) t = x / a.n_rows;
                else for (int s = top / 2; s > 0; s /= 2) t += upto[t + s - 1] <= x ? s : 0;           // (entries behind the last sequence are all there is, which is more than x)
                const int i = x - (!PACKED && kind == ROWS ? t * a.n_rows : t ? upto[t - 1] : before), from = from_s[t];
                if (kind == ROWS) {
                    const int64_t at = PACKED ? x : (int64_t)b0 * a.n_rows + x;
                    const int had = PACKED || i < upto[t] ? old_s[t] : -1;
                    int64_t slot = -1;
                    const int p = had < 0 ? 0 : had + i, nth = p >> a.page_log;
                    if (had >= 0 && a.slots) {
                        const int page = *(nth < from ? a.table + (int64_t)(b0 + t) * a.max_pages + nth : a.free + ring(head, (t ? upto_s[TAKE][t - 1] : taken1) + nth - from));
                        if ((uint32_t)page < (uint32_t)a.pages) slot = ((int64_t)page << a.page_log) + (p & ((1 << a.page_log) - 1));
                        else bad = STAT_PAGE_RANGE;
                    }
                    if (a.positions) a.positions[at] = p;
                    if (a.slots) a.slots[at] = slot;
                } else {
                    int32_t* const entry = a.table + (int64_t)(b0 + t) * a.max_pages + from + i;
                    int32_t* const place = a.free + (kind == GIVE ? ring(tail, x) : ring(head, x));
                    const int page = *(kind == GIVE ? entry : place);
                    *(kind == GIVE ? place : entry) = page;
                }
            }
        }
        turn = turn ? turn - 1 : gridDim.x - 1;
        if (b0 + THREADS < a.B) __syncthreads();
    }
    if (a.bulk && PACKED)                                      // rows of no sequence
        for (int64_t x = fits0 + me; x < a.n_rows; x += step) {
            if (a.positions) a.positions[x] = 0;
            if (a.slots) a.slots[x] = -1;
        }
    if (give0 > spare) odd |= STAT_PAGE_RANGE;
    if (a.finish && first) {
        if (tid == 0) {
            if (PACKED) a.starts[0] = 0;
            const int given = give0 < spare ? (int)give0 : spare;
            a.new_state[0] = ring(head, taken0);
            a.new_state[1] = count - taken0 + given;
        }
        bad |= odd;
    }
    if (bad) atomicOr(a.status, bad);
}

hipError_t run_resize(ResizeArgs a, hipStream_t st) {
    const bool in_place = a.new_len == a.len || a.new_state == a.state;
    const int64_t rows = a.starts ? a.n_rows : (int64_t)a.B * a.n_rows, groups = (rows + RESIZE_THREADS - 1) / RESIZE_THREADS;
    // In place one workgroup does it alone up to here: a launch more takes 3 us.  (64 sequences that grow and shrink in turn, us, alone / in two launches: 2048 rows 5.3 / 8.5, 4096 5.9 / 8.7, 8192 7.8 / 8.0 to 9.0, 16384 12.3 / 8.9.)
    const int grid = in_place && rows <= RESIZE_ALONE ? 1 : groups < 256 ? (int)groups : 256;
    a.bulk = 1;
    a.finish = grid == 1 || !in_place;
    auto launch = [&](int n) {
        if (a.starts) hipLaunchKernelGGL((resize_kernel<true>), dim3(n), dim3(RESIZE_THREADS), 0, st, a);
        else hipLaunchKernelGGL((resize_kernel<false>), dim3(n), dim3(RESIZE_THREADS), 0, st, a);
    };
    launch(grid);
    if (!a.finish) {
        a.bulk = 0; a.finish = 1;
        launch(1);
    }
    return hipGetLastError();
}

}  // namespace ls
