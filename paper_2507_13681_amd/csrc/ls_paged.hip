// One new token of each sequence over its pages (ls_paged_attend):
//     out = softmax(scale * q K^T) V   over the first len[b] positions of sequence b's cache.
//
// The step reads every K and V row once and does 4 d FLOP per (query head, key): it is bound by HBM bandwidth, at small sizes by latency.
// The query heads of a KV head are the columns of 16x16x32 products (NH blocks of 16), so that the rows are read once for all of them.
//   Work.  What there is to do follows from the lengths, which only the device knows: every wave adds them up, cuts each KV head's 32-key tiles into parts of about
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
#include "ls_device.h"
#include "ls_internal.h"

namespace ls {

constexpr int PG_WAVES = 8, PG_THREADS = 64 * PG_WAVES, PG_BATCH = 8;
// Parts x query heads that the last workgroup of a head puts together itself; it reads their results alone, 30 to 50 KB a us.  Itself / by a launch more, us: 32 x 4 96.7 / 97.0, 8 x 8 31.1 / 32.9,
// 17 x 8 12.2 / 13.4, 128 x 8 15.2 / 12.4, 128 x 32 48 / 13, 256 x 32 158 / 23.
constexpr int PAGED_JOIN = 320;

template <int D, bool E4M3>
struct PagedCfg {
    static constexpr int RB = D * (E4M3 ? 1 : 2);         // bytes per row
    static constexpr int DS = RB / 16;                    // 16-byte slots per row
    static constexpr int RPI = 64 / DS;                   // rows per transfer instruction
    static constexpr int NIV = PAGED_TILE / RPI;          // transfers per V tile
    static constexpr int V_BYTES = PAGED_TILE * RB;       // one wave's V stage
    static constexpr int KC = D / 32;                     // 32-wide contraction chunks of a row
    static constexpr int KL = RB / 64;                    // 16-byte loads of a lane for a key (a key's row is four lanes')
    static constexpr int DB = D / 16;                     // 16-wide output blocks
    static constexpr int PS = D + 4;                      // floats of a partial result: output, reference, normaliser, 2 unused
    // slot swizzle of the staged V rows (XOR on the 16-byte slot index): the rows a transpose read touches fall into different banks
    __device__ static constexpr int vswz(int row) {
        if (E4M3) return D == 128 ? ((row ^ row >> 4) & 7) : ((row >> 1 ^ (row >> 4 & 1)) & 3);
        return D == 128 ? 2 * (row & 7) : 2 * ((row >> 1) & 3);
    }
};

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) int i32x2;
__device__ __forceinline__ bf16x8 bf16_of(uint32_t lo, uint32_t hi, float f) {      // eight e4m3 codes times the power of two f
    struct U { bf16x2 v[4]; } u = {{__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, f, true),
                                    __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, f, true)}};
    return __builtin_bit_cast(bf16x8, u);
}
// Byte i of w as the scale of a conversion, which looks at the exponent alone (0: 2^-127, 255: the result is NaN), ..
__device__ __forceinline__ float scale_of_byte(uint32_t w, int i) { return __builtin_bit_cast(float, (w >> (8 * i) & 0xFFu) << 23); }
// .. and as a number, which that of the code of one is (0 and 255 as bits of a float would be zero and infinity)
__device__ __forceinline__ float power_of_byte(uint32_t w, int i) { return __builtin_amdgcn_cvt_scalef32_f32_fp8(0x38, scale_of_byte(w, i), 0); }

__device__ __forceinline__ int paged_tiles(int n) { return (int)(((uint32_t)n + PAGED_TILE - 1) / PAGED_TILE); }

// The units of a call, as the lengths have them: a lane has a sequence of the 64 at hand.  Of those the ones with the longest parts come first, so that the short ones
// fill what these leave.
struct PagedUnits {
    int b, kvh, cut, cuts, n; // sequence, KV head, part, parts of the head, length
    int base;                 // first unit of the head
    int64_t most;             // no sequence is longer
    __device__ int length_of(const PagedArgs& a, int i) const {                // of sequence i, as far as it can be
        const int x = i < a.B ? a.len[i] : 0;
        return x < 0 ? 0 : x < most ? x : (int)most;
    }
    // f(lane of the sequence in order, parts, units up to and with it, lane of it): called for 64 sequences after the other until it returns true
    template <typename F>
    __device__ bool walk(const PagedArgs& a, int lane, F f) {
        const int64_t room = (int64_t)a.cache.max_pages << a.cache.page_log;
        most = a.most < room ? a.most : room;
        int x = length_of(a, lane);
        int64_t tiles = 0;
        for (int b0 = 0; b0 < a.B; b0 += 64)                   // (64 sequences of 2^31 keys have less than 2^32 tiles)
            tiles += (uint32_t)__builtin_amdgcn_readlane((int)lanes_upto((uint32_t)paged_tiles(b0 ? length_of(a, b0 + lane) : x)), 63);
        PagedLength l(tiles * a.Hkv, (int64_t)a.B * a.Hkv);
        if (a.B > 64) l.length = l.enough;
        int before = 0;
        for (int b0 = 0; b0 < a.B; b0 += 64) {
            if (b0) x = length_of(a, b0 + lane);
            const int here = a.B - b0 < 64 ? a.B - b0 : 64, t = paged_tiles(x);
            int c, upto;
            do {
                c = lane < here ? 1 : 0;
                if (__ballot(t > PAGED_WHOLE) != 0ull && lane < here) c = paged_cuts(t, l.length);
                upto = before + (int)lanes_upto((uint32_t)(c * a.Hkv));
            } while (!l.accepts(__builtin_amdgcn_readlane(upto, 63)));
            int lane_in = lane;
            const int each = c ? (t + c - 1) / c : -1;
            if (l.sorts && a.B <= 64 && __ballot(lane < here && each != __builtin_amdgcn_readfirstlane(each)) != 0ull) {
                int rank = lane < here ? 0 : lane;             // how many come before this lane's
                for (int i = 0; i < here; ++i) {
                    const int o = __builtin_amdgcn_readlane(each, i);
                    rank += lane < here && (o > each || (o == each && i < lane)) ? 1 : 0;
                }
                c = __builtin_amdgcn_ds_permute(4 * rank, c);
                lane_in = __builtin_amdgcn_ds_permute(4 * rank, lane);
                upto = before + (int)lanes_upto((uint32_t)(c * a.Hkv));
            }
            if (f(b0, x, c, lane_in, upto)) return true;
            before = __builtin_amdgcn_readlane(upto, 63);
        }
        return false;
    }
    __device__ bool find(const PagedArgs& a, int unit, int lane) {
        auto u = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
        return walk(a, lane, [&](int b0, int x, int c, int l, int upto) {
            const uint64_t in = __ballot(unit < upto);
            if (in == 0ull) return false;
            const int at = __builtin_ctzll(in);
            const int seq = __builtin_amdgcn_readlane(l, at);
            cuts = u(__builtin_amdgcn_readlane(c, at));
            b = u(b0 + seq);
            n = u(__builtin_amdgcn_readlane(x, seq));
            const int i = unit - (__builtin_amdgcn_readlane(upto, at) - cuts * a.Hkv);
            kvh = u(i / cuts);
            cut = u(i - kvh * cuts);
            base = unit - cut;
            return true;
        });
    }
    __device__ bool find_head(const PagedArgs& a, int seq, int head, int lane) {       // the parts of one KV head
        return walk(a, lane, [&](int b0, int x, int c, int l, int upto) {
            const uint64_t in = __ballot(b0 + l == seq);
            if (in == 0ull || seq < b0 || seq >= b0 + 64) return false;
            const int at = __builtin_ctzll(in);
            cuts = __builtin_amdgcn_readfirstlane(__builtin_amdgcn_readlane(c, at));
            b = seq; kvh = head; cut = 0;
            base = __builtin_amdgcn_readfirstlane(__builtin_amdgcn_readlane(upto, at) - cuts * a.Hkv + head * cuts);
            return true;
        });
    }
};

template <int D, int NH, bool E4M3>
__global__ __launch_bounds__(PG_THREADS, NH == 1 ? 4 : 2) void paged_kernel(PagedArgs a) {
    using C = PagedCfg<D, E4M3>;
    using T = bf16_t;
    constexpr int PS = C::PS;
    extern __shared__ __align__(16) unsigned char pg_lds[];    // a V stage per wave; later the waves' partial results
    __shared__ int last_s;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m16 = lane & 15, q = lane >> 4;
    const int G = a.G, page_log = a.cache.page_log;

    // ---- which part of which head this workgroup has
    PagedUnits w;
    if (!w.find(a, (int)blockIdx.x, lane)) return;             // (all waves of the workgroup alike)
    const int b = w.b, kvh = w.kvh, cut = w.cut, cuts = w.cuts, n = w.n;
    const int bk = b * a.Hkv + kvh;
    if (cut == 0 && kvh == 0 && tid == 0 && a.len[b] > w.most) atomicOr(a.status, STAT_PAGE_RANGE);
    const int all = paged_tiles(n), each = (all + cuts - 1) / cuts;
    const int tile0 = cut * each, tend = tile0 + each < all ? tile0 + each : all;

    unsigned char* stage = pg_lds + wv * C::V_BYTES;
    const uint32_t stage_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)stage;
    // ---- pages: lane l has that of half l & 1 of this wave's tile t0 + 8 (l / 2); -1: nowhere
    int pages = -1, t0 = tile0 + wv;
    auto ask_pages = [&](int t) {
        t0 = t;
        const int64_t key = (int64_t)PAGED_TILE * (t + PG_WAVES * (lane >> 1)) + 16 * (lane & 1);
        pages = key < n ? page_of(a.cache, b, key) : -1;
        if (key < n && pages < 0) atomicOr(a.status, STAT_PAGE_RANGE);
    };
    const int64_t head = (int64_t)kvh << page_log;
    const int in_page = (1 << page_log) - 1;
    struct Half { int64_t row; bool on; };                     // first row of a half of a tile, as rows of the pool
    auto half_at = [&](int t, int h) -> Half {
        const int p = __builtin_amdgcn_readlane(pages, ((t - t0) / PG_WAVES) * 2 + h);
        return Half{((int64_t)(p < 0 ? 0 : p) * a.cache.Hkv << page_log) + head + ((PAGED_TILE * t + 16 * h) & in_page), p >= 0};
    };
    const int trow = lane / C::DS, sl = lane % C::DS;          // a transfer: this lane fills slot sl of tile row RPI * i + trow
    auto request_v = [&](const Half (&hf)[2]) {
#pragma unroll
        for (int i = 0; i < C::NIV; ++i) {
            const int r0 = C::RPI * i, row = r0 + trow;
            const unsigned char* base = a.cache.v + (hf[r0 / 16].row + (r0 & 15)) * C::RB;
            dma16(uniform_ptr(base), (uint32_t)(trow * C::RB + 16 * (sl ^ C::vswz(row))), stage_lds + (uint32_t)(i * 1024));
        }
    };
    f32x4 kr[2][C::KL];                                        // keys m16 and 16 + m16 of the tile: bytes 64 j + 16 q .. of the row
    uint32_t kx[2], vx[2];                                     // e4m3: the exponent of key 16 h + m16 of K, of keys 16 h + 4 q .. + 3 of V
    auto request_k = [&](const Half (&hf)[2]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const unsigned char* krow = a.cache.k + (hf[h].row + m16) * C::RB + 16 * q;
#pragma unroll
            for (int j = 0; j < C::KL; ++j) kr[h][j] = *reinterpret_cast<const f32x4*>(krow + 64 * j);
            if constexpr (E4M3) {
                kx[h] = a.cache.kx[hf[h].row + m16];
                vx[h] = *reinterpret_cast<const uint32_t*>(a.cache.vx + hf[h].row + 4 * q);
            }
        }
    };
    int t = tile0 + wv;
    Half hf[2], hn[2];
    ask_pages(t);
    if (t < tend) {
        hf[0] = half_at(t, 0); hf[1] = half_at(t, 1);
        request_v(hf);
        request_k(hf);
    }
    // ---- the queries.  Chunk c of a row: values 32 c + 8 q .., or for e4m3, whose 16-byte loads have two chunks' values, 64 (c / 2) + 16 q + 8 (c % 2) ..
    bf16x8 qf[NH][C::KC];                                      // head 16 h + m16 of the group
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int c = 0; c < C::KC; ++c) {
            const f32x4 z = {0.f, 0.f, 0.f, 0.f};
            qf[h][c] = __builtin_bit_cast(bf16x8, z);
            const int at = E4M3 ? 64 * (c / 2) + 16 * q + 8 * (c % 2) : 32 * c + 8 * q;
            if (16 * h + m16 < G)
                qf[h][c] = *reinterpret_cast<const bf16x8*>(reinterpret_cast<const T*>(a.q) + ((int64_t)b * a.Hq + kvh * G + 16 * h + m16) * D + at);
        }
    f32x4 oacc[NH][C::DB];                                     // O^T: element r of block i is d = 16 i + 4 q + r of head m16
    float m_run[NH], l_run[NH];                                // reference in raw logit units; this lane's share of the normaliser
#pragma unroll
    for (int h = 0; h < NH; ++h) {
        m_run[h] = -INFINITY; l_run[h] = 0.f;
#pragma unroll
        for (int i = 0; i < C::DB; ++i) oacc[h][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const float sc2 = a.scale_log2e;
    // transpose reads.  16 bit: in a block of 16 lanes lane s points at key 4 q + s / 4 (+ 16) and value 4 (s % 4) of block i, and receives four keys of
    // column d = 16 i + s.  8 bit: lane s points at key 16 (s / 8) + 4 q + s / 2 % 4 and value 8 (s % 2), and receives the eight keys.
    const int vrow = E4M3 ? 16 * (m16 >> 3) + 4 * q + ((m16 >> 1) & 3) : 4 * q + (m16 >> 2);
    // of block 0; block i's differs in the bits of its slot (kept as one value: the addresses of all blocks would be eight registers)
    int vat = vrow * C::RB + 16 * (C::vswz(vrow) + (E4M3 ? 0 : (m16 >> 1) & 1)) + 8 * (m16 & 1);

    for (; t < tend; t += PG_WAVES) {
        wait_transfers();                                              // this tile's rows are here (the same wave reads them)
        const int left = n - PAGED_TILE * t;                           // keys of the tile that exist
        const bool whole = left >= PAGED_TILE && hf[0].on && hf[1].on;
        if (!whole) {                                                  // the V rows of masked keys meet weight 0: make them finite
#pragma unroll
            for (int i = 0; i < C::NIV; ++i)
                if (C::RPI * i + trow >= left || !hf[C::RPI * i / 16].on) *reinterpret_cast<f32x4*>(stage + i * 1024 + 16 * lane) = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        f32x4 s[NH][2];
#pragma unroll
        for (int h = 0; h < NH; ++h) s[h][0] = s[h][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int c = 0; c < C::KC; ++c) {
                bf16x8 kf;
                if constexpr (E4M3) {
                    const uint4 w = __builtin_bit_cast(uint4, kr[e][c / 2]);
                    kf = c % 2 ? bf16_of(w.z, w.w, scale_of_byte(kx[e], 0)) : bf16_of(w.x, w.y, scale_of_byte(kx[e], 0));
                } else {
                    kf = __builtin_bit_cast(bf16x8, kr[e][c]);
                }
#pragma unroll
                for (int h = 0; h < NH; ++h)                           // s[h][e][r] = <k_{16 e + 4 q + r}, q_{head 16 h + m16}>
                    s[h][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[h][c], s[h][e], 0, 0, 0);
            }
        float vp[8];                                                   // the powers of V's rows
        if constexpr (E4M3) {
#pragma unroll
            for (int r = 0; r < 8; ++r) vp[r] = power_of_byte(vx[r >> 2], r & 3);
        }
        const bool more = t + PG_WAVES < tend;
        if (more) {
            if ((t + PG_WAVES - t0) / PG_WAVES >= 32) { ask_pages(t + PG_WAVES); wait_transfers(); }
            hn[0] = half_at(t + PG_WAVES, 0); hn[1] = half_at(t + PG_WAVES, 1);
            request_k(hn);
        }
        bf16x8 pf[NH];
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            float x[8], mx = -INFINITY;
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                x[r] = s[h][r >> 2][r & 3];
                if (!whole) x[r] = 16 * (r >> 2) + 4 * q + (r & 3) < left && hf[r >> 2].on ? x[r] : -INFINITY;
                mx = fmaxf(mx, x[r]);
            }
            mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            const float m_new = fmaxf(m_run[h], mx);
            const bool seen = m_new > -INFINITY;                       // (halves that are nowhere: perhaps no key yet)
            const float corr = seen ? fast_exp2((m_run[h] - m_new) * sc2) : 1.f;
            const float mneg = seen ? -m_new * sc2 : 0.f;
            m_run[h] = m_new;
            float ps = 0.f;
#pragma unroll
            for (int r = 0; r < 8; ++r) { x[r] = fast_exp2(__builtin_fmaf(x[r], sc2, mneg)); ps += x[r]; }
            l_run[h] = l_run[h] * corr + ps;
            if (__ballot(corr != 1.0f) != 0ull) {
#pragma unroll
                for (int i = 0; i < C::DB; ++i) oacc[h][i] *= corr;
            }
            if constexpr (E4M3) {
#pragma unroll
                for (int r = 0; r < 8; ++r) x[r] = whole || (16 * (r >> 2) + 4 * q + (r & 3) < left && hf[r >> 2].on) ? x[r] * vp[r] : 0.f;        // (behind the length the bytes may be anything)
            }
            Frag<T> f;
            pack_frag(f, x);                                           // contraction index 8 q + r <-> key 16 (r / 4) + 4 q + r % 4; bf16 as the products with V take it, not in the normaliser
            pf[h] = f.v;
        }
        asm volatile("" : "+v"(vat));
#pragma unroll
        for (int i = 0; i < C::DB; ++i) {
            Frag<T> vf;
            const unsigned char* va = stage + (vat ^ (E4M3 ? 16 : 32) * i);
            if constexpr (E4M3) {
                const i32x2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32((i32x2 __attribute__((address_space(3)))*)(va));
                vf.v = bf16_of((uint32_t)w.x, (uint32_t)w.y, 1.0f);
            } else {
                load_frag_tr(vf, va, va + 16 * C::RB);                 // vswz(vrow + 16) is the same
            }
#pragma unroll
            for (int h = 0; h < NH; ++h) oacc[h][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf.v, pf[h], oacc[h][i], 0, 0, 0);
        }
        if (more) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // the stage has been read
            request_v(hn);
            hf[0] = hn[0]; hf[1] = hn[1];
        }
    }

    // ---- merge the waves through LDS: part[wv][head][PS]
    wait_transfers();
    __syncthreads();                                                   // every wave is done with its V stage
    float* part = reinterpret_cast<float*>(pg_lds);
#pragma unroll
    for (int h = 0; h < NH; ++h) {
        float l = l_run[h] + __shfl_xor(l_run[h], 16, 64);
        l += __shfl_xor(l, 32, 64);
        if (16 * h + m16 < G) {
            float* mine = part + (wv * G + 16 * h + m16) * PS;
#pragma unroll
            for (int i = 0; i < C::DB; ++i) *reinterpret_cast<f32x4*>(mine + 16 * i + 4 * q) = oacc[h][i];
            if (q == 0) { mine[D] = m_run[h]; mine[D + 1] = l; }
        }
    }
    __syncthreads();
    bf16_t* out = reinterpret_cast<bf16_t*>(a.out) + ((int64_t)b * a.Hq + kvh * G) * D;
    float* lse = a.lse ? a.lse + (int64_t)b * a.Hq + kvh * G : nullptr;
    auto finish = [&](int head, int dd, float m, float o0, float o1, float l) {   // two output elements (dd == 0 also writes lse); l: 0 without a key, NaN where a logit is
        *reinterpret_cast<uint32_t*>(out + head * D + dd) = (uint32_t)f2bf(l != 0.f ? o0 / l : 0.f) | ((uint32_t)f2bf(l != 0.f ? o1 / l : 0.f) << 16);
        if (lse && dd == 0) lse[head] = l != 0.f ? (m * sc2 + log2f(l)) * 0.69314718055994531f : -INFINITY;
    };
    float* shared_part = a.part + (int64_t)w.base * G * PS;           // [part][head][PS]
    const int items = G * (D / 2);                                     // two neighbouring elements of a head
    for (int idx = tid; idx < items; idx += PG_THREADS) {
        const int hd = idx / (D / 2), dd = 2 * (idx % (D / 2));
        float m = -INFINITY, o0 = 0.f, o1 = 0.f, l = 0.f;
        float2 ml[PG_WAVES], x[PG_WAVES];                              // (a wave without a key: reference -inf, zeros)
#pragma unroll
        for (int w = 0; w < PG_WAVES; ++w) {
            const float* pw = part + (w * G + hd) * PS;
            ml[w] = *reinterpret_cast<const float2*>(pw + D);
            x[w] = *reinterpret_cast<const float2*>(pw + dd);
            m = fmaxf(m, ml[w].x);
        }
#pragma unroll
        for (int w = 0; w < PG_WAVES; ++w) {
            const float wgt = ml[w].x > -INFINITY ? fast_exp2((ml[w].x - m) * sc2) : 0.f;
            o0 += x[w].x * wgt; o1 += x[w].y * wgt;
            l += ml[w].y * wgt;
        }
        if (cuts == 1) { finish(hd, dd, m, o0, o1, l); continue; }
        float* dst = shared_part + ((int64_t)cut * G + hd) * PS;
        if (!a.done) {                                                 // paged_join_kernel's
            *reinterpret_cast<float2*>(dst + dd) = make_float2(o0, o1);
            if (dd == 0) *reinterpret_cast<float2*>(dst + D) = make_float2(m, l);
            continue;
        }
        put_shared2(dst + dd, o0, o1);
        if (dd == 0) put_shared2(dst + D, m, l);
    }
    if (!a.done) return;
    if (blockIdx.x == 0)                                               // whatever an earlier call has left there
        for (int h = tid; h < a.clear_heads; h += PG_THREADS) clear_shared(a.done_clear + h);
    if (cuts == 1) return;

    // ---- the last workgroup of this KV head to get here merges the parts
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                   // this wave's part of the result has been written
    __syncthreads();
    if (tid == 0) {
        last_s = count_shared(a.done + bk) == (uint32_t)cuts - 1u;
        if (last_s) clear_shared(a.done + bk);                         // for the call that uses these counters next
    }
    __syncthreads();
    if (!last_s) return;
    // A thread owns two elements of a head and every `subs`-th part; the subsets are added through LDS.
    const int subs = items >= PG_THREADS ? 1 : PG_THREADS / items;
    float2* ml = reinterpret_cast<float2*>(pg_lds);                    // [head][part] reference, normaliser
    float* add = reinterpret_cast<float*>(pg_lds) + 2 * G * cuts;      // [sub][item][4]
    for (int idx0 = 0; idx0 < items; idx0 += PG_THREADS) {
        const int idx = idx0 + (subs == 1 ? tid : tid % items), sub = subs == 1 ? 0 : tid / items;
        const bool on = idx < items && sub < subs;
        const int hd = on ? idx / (D / 2) : 0, dd = on ? 2 * (idx % (D / 2)) : 0;
        const float* src = shared_part + (int64_t)hd * PS + dd;
        float2 x[PG_BATCH];
        auto fetch = [&](int s0) {
#pragma unroll
            for (int e = 0; e < PG_BATCH; ++e) {
                const int s = s0 + e * subs;
                x[e] = get_shared2(src + (int64_t)(s < cuts ? s : cuts - 1) * G * PS);
            }
        };
        fetch(sub);
        if (idx0 == 0) {
            for (int i = tid; i < G * cuts; i += PG_THREADS) ml[i] = get_shared2(shared_part + ((int64_t)(i % cuts) * G + i / cuts) * PS + D);
            __syncthreads();
        }
        const float2* mh = ml + hd * cuts;
        float m = -INFINITY, o0 = 0.f, o1 = 0.f, l = 0.f;
        for (int s = 0; s < cuts; ++s) m = fmaxf(m, mh[s].x);
        for (int s0 = sub; s0 < cuts; s0 += PG_BATCH * subs) {
            if (s0 != sub) fetch(s0);
#pragma unroll
            for (int e = 0; e < PG_BATCH; ++e) {
                const int s = s0 + e * subs;
                if (s < cuts) {
                    const float wgt = mh[s].x > -INFINITY ? fast_exp2((mh[s].x - m) * sc2) : 0.f;        // (NaN times 0 stays NaN)
                    o0 += x[e].x * wgt; o1 += x[e].y * wgt;
                    l += mh[s].y * wgt;
                }
            }
        }
        if (subs > 1) {
            if (on && sub > 0) { float* p = add + 4 * ((sub - 1) * items + idx); p[0] = o0; p[1] = o1; p[2] = l; }
            __syncthreads();
            if (on && sub == 0)
                for (int u = 1; u < subs; ++u) { const float* p = add + 4 * ((u - 1) * items + idx); o0 += p[0]; o1 += p[1]; l += p[2]; }
        }
        if (on && sub == 0) finish(hd, dd, m, o0, o1, l);
    }
}

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

// A head's tiles are at most all there are, and a part no shorter than these by the slots: t / paged_length(..) <= slots / Hkv, whatever t is.
int paged_most_cuts(int B, int Hkv, int64_t most) {
    const int64_t heads = (int64_t)B * Hkv, tiles = (most + PAGED_TILE - 1) / PAGED_TILE, by_work = (paged_slots(heads) + Hkv - 1) / Hkv;
    const int64_t by_tiles = paged_cuts((int)tiles, paged_at_once(heads) ? PAGED_SHORTEST : PAGED_SHORTEST_MANY);
    return (int)(by_work < by_tiles ? by_work : by_tiles);
}
int paged_units(int B, int Hkv, int64_t most) {
    // no more than the slots, or beside those the head that each part begins; and no more than all heads of the longest would be
    const int64_t heads = (int64_t)B * Hkv, full = heads * paged_most_cuts(B, Hkv, most), slots = paged_slots(heads) + (paged_at_once(heads) ? 0 : heads);
    return (int)(full < slots ? full : slots);
}

bool paged_joins(int B, int Hkv, int G, int64_t most) { return paged_most_cuts(B, Hkv, most) * G <= PAGED_JOIN; }

template <int D, int NH, bool E4M3>
static size_t paged_smem_t(int G, int cuts, bool joins) {
    using C = PagedCfg<D, E4M3>;
    const size_t stages = (size_t)PG_WAVES * C::V_BYTES;
    const size_t merge = (size_t)PG_WAVES * G * C::PS * 4;
    const size_t parts = cuts == 1 || !joins ? 0 : 2 * (size_t)G * cuts * 4 + 4 * (size_t)PG_THREADS * 4;
    const size_t m = stages > merge ? stages : merge;
    return m > parts ? m : parts;
}
template <int D, int NH, bool E4M3>
static hipError_t run_paged_t(const PagedArgs& a, int units, hipStream_t st) {
    size_t smem = paged_smem_t<D, NH, E4M3>(a.G, paged_most_cuts(a.B, a.Hkv, a.most), a.done != nullptr);
    if (a.B * a.Hkv <= PAGED_ALONE && smem <= 80 * 1024) smem = 80 * 1024 + 256;     // (a workgroup a compute unit, and none with two while another has none)
    hipLaunchKernelGGL((paged_kernel<D, NH, E4M3>), dim3(units), dim3(PG_THREADS), smem, st, a);
    if (!a.done) hipLaunchKernelGGL((paged_join_kernel<D>), dim3(a.B * a.Hq), dim3(2 * D), 0, st, a);
    return hipGetLastError();
}
template <int D, bool E4M3>
static hipError_t init_paged_t() {
    const hipError_t e = allow_full_lds(&paged_kernel<D, 1, E4M3>);
    return e != hipSuccess ? e : allow_full_lds(&paged_kernel<D, 2, E4M3>);
}
hipError_t init_paged_kernels() {
    hipError_t e;
    if ((e = init_paged_t<128, false>()) != hipSuccess || (e = init_paged_t<128, true>()) != hipSuccess || (e = init_paged_t<64, false>()) != hipSuccess) return e;
    return init_paged_t<64, true>();
}
template <int D, bool E4M3>
static hipError_t run_paged_d(const PagedArgs& a, int units, hipStream_t st) {
    return a.G <= 16 ? run_paged_t<D, 1, E4M3>(a, units, st) : run_paged_t<D, 2, E4M3>(a, units, st);
}
hipError_t run_paged(const PagedArgs& a, int type, int d, int units, hipStream_t st) {
    if (type) return d == 128 ? run_paged_d<128, true>(a, units, st) : run_paged_d<64, true>(a, units, st);
    return d == 128 ? run_paged_d<128, false>(a, units, st) : run_paged_d<64, false>(a, units, st);
}

}  // namespace ls
