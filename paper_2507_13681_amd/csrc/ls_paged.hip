// One new token of each sequence over its pages (ls_paged_attend):
//     out = softmax(scale * q K^T) V   over the first len[b] positions of sequence b's cache.
//
// The step reads every K and V row once and does 4 d FLOP per (query head, key): it is bound by HBM bandwidth, at small sizes by latency.
// The query heads of a KV head are the columns of 16x16x32 products (NH blocks of 16), so that the rows are read once for all of them.
//   Work.  What there is to do follows from the lengths, which only the device knows: every wave adds them up, cuts each KV head's 32-key tiles into parts of about
//   equal length and finds the part that its workgroup has (paged_length, paged_cuts), so a batch of one long and many short sequences fills the chip as one of equals does.
//   A part.  The waves of a workgroup take its tiles in turn.  S^T = K Q^T with K fragments straight from global memory, online softmax per head in a lane,
//   P -> bf16, O^T += V^T P^T with the V^T fragments read transposed from a wave-private, swizzled LDS copy of the 32 V rows that a global -> LDS transfer filled.
//   e4m3: K codes become bf16 with their row's power of two in one instruction for two of them, exactly; V codes come through the 8-bit transpose read and
//   become bf16 as they are, and their rows' powers go into the probabilities, exactly too.
//   The waves' partial results are merged through LDS; where a head is in parts, the workgroup that finishes it last merges those.
// Pages.  A page holds a multiple of 16 positions, so that each half of a tile lies in one: lane l of a wave keeps the page of half l of its next 64, and a
// tile's two are lane reads.  What lies behind the length in the last page is read with it, and left out by selects; a half in no page at all is read from page 0 and left out.
#include "ls_device.h"
#include "ls_internal.h"

namespace ls {

constexpr int PG_WAVES = 8, PG_THREADS = 64 * PG_WAVES, PG_BATCH = 8;

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
        if (E4M3) return D == 128 ? (row & 7) : ((row >> 1) & 3);
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
__device__ __forceinline__ float power_of_byte(uint32_t w, int i) { return __builtin_bit_cast(float, (w >> (8 * i) & 0xFFu) << 23); }

template <int D, int NH, bool E4M3>
__global__ __launch_bounds__(PG_THREADS) void paged_kernel(PagedArgs a) {
    using C = PagedCfg<D, E4M3>;
    using T = bf16_t;
    constexpr int PS = C::PS;
    extern __shared__ __align__(16) unsigned char pg_lds[];    // a V stage per wave; later the waves' partial results
    __shared__ int last_s;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m16 = lane & 15, q = lane >> 4;
    const int G = a.G, page_log = a.cache.page_log;
    auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };

    // ---- which part of which head this workgroup has
    const int64_t room = (int64_t)a.cache.max_pages << page_log, most = a.most < room ? a.most : room;
    auto length_of = [&](int b) -> int {                       // of sequence b, as far as it can be
        const int n = b < a.B ? a.len[b] : 0;
        return n < 0 ? 0 : n < most ? n : (int)most;
    };
    auto tiles_of = [](int n) { return (int)(((uint32_t)n + PAGED_TILE - 1) / PAGED_TILE); };
    int n_lane = length_of(lane);                              // of the 64 sequences at hand
    int64_t tiles = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        if (b0) n_lane = length_of(b0 + lane);
        const uint32_t s = lanes_upto((uint32_t)tiles_of(n_lane));                // (64 sequences of 2^31 keys are 2^32 tiles: counted one bit short of that)
        tiles += (uint32_t)__builtin_amdgcn_readlane((int)s, 63);
    }
    const int length = paged_length(tiles, a.Hkv);
    int b = -1, kvh = 0, cut = 0, cuts = 0, n = 0, before = 0;
    for (int b0 = 0; b0 < a.B && b < 0; b0 += 64) {
        if (a.B > 64) n_lane = length_of(b0 + lane);
        const int mine = b0 + lane < a.B ? paged_cuts(tiles_of(n_lane), length) * a.Hkv : 0;
        const int upto = before + (int)lanes_upto((uint32_t)mine);
        const uint64_t in = __ballot((int)blockIdx.x < upto);
        if (in != 0ull) {
            const int l = __builtin_ctzll(in);
            b = b0 + l;
            n = __builtin_amdgcn_readlane(n_lane, l);
            const int units = __builtin_amdgcn_readlane(mine, l), at = (int)blockIdx.x - (__builtin_amdgcn_readlane(upto, l) - units);
            cuts = units / a.Hkv;
            kvh = uniform(at / cuts);
            cut = at - kvh * cuts;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    if (b < 0) return;                                         // (all waves of the workgroup alike)
    cuts = uniform(cuts); cut = uniform(cut); n = uniform(n);
    const int bk = b * a.Hkv + kvh;
    if (cut == 0 && kvh == 0 && tid == 0 && a.len[b] > most) atomicOr(a.status, STAT_PAGE_RANGE);
    const int all = tiles_of(n), each = (all + cuts - 1) / cuts;
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
    const int vbase = vrow * C::RB + 8 * (m16 & 1);
    const int vslot = E4M3 ? 0 : (m16 >> 1) & 1;               // 16-byte slot inside block i's bytes

    for (; t < tend; t += PG_WAVES) {
        wait_transfers();                                              // this tile's rows are here (the same wave reads them)
        const int left = n - PAGED_TILE * t;                           // keys of the tile that exist
        const bool whole = left >= PAGED_TILE && hf[0].on && hf[1].on;
        if (!whole) {                                                  // the V rows of masked keys meet weight 0: make them finite
#pragma unroll
            for (int i = 0; i < C::NIV; ++i)
                if (C::RPI * i + trow >= left || !hf[C::RPI * i / 16].on) *reinterpret_cast<f32x4*>(stage + i * 1024 + 16 * lane) = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        bf16x8 kf[2][C::KC];
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int c = 0; c < C::KC; ++c) {
                if constexpr (E4M3) {
                    const uint4 w = __builtin_bit_cast(uint4, kr[e][c / 2]);
                    kf[e][c] = c % 2 ? bf16_of(w.z, w.w, power_of_byte(kx[e], 0)) : bf16_of(w.x, w.y, power_of_byte(kx[e], 0));
                } else {
                    kf[e][c] = __builtin_bit_cast(bf16x8, kr[e][c]);
                }
            }
        f32x4 s[NH][2];
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                s[h][e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < C::KC; ++c)                        // s[h][e][r] = <k_{16 e + 4 q + r}, q_{head 16 h + m16}>
                    s[h][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[e][c], qf[h][c], s[h][e], 0, 0, 0);
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
                for (int r = 0; r < 8; ++r) x[r] = whole || x[r] > 0.f ? x[r] * vp[r] : 0.f;        // (behind the length the bytes may be anything)
            }
            Frag<T> f;
            pack_frag(f, x);                                           // contraction index 8 q + r <-> key 16 (r / 4) + 4 q + r % 4
            pf[h] = f.v;
        }
#pragma unroll
        for (int i = 0; i < C::DB; ++i) {
            Frag<T> vf;
            if constexpr (E4M3) {
                const i32x2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32((i32x2 __attribute__((address_space(3)))*)(stage + vbase + 16 * (i ^ C::vswz(vrow))));
                vf.v = bf16_of((uint32_t)w.x, (uint32_t)w.y, 1.0f);
            } else {
                const unsigned char* va = stage + vbase + 16 * ((2 * i + vslot) ^ C::vswz(vrow));      // vswz(vrow + 16) is the same
                load_frag_tr(vf, va, va + 16 * C::RB);
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
    auto finish = [&](int head, int dd, float m, float o0, float o1, float l) {   // two output elements (dd == 0 also writes lse)
        *reinterpret_cast<uint32_t*>(out + head * D + dd) = (uint32_t)f2bf(l > 0.f ? o0 / l : 0.f) | ((uint32_t)f2bf(l > 0.f ? o1 / l : 0.f) << 16);
        if (lse && dd == 0) lse[head] = l > 0.f ? (m * sc2 + log2f(l)) * 0.69314718055994531f : -INFINITY;
    };
    float* shared_part = a.part + (int64_t)(blockIdx.x - cut) * G * PS;           // [part][head][PS]
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
        put_shared2(dst + dd, o0, o1);
        if (dd == 0) put_shared2(dst + D, m, l);
    }
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
                if (s < cuts && mh[s].x > -INFINITY) {
                    const float wgt = fast_exp2((mh[s].x - m) * sc2);
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

// A head's tiles are at most all there are: t / paged_length(t * Hkv ..) <= PAGED_WORKERS / Hkv, whatever t is.
int paged_most_cuts(int Hkv, int64_t most) {
    const int64_t tiles = (most + PAGED_TILE - 1) / PAGED_TILE, by_work = (PAGED_WORKERS + Hkv - 1) / Hkv, by_tiles = paged_cuts((int)tiles, 4);
    return (int)(by_work < by_tiles ? by_work : by_tiles);
}
int paged_units(int B, int Hkv, int64_t most) {
    // heads x cuts: at most one each beside the PAGED_WORKERS that the whole is cut into, and no more than all of the longest would be
    const int64_t heads = (int64_t)B * Hkv, full = heads * paged_most_cuts(Hkv, most);
    return (int)(full < heads + PAGED_WORKERS ? full : heads + PAGED_WORKERS);
}

template <int D, int NH, bool E4M3>
static size_t paged_smem_t(int G, int cuts) {
    using C = PagedCfg<D, E4M3>;
    const size_t stages = (size_t)PG_WAVES * C::V_BYTES;
    const size_t merge = (size_t)PG_WAVES * G * C::PS * 4;
    const size_t parts = cuts == 1 ? 0 : 2 * (size_t)G * cuts * 4 + 4 * (size_t)PG_THREADS * 4;
    const size_t m = stages > merge ? stages : merge;
    return m > parts ? m : parts;
}
template <int D, int NH, bool E4M3>
static hipError_t run_paged_t(const PagedArgs& a, int units, hipStream_t st) {
    const size_t smem = paged_smem_t<D, NH, E4M3>(a.G, paged_most_cuts(a.Hkv, a.most));
    hipLaunchKernelGGL((paged_kernel<D, NH, E4M3>), dim3(units), dim3(PG_THREADS), smem, st, a);
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
