// Causal attention of packed sequences (ls_packed_prefill):
//     out[a] = sum_b softmax_b(scale * <q_a, k_b>) v_b,  b <= p_a,
// one pass over the keys with a running softmax reference and normaliser; 4 d FLOP a (query head, query, key), bound by the matrix pipeline.
//
// Rows.  A workgroup (4 waves) owns 128 rows of one KV head, a wave 32, where the G query heads of a query are G neighbouring rows: they share
// their keys, so that a block of 128 rows spans 128 / G positions, its waves end within so many keys of each other, and the masks touch few of its steps.
// (A block of 128 positions of one head waits 48 keys a wave for its last one, a fifth of what 512 positions take.)
// Steps.  32 keys, from barrier to barrier: K and V rows of the next step go global -> LDS while S^T = K Q^T, softmax and O^T += V^T P^T of this one run, from two
// buffers, by the 32x32 products of ls_device.h; bf16 V^T fragments come from the LDS transpose read.  No maximum is looked for on the way: the exponentials are
// taken with the reference as it stands, and where a lane's sum exceeds a limit the step's softmax is done again with its maximum as the reference.
// One sequence of 32768, 32 query and 8 KV heads of 128, bf16: 7.2 to 7.6 ms by card (1.16 to 1.22 PFLOP/s; a library product of 16384^3 reaches 1.33); 32 of 700 188 us; fp32, 4 query heads of 64, 1024, 300 and 37: 22 us.
// Three workgroups a CU at d = 128.  With queries of zeros, the same work, it takes 5.6 ms, and with the softmax left out 6.5: the clock under load counts for more than any one pipeline.
// What a row does not see weighs nothing, whatever it holds, and a row's reference moves for that row alone: of an item that is not cut its result has the same bits whatever its neighbours are.
// (How long parts are, and so the order of the sums of a row in parts, follows from the work of the whole call.)
// Items.  Which item a workgroup has follows from the starts, which only the device knows: a wave's lanes keep a sequence each and add up their blocks, those of the longest
// sequences first where one is long beside the rest, the last block of each first; no launch ahead of this one puts them in order.
#include <algorithm>
#include <type_traits>
#include "ls_device.h"
#include "ls_internal.h"

namespace ls {

constexpr int PK_THREADS = 256;
constexpr int PK_RING_S = 4, PK_RING_P = 2;      // fragments in flight ahead of the products of S, of P V
// The longest item against the mean work of the workgroups that are resident at once, beyond which the sequences are sorted: at its end the call would wait for it.  Sorted / as they come, us, 4 or 8 KV
// heads, the longest sequence the last: 0.15 times 1507 / 1483, 0.3 457 / 442, 0.7 562 / 546, 1.24 207 / 202, 1.27 245 / 277, 1.4 285 / 318, 1.9 177 / 228, 6.7 690 / 711; the first, 1.4 285 / 277.
constexpr float PK_WAITS = 1.25f;
constexpr float PK_LIMIT = 32.f;                 // what a lane's probabilities of a step may sum to

template <typename T, int D>
struct PackCfg {
    static_assert(D == 128 || D == 64, "head dimension");
    static constexpr bool F32 = std::is_same<T, float>::value;
    static constexpr int RB = D * Elem<T>::bytes;         // bytes per row
    static constexpr int DS = RB / 16;                    // 16-byte slots per row
    static constexpr int RPI = 64 / DS;                   // rows per transfer instruction
    static constexpr int NI = PACKED_KEYS / RPI;          // transfers per operand and step
    static constexpr int IPW = NI / 4;                    // ... per wave
    static constexpr int K_ISTR = !F32 && D == 128 ? 1088 : 1024;             // LDS bytes from one K transfer to the next
    static constexpr int K_BYTES = NI * K_ISTR, STEP_BYTES = K_BYTES + NI * 1024;
    static constexpr int OUT_ROW = RB + 16;               // results on their way out: LDS bytes from row to row
    static constexpr int LDS = 2 * STEP_BYTES > PACKED_ROWS * OUT_ROW ? 2 * STEP_BYTES : PACKED_ROWS * OUT_ROW;
    static constexpr int KSTEPS = D / 16, DBLK = D / 32;
    static constexpr int RESIDENT = F32 ? (D == 128 ? 1 : 2) : D == 64 ? 4 : 3;         // workgroups of a CU, at least (fp32 at d = 128 spills with two)
    // slot swizzles (XOR on the 16-byte slot index inside a row), so that fragment reads touch each bank once
    __device__ static constexpr int kswz(int row) { return F32 ? row & 15 : D == 128 ? (row & 3) : (((row >> 1) & 3) | (((row >> 3) & 1) << 2)); }
    __device__ static constexpr int vswz(int row) { return F32 ? row & 15 : D == 128 ? ((row & 3) << 2) : (((row >> 1) & 1) << 2); }
};

__device__ __forceinline__ uint32_t lanes_sum(uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)lanes_upto(x), 63); }

// The sequences, one a lane, and what a workgroup has of them
struct PackedWork {
    PackedSeq seq;            // of sequence `lane` (of 64 at a time), or `index`
    int G, lane, index;
    int q0, k0;               // first rows of sequence `lane` (of 64 at a time; not of `index`), packed
    // the item, its part, and the unit it is
    int s, block, part, length;
    bool stopped = false;     // a sequence before had starts that are none
    __device__ void keep(const PackedArgs& a, int s0) {    // sequences s0 ..
        const int i = s0 + lane;
        bool bad = false;
        seq = PackedSeq{0, 0};
        q0 = k0 = 0;
        if (i < a.B) {
            if (a.q_starts) {
                q0 = a.q_starts[i]; k0 = a.k_starts[i];
                const int32_t q1 = a.q_starts[i + 1], k1 = a.k_starts[i + 1];
                bad = !starts_ok(q0, q1, a.n_hat) || !starts_ok(k0, k1, a.n);
                seq = PackedSeq{k1 - k0, q1 - q0};
            } else {
                seq = PackedSeq{a.n, a.n_hat};
            }
        }
        const uint64_t none = __ballot(bad);
        if (stopped || (none != 0ull && lane >= __builtin_ctzll(none))) seq = PackedSeq{0, 0};
        // Whoever comes upon them says so: one always does, since with starts a KV head has fewer items than workgroups (packed_items), and the ones without an item look at all sequences.
        if (none != 0ull && !stopped && lane == 0) atomicOr(a.status, STAT_STARTS);
        stopped = stopped || none != 0ull;
    }
    __device__ int longer(int x) const { return (int)lanes_sum((uint32_t)packed_longer(seq, G, x)); }
    // the sequences (at most 64) by their longest items, where the longest of all takes so much of what a resident workgroup has to do that the call would wait for it
    __device__ void sort(const PackedArgs& a) {
        if (!((float)longest() * (float)a.sorted > PK_WAITS * wave_sum(packed_work(seq, G)) * (float)a.Hkv)) return;
        const int steps = seq.queries > 0 ? packed_steps(seq, G, packed_blocks(seq.queries, G) - 1) : -1;
        if (__ballot(lane < a.B && steps != __builtin_amdgcn_readfirstlane(steps)) == 0ull) return;
        int rank = lane < a.B ? 0 : lane;
        for (int i = 0; i < a.B; ++i) {
            const int o = __builtin_amdgcn_readlane(steps, i);
            rank += lane < a.B && (o > steps || (o == steps && i < lane)) ? 1 : 0;
        }
        seq.keys = __builtin_amdgcn_ds_permute(4 * rank, seq.keys);
        seq.queries = __builtin_amdgcn_ds_permute(4 * rank, seq.queries);
        index = __builtin_amdgcn_ds_permute(4 * rank, lane);
    }
    // by sequence, however many there are
    __device__ bool find_in_order(const PackedArgs& a, int r) {
        int before = 0;
        for (int s0 = 0; s0 < a.B; s0 += 64) {
            if (s0) keep(a, s0);
            const int mine = packed_blocks(seq.queries, G), upto = before + (int)lanes_upto((uint32_t)mine);
            const uint64_t in = __ballot(r < upto);
            if (in != 0ull) {
                const int l = __builtin_ctzll(in);
                s = s0 + l;                                // (of a call that sorts them: the place)
                block = __builtin_amdgcn_readlane(upto, l) - 1 - r;            // (the last of a sequence first)
                return true;
            }
            before = __builtin_amdgcn_readlane(upto, 63);
        }
        return false;
    }
    __device__ int longest() const {                       // steps of the longest item, or nearly (a float)
        const float most = seq.queries > 0 ? (float)packed_steps(seq, G, packed_blocks(seq.queries, G) - 1) : 0.f;
        return __builtin_amdgcn_readfirstlane((int)wave_largest(most));
    }
    __device__ void cut_length(const PackedArgs& a) {      // steps of a part, of a call that cuts its items
        length = __builtin_amdgcn_readfirstlane(packed_length(a.cut, a.Hkv, wave_sum(packed_work(seq, G)), longer(-1), longest()));
    }
    __device__ int longer_than_part(const PackedSeq& x, int p) const {          // blocks that have a part p
        const int64_t steps = (int64_t)p * length;
        return p == 0 ? packed_longer(x, G, -1) : steps > 1 << 28 ? 0 : packed_longer(x, G, (int)steps);
    }
    // blocks that have a part p0 + lane (and in *before those of the sequences before `stop`)
    __device__ int having(const PackedArgs& a, int p0, int stop = 0, int* before = nullptr) const {
        int sum = 0;
        for (int i = 0; i < a.B; ++i) {
            if (before && i == stop) *before = sum;
            const PackedSeq x{__builtin_amdgcn_readlane(seq.keys, i), __builtin_amdgcn_readlane(seq.queries, i)};
            if (x.queries > 0) sum += longer_than_part(x, p0 + lane);
        }
        return sum;
    }
    // Units of a KV head go by part, those of a part by sequence, the last block of each first: unit r is ..  (All run at once, so that the order does not matter.)
    __device__ bool find_part(const PackedArgs& a, int r) {
        cut_length(a);
        int before = 0;
        part = -1;
        for (int p0 = 0; part < 0; p0 += 64) {
            const int mine = having(a, p0), upto = before + (int)lanes_upto((uint32_t)mine);
            const uint64_t in = __ballot(r < upto);
            if (in != 0ull) {
                const int l = __builtin_ctzll(in);
                part = p0 + l;
                r -= __builtin_amdgcn_readlane(upto - mine, l);
            } else if (__builtin_amdgcn_readlane(mine, 63) == 0) {
                return false;
            }
            before = __builtin_amdgcn_readlane(upto, 63);
        }
        const int upto = (int)lanes_upto((uint32_t)longer_than_part(seq, part));
        s = __builtin_ctzll(__ballot(r < upto));
        block = packed_blocks(__builtin_amdgcn_readlane(seq.queries, s), G) - 1 - (r - (s > 0 ? __builtin_amdgcn_readlane(upto, s - 1) : 0));          // (the longest first)
        return true;
    }
};

template <typename T, int D>
__global__ __launch_bounds__(PK_THREADS, (PackCfg<T, D>::RESIDENT)) void packed_kernel(PackedArgs a) {
    using C = PackCfg<T, D>;
    extern __shared__ __align__(16) unsigned char pk_lds[];              // [2][K rows, V rows]; later the results on their way out
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)pk_lds;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r32 = lane & 31, g = lane >> 5;
    auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
    auto apart = [](int x) { asm volatile("" : "+v"(x)); return __builtin_amdgcn_readfirstlane(x); };      // a condition that is not joined with others
    const int G = a.G;

    // ---- the item.  Workgroups go round the XCDs: those of one keep to one KV head, or to an eighth of them
    PackedWork w;
    w.G = G; w.lane = lane; w.part = 0; w.length = 1 << 28; w.s = 0; w.block = 0;
    w.keep(a, 0);
    int kvh, rank;
    {
        const int u = blockIdx.x, x = u & 7, i = u >> 3;
        if (8 % a.Hkv == 0) { const int per = 8 / a.Hkv; kvh = x / per; rank = i * per + x % per; }
        else if (a.Hkv % 8 == 0) { kvh = x + 8 * (i % (a.Hkv / 8)); rank = i / (a.Hkv / 8); }
        else { kvh = u % a.Hkv; rank = u / a.Hkv; }
    }
    w.index = lane;
    if (a.sorted) w.sort(a);
    if (!(a.cut.units ? w.find_part(a, rank) : w.find_in_order(a, rank))) return;
    const int sl64 = uniform(w.s) & 63, s = a.sorted ? __builtin_amdgcn_readlane(w.index, sl64) : uniform(w.s), block = uniform(w.block);
    const int nk = __builtin_amdgcn_readlane(w.seq.keys, sl64), nq = __builtin_amdgcn_readlane(w.seq.queries, sl64);
    // (loaded again from the starts they would be waited for once more)
    const int64_t q0 = __builtin_amdgcn_readlane(w.q0, s & 63), k0 = __builtin_amdgcn_readlane(w.k0, s & 63), pad = a.q_starts ? 0 : s;
    const int steps = packed_steps(PackedSeq{nk, nq}, G, block);
    const int length = uniform(w.length), h0 = uniform(w.part) * length, h1 = steps - h0 > length ? h0 + length : steps;         // steps of this part
    const bool cut = steps > length;
    // rows
    const int64_t rows = (int64_t)nq * G, rho0 = (int64_t)PACKED_ROWS * block + 32 * wv;
    const bool rows_here = rho0 < rows;
    const int64_t rho = rho0 + r32;
    const bool on = rho < rows;
    const int qi = (int)((on ? (uint32_t)rho : 0u) / (uint32_t)G), hd = kvh * G + (int)(on ? (uint32_t)rho : 0u) - qi * G;
    const uint32_t rho_end = (uint32_t)(rho0 + 31 < rows ? rho0 + 31 : rows - 1);
    const int pos_most = rows_here ? nk - nq + uniform((int)(rho_end / (uint32_t)G)) : -1;
    const int pos = on ? nk - nq + qi : pos_most;          // last key that this lane's row sees (one that does not exist has zeros for a query, and finite results)

    const unsigned char* Kg = uniform_ptr(a.k.data + (pad * a.k.seq + k0 * a.k.row + (int64_t)kvh * a.k.head) * Elem<T>::bytes);
    const unsigned char* Vg = uniform_ptr(a.v.data + (pad * a.v.seq + k0 * a.v.row + (int64_t)kvh * a.v.head) * Elem<T>::bytes);
    Frag<T> qf[C::KSTEPS];
    if (on) {
        const unsigned char* qrow = a.q.data + (pad * a.q.seq + (q0 + qi) * a.q.row + (int64_t)hd * a.q.head) * Elem<T>::bytes;
#pragma unroll
        for (int c = 0; c < C::KSTEPS; ++c) load_frag(qf[c], qrow + (16 * c + 8 * g) * Elem<T>::bytes);
    } else {
#pragma unroll
        for (int c = 0; c < C::KSTEPS; ++c) zero_frag(qf[c]);
    }

    // ---- transfers: this lane fills slot sl of row rowlane + RPI i of a step and fetches the chunk that the swizzle assigns to that slot
    const int rowlane = C::IPW * C::RPI * wv + lane / C::DS, sl = lane % C::DS;
    const uint32_t kstride = (uint32_t)(a.k.row * Elem<T>::bytes), vstride = (uint32_t)(a.v.row * Elem<T>::bytes);
    uint32_t kat[C::IPW], vat[C::IPW];
#pragma unroll
    for (int i = 0; i < C::IPW; ++i) {
        const int row = rowlane + C::RPI * i;
        kat[i] = (uint32_t)row * kstride + 16u * (uint32_t)(sl ^ C::kswz(row));
        vat[i] = (uint32_t)row * vstride + 16u * (uint32_t)(sl ^ C::vswz(row));
    }
    const uint32_t kdst0 = lds0 + (uint32_t)(wv * C::IPW * C::K_ISTR), vdst0 = lds0 + (uint32_t)(C::K_BYTES + wv * C::IPW * 1024);
    const unsigned char *ka = Kg, *va = Vg;
    uint32_t to = 0u;
    auto aim = [&](int h) {
        ka = Kg + (uint64_t)(uint32_t)h * PACKED_KEYS * kstride;
        va = Vg + (uint64_t)(uint32_t)h * PACKED_KEYS * vstride;
        to = (uint32_t)(h & 1) * (uint32_t)C::STEP_BYTES;
    };
    auto send = [&](int i) {                               // of 2 IPW transfers
        const int j = i / 2;
        if (i & 1) dma16(va, vat[j], vdst0 + to + (uint32_t)(j * 1024));
        else dma16(ka, kat[j], kdst0 + to + (uint32_t)(j * C::K_ISTR));
    };
    auto fetch = [&](int h) {                              // a whole step; rows behind the last key repeat it (they are masked: finite is enough)
        aim(h);
        const int last = nk - 1 - PACKED_KEYS * h;
        if (last >= PACKED_KEYS - 1) {
#pragma unroll
            for (int i = 0; i < 2 * C::IPW; ++i) send(i);
            return;
        }
#pragma unroll
        for (int i = 0; i < C::IPW; ++i) {
            const int row = rowlane + C::RPI * i, r = row <= last ? row : last;
            dma16(ka, (uint32_t)r * kstride + 16u * (uint32_t)(sl ^ C::kswz(row)), kdst0 + to + (uint32_t)(i * C::K_ISTR));
            dma16(va, (uint32_t)r * vstride + 16u * (uint32_t)(sl ^ C::vswz(row)), vdst0 + to + (uint32_t)(i * 1024));
        }
    };

    // ---- fragment reads
    constexpr int KA = C::F32 ? 1 : D == 128 ? 2 : 4;
    int kaddr[KA];
    if constexpr (!C::F32) {                               // chunk 2 c + g of key r32 sits in slot (2 c + g) ^ kswz
        const int x = C::kswz(r32), krow = r32 / C::RPI * C::K_ISTR + r32 % C::RPI * C::RB;
#pragma unroll
        for (int j = 0; j < KA; ++j) kaddr[j] = krow + 32 * (j ^ (x >> 1)) + 16 * (g ^ (x & 1));
    }
    auto kload = [&](Frag<T>& f, const unsigned char* base, int c) {           // key r32, values 16 c + 8 g ..
        if constexpr (C::F32) {
            const unsigned char* row = base + r32 * C::RB;
            const f32x4 x = *reinterpret_cast<const f32x4*>(row + 16 * ((4 * c + 2 * g) ^ C::kswz(r32)));
            const f32x4 y = *reinterpret_cast<const f32x4*>(row + 16 * ((4 * c + 2 * g + 1) ^ C::kswz(r32)));
#pragma unroll
            for (int e = 0; e < 4; ++e) { f.v[e] = x[e]; f.v[4 + e] = y[e]; }
        } else {
            load_frag(f, base + kaddr[c & (KA - 1)] + 32 * (c & ~(KA - 1)));
        }
    };
    int vaddr[C::DBLK];
    if constexpr (!C::F32) {                               // key 4 g + L16 / 4 (+ 8), 64-byte block i
        const int L16 = lane & 15, beta = (lane >> 4) & 1, lrow = 4 * g + (L16 >> 2), y = C::vswz(lrow) >> 2;
#pragma unroll
        for (int i = 0; i < C::DBLK; ++i) vaddr[i] = C::K_BYTES + lrow * C::RB + 64 * (i ^ y) + 32 * beta + 8 * (L16 & 3);
    }
    auto vload = [&](Frag<T>& f, const unsigned char* base, int k) {           // keys 16 (k / DBLK).., output block k % DBLK
        const int half = k / C::DBLK, i = k % C::DBLK;
        if constexpr (C::F32) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int row = 16 * half + 8 * (e / 4) + 4 * g + e % 4;
                f.v[e] = *reinterpret_cast<const float*>(base + C::K_BYTES + row * C::RB + 16 * ((8 * i + r32 / 4) ^ C::vswz(row)) + 4 * (r32 & 3));
            }
        } else {
            const unsigned char* at = base + vaddr[i] + 16 * half * C::RB;
            load_frag_tr(f, at, at + 8 * C::RB);
        }
    };
    // Weights on their way to fragments: of bf16 inputs they become bf16, half a step of 2^-8 each, as the matrix instruction takes them beside V (fp32 products have a sixteenth of its rate);
    // the normaliser adds them up as they were.
    struct Probs {
        std::conditional_t<C::F32, float, uint32_t> w[C::F32 ? 16 : 8];
        __device__ void set(int r, float lo, float hi) {   // registers r, r + 1
            if constexpr (C::F32) { w[r] = lo; w[r + 1] = hi; }
            else {
                typedef __attribute__((ext_vector_type(2))) float f32x2;
                typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
                uint32_t u = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
                asm volatile("" : "+v"(u));                // here, and not where it is used
                w[r / 2] = u;
            }
        }
        __device__ Frag<T> frag(int h) const {
            Frag<T> f;
            if constexpr (C::F32) {
#pragma unroll
                for (int e = 0; e < 8; ++e) f.v[e] = w[8 * h + e];
            } else {
                struct U { uint32_t w[4]; } u = {w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]};
                f.v = __builtin_bit_cast(bf16x8, u);
            }
            return f;
        }
    };

    // ---- a step
    f32x16 oacc[C::DBLK];
#pragma unroll
    for (int i = 0; i < C::DBLK; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[i][r] = 0.f;
    const float sc2 = a.scale_log2e;
    float mneg = INFINITY, l_run = 0.f;  // the softmax reference of this lane's row in base 2, negated (+inf: no key seen yet); its share of the normaliser
    constexpr int NS = C::KSTEPS, NV = 2 * C::DBLK;
    constexpr int RS = PK_RING_S < NS ? PK_RING_S : NS, RV = PK_RING_P;
    // Where some rows do not see all of a step's keys, an infinity or NaN in V must not reach those with weight zero: they are taken out of the fragments (`odd`: there were any), ..
    auto only_finite = [](Frag<T>& f, uint32_t& odd) {
        if constexpr (C::F32) {
#pragma unroll
            for (int e = 0; e < 8; ++e) { const bool is = fabsf(f.v[e]) < INFINITY; odd |= is ? 0u : 1u; f.v[e] = is ? f.v[e] : 0.f; }
        } else {
            typedef __attribute__((ext_vector_type(2))) short s16x2;
            struct U { uint32_t w[4]; } u = __builtin_bit_cast(U, f.v);
#pragma unroll
            for (int e = 0; e < 4; ++e) {                  // an exponent of ones carries into the sign
                const s16x2 up = (__builtin_bit_cast(s16x2, u.w[e] & 0x7F807F80u) + s16x2{0x80, 0x80}) >> 15;
                const uint32_t is = __builtin_bit_cast(uint32_t, up);
                odd |= is;
                u.w[e] &= ~is;
            }
            f.v = __builtin_bit_cast(bf16x8, u);
        }
    };
    // .. and what a row sees of them is added by its kind: how many of each it sees is one more product
    auto ones = [](auto is) {                              // a fragment of ones and zeros
        Frag<T> f;
        if constexpr (C::F32) {
#pragma unroll
            for (int e = 0; e < 8; ++e) f.v[e] = is(e) ? 1.f : 0.f;
        } else {
            struct U { uint32_t w[4]; } u;
#pragma unroll
            for (int e = 0; e < 4; ++e) { u.w[e] = (is(2 * e) ? 0x3F80u : 0u) | (is(2 * e + 1) ? 0x3F800000u : 0u); asm volatile("" : "+v"(u.w[e])); }
            f.v = __builtin_bit_cast(bf16x8, u);
        }
        return f;
    };
    auto add_odd = [&](const unsigned char* base, int last) {                // last: key of the step that the lane's row sees at most
#pragma unroll
        for (int i = 0; i < C::DBLK; ++i)
#pragma unroll 1
            for (int kind = 0; kind < 3; ++kind) {         // +inf, -inf, NaN
                const float what = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : NAN;
                f32x16 c = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    Frag<T> f;
                    vload(f, base, half * C::DBLK + i);
                    f = ones([&](int e) { const float x = (float)f.v[e]; return kind < 2 ? x == what : x != x; });
                    mma(c, f, ones([&](int e) { return 16 * half + 8 * (e / 4) + 4 * g + e % 4 <= last; }));
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) oacc[i][r] += c[r] > 0.f ? what : 0.f;
            }
    };
    auto process = [&](auto SENDS, auto MASKED, int h) {
        constexpr int SN = decltype(SENDS)::value;
        constexpr bool masked = decltype(MASKED)::value;
        const unsigned char* base = pk_lds + (h & 1) * C::STEP_BYTES;
        f32x16 x = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        Frag<T> kf[NS];
#pragma unroll
        for (int c = 0; c < RS; ++c) kload(kf[c], base, c);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c = 0; c < NS; ++c) {
            mma(x, kf[c], qf[c]);                          // x[r] = <k_{8(r/4)+4g+r%4}, q_row>
            if (c + RS < NS) kload(kf[c + RS], base, c + RS);
            if constexpr (SN > 0) {
#pragma unroll
                for (int i = c * SN / NS; i < (c + 1) * SN / NS; ++i) send(i);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (masked) {
            const int lim = pos - PACKED_KEYS * h - 4 * g;
#pragma unroll
            for (int r = 0; r < 16; ++r) x[r] = 8 * (r / 4) + r % 4 <= lim ? x[r] : -INFINITY;
        }
        Frag<T> vf[NV];
#pragma unroll
        for (int k = 0; k < RV; ++k) vload(vf[k], base, k);                      // ahead of the softmax
        Probs pr;
        float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
            const float e0 = fast_exp2(__builtin_fmaf(x[r], sc2, mneg)), e1 = fast_exp2(__builtin_fmaf(x[r + 1], sc2, mneg));
            sum0 += e0; sum1 += e1;
            pr.set(r, e0, e1);
        }
        float sum = sum0 + sum1;
        const uint64_t again = __ballot(!(sum <= PK_LIMIT));                     // lanes whose reference has to move; without one yet the sum is infinite or none
        if (apart(again != 0ull)) {                        // with a new reference for their rows; the others' stays, so that no row's result depends on its neighbours'
            float mx = -INFINITY;
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, x[r]);
            mx = fmaxf(mx, xor32(mx)) * sc2;
            const float m_new = (again >> r32 | again >> (r32 + 32)) & 1ull ? fmaxf(mx, -mneg) : -mneg;
            const bool seen = m_new > -INFINITY;
            const float corr = seen ? fast_exp2(-mneg - m_new) : 1.f, safe = seen ? -m_new : 0.f;
            mneg = -m_new;
            l_run *= corr;
#pragma unroll
            for (int i = 0; i < C::DBLK; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) oacc[i][r] *= corr;
            sum0 = 0.f; sum1 = 0.f;                        // (added up in the same order, for the lanes whose reference stays)
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                const float e0 = fast_exp2(__builtin_fmaf(x[r], sc2, safe)), e1 = fast_exp2(__builtin_fmaf(x[r + 1], sc2, safe));
                sum0 += e0; sum1 += e1;
                pr.set(r, e0, e1);
                if (r % 4 == 2) __builtin_amdgcn_sched_barrier(0);
            }
            sum = sum0 + sum1;
        }
        l_run += sum;
        __builtin_amdgcn_sched_barrier(0);
        uint32_t odd = 0u;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if constexpr (masked) only_finite(vf[k], odd);
            mma(oacc[k % C::DBLK], vf[k], pr.frag(k / C::DBLK));
            if (k + RV < NV) vload(vf[k + RV], base, k + RV);
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (masked) {
            if (apart(__ballot(odd != 0u) != 0ull)) add_odd(base, pos - PACKED_KEYS * h);
        }
    };

    if (h0 < h1) {
        fetch(h0);
        wait_transfers();
        __syncthreads();
        int h = h0;
        // As long as all rows of the workgroup see all keys of a step, and the next step lies inside the keys, whose transfers go out between the products of this one
        const int least = nk - nq + uniform((int)((uint32_t)(PACKED_ROWS * block) / (uint32_t)G)), clear = least < 0 ? 0 : (least + 1) / PACKED_KEYS;
        const int inside = (nk / PACKED_KEYS < h1 ? nk / PACKED_KEYS : h1) - 1, plain = clear < inside ? clear : inside;
        for (; h < plain; ++h) {
            aim(h + 1);
            if (rows_here) process(std::integral_constant<int, 2 * C::IPW>{}, std::false_type{}, h);
            if (apart(rows_here) == 0) {
#pragma unroll
                for (int i = 0; i < 2 * C::IPW; ++i) send(i);
            }
            wait_transfers();
            __syncthreads();
        }
        for (; h < h1; ++h) {
            if (h + 1 < h1) fetch(h + 1);
            if (PACKED_KEYS * h <= pos_most) process(std::integral_constant<int, 0>{}, std::true_type{}, h);
            wait_transfers();
            __syncthreads();
        }
    }

    float l_tot = l_run + xor32(l_run);
    if (cut) {
        if (!rows_here) return;
        float* o = a.part_o + (int64_t)blockIdx.x * (PACKED_ROWS * D) + wv * (C::DBLK * 4 * 256) + lane * 4;
#pragma unroll
        for (int i = 0; i < C::DBLK; ++i)
#pragma unroll
            for (int rq = 0; rq < 4; ++rq)
                *reinterpret_cast<f32x4*>(o + (i * 4 + rq) * 256) = f32x4{oacc[i][4 * rq], oacc[i][4 * rq + 1], oacc[i][4 * rq + 2], oacc[i][4 * rq + 3]};
        if (lane < 32) reinterpret_cast<float2*>(a.part_ml)[(int64_t)blockIdx.x * PACKED_ROWS + 32 * wv + lane] = make_float2(-mneg, l_tot);
        return;
    }
    if (!rows_here) return;
    const float inv = l_tot != 0.f ? 1.0f / l_tot : 0.f;                     // 0 without a key, NaN where a logit is
    if (a.lse && g == 0 && on)
        a.lse[(a.q_starts ? (int64_t)hd * a.n_hat + q0 : ((int64_t)s * a.Hq + hd) * a.n_hat) + qi] =
            l_tot != 0.f ? (log2f(l_tot) - mneg) * 0.69314718055994531f : -INFINITY;
    // A lane holds four neighbouring values of its row at a time; through LDS (32 rows of this wave in the buffers, which nobody reads any more) they become whole rows
    unsigned char* ow = pk_lds + wv * (32 * C::OUT_ROW);
#pragma unroll
    for (int i = 0; i < C::DBLK; ++i)
#pragma unroll
        for (int rq = 0; rq < 4; ++rq) {
            unsigned char* dst = ow + r32 * C::OUT_ROW + (32 * i + 8 * rq + 4 * g) * Elem<T>::bytes;
            const f32x4 y = {oacc[i][4 * rq] * inv, oacc[i][4 * rq + 1] * inv, oacc[i][4 * rq + 2] * inv, oacc[i][4 * rq + 3] * inv};
            if constexpr (C::F32) *reinterpret_cast<f32x4*>(dst) = y;
            else *reinterpret_cast<__attribute__((ext_vector_type(4))) __bf16*>(dst) = __builtin_convertvector(y, __attribute__((ext_vector_type(4))) __bf16);
        }
    __builtin_amdgcn_wave_barrier();
    unsigned char* og = a.out.data + (pad * a.out.seq + q0 * a.out.row + (int64_t)kvh * G * a.out.head) * Elem<T>::bytes;
    const int cr = lane / C::DS, cs = lane % C::DS;
    // the query and head of the lane's row, and from one store to the next RPI rows on
    uint32_t i = (uint32_t)(rho0 + cr) / (uint32_t)G, e = (uint32_t)(rho0 + cr) - i * (uint32_t)G;
    const uint32_t more_i = (uint32_t)C::RPI / (uint32_t)G, more_e = (uint32_t)C::RPI % (uint32_t)G;
#pragma unroll
    for (int j = 0; j < 32 / C::RPI; ++j) {
        const int r = C::RPI * j + cr;
        const f32x4 y = *reinterpret_cast<const f32x4*>(ow + r * C::OUT_ROW + 16 * cs);
        if (rho0 + r < rows) *reinterpret_cast<f32x4*>(og + ((int64_t)i * a.out.row + (int64_t)e * a.out.head) * Elem<T>::bytes + 16 * cs) = y;
        i += more_i; e += more_e;
        if (e >= (uint32_t)G) { e -= (uint32_t)G; ++i; }
    }
}

// The parts of items put together: for each item 4 waves' rows x blocks of 32 output values, a workgroup for one after the other, a wave of it for every fourth part.
constexpr int PK_JOIN_GROUPS = 1024;
template <typename T, int D>
__global__ __launch_bounds__(256) void packed_join_kernel(PackedArgs a) {
    using C = PackCfg<T, D>;
    constexpr int SUBS = 4, NB = 4;                        // subsets of parts, parts in flight
    __shared__ f32x4 red[SUBS][4][64];
    __shared__ float2 red_ml[SUBS][32];
    const int tid = threadIdx.x, lane = tid & 63;
    const int sub = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r32 = lane & 31, g = lane >> 5, G = a.G;
    PackedWork w;
    w.G = G; w.lane = lane; w.s = 0; w.block = 0;
    w.keep(a, 0);
    w.cut_length(a);
    if (w.length == 1 << 28) return;                       // there are none
    constexpr int PER = 4 * C::DBLK;
    const int items = w.longer(-1) * a.Hkv;
    for (int64_t at = blockIdx.x; at < (int64_t)items * PER; at += gridDim.x) {
    const int item = (int)(at / PER), wv = (int)(at % PER) / C::DBLK, i = (int)(at % PER) % C::DBLK;        // item, wave whose rows these are, output block
    const int kvh = item % a.Hkv;
    w.find_in_order(a, item / a.Hkv);
    const int s = __builtin_amdgcn_readfirstlane(w.s), block = __builtin_amdgcn_readfirstlane(w.block);
    const int nk = __builtin_amdgcn_readlane(w.seq.keys, s), nq = __builtin_amdgcn_readlane(w.seq.queries, s);
    const int64_t rows = (int64_t)nq * G, rho0 = (int64_t)PACKED_ROWS * block + 32 * wv;
    const int steps = packed_steps(PackedSeq{nk, nq}, G, block);
    const int parts = (steps + w.length - 1) / w.length;
    if (rho0 >= rows || parts <= 1) continue;
    f32x4 acc[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[k] = f32x4{0.f, 0.f, 0.f, 0.f};
    float M = -INFINITY, L = 0.f;
    int before = 0;                                        // units of the parts before those at hand
    for (int p0 = 0; p0 < parts; p0 += 64) {
        int ahead = 0;                                     // of the part of a lane: units of the sequences before this one
        const int mine = w.having(a, p0, s, &ahead), upto = before + (int)lanes_upto((uint32_t)mine);
        // this block's unit of the part of a lane (packed_kernel), and which workgroup that was
        const int rank = upto - mine + ahead + packed_blocks(nq, G) - 1 - block;
        int unit;
        if (8 % a.Hkv == 0) { const int per = 8 / a.Hkv; unit = rank / per * 8 + kvh * per + rank % per; }
        else if (a.Hkv % 8 == 0) unit = (rank * (a.Hkv / 8) + kvh / 8) * 8 + kvh % 8;
        else unit = rank * a.Hkv + kvh;
        unit = unit < a.cut.units ? unit : a.cut.units - 1;
        const int here = parts - p0 < 64 ? parts - p0 : 64;
        for (int e0 = sub; e0 < here; e0 += SUBS * NB) {
            float2 ml[NB];
            f32x4 x[NB][4];
#pragma unroll
            for (int e = 0; e < NB; ++e) {
                const int u = __builtin_amdgcn_readlane(unit, e0 + e * SUBS < here ? e0 + e * SUBS : e0);
                ml[e] = reinterpret_cast<const float2*>(a.part_ml)[(int64_t)u * PACKED_ROWS + 32 * wv + r32];
                const float* o = a.part_o + (int64_t)u * (PACKED_ROWS * D) + wv * (C::DBLK * 4 * 256) + i * 4 * 256 + lane * 4;
#pragma unroll
                for (int k = 0; k < 4; ++k) x[e][k] = *reinterpret_cast<const f32x4*>(o + k * 256);
            }
            float m_new = M;
#pragma unroll
            for (int e = 0; e < NB; ++e) m_new = fmaxf(m_new, ml[e].x);
            const float corr = M > -INFINITY ? fast_exp2(M - m_new) : 0.f;
            M = m_new;
            L *= corr;
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[k] *= corr;
#pragma unroll
            for (int e = 0; e < NB; ++e) {
                if (e0 + e * SUBS >= here) break;          // (part e0 once more: with a weight of 0 its infinities would become NaN)
                const float wgt = ml[e].x > -INFINITY ? fast_exp2(ml[e].x - M) : 0.f;
                L += ml[e].y * wgt;
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[k] += x[e][k] * wgt;
            }
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) red[sub][k][lane] = acc[k];
    if (lane < 32) red_ml[sub][lane] = make_float2(M, L);
    __syncthreads();
    // wave `sub` finishes values 8 sub + 4 g .. of the block
    float top = -INFINITY;
    float2 ml[SUBS];
#pragma unroll
    for (int u = 0; u < SUBS; ++u) { ml[u] = red_ml[u][r32]; top = fmaxf(top, ml[u].x); }
    f32x4 y = f32x4{0.f, 0.f, 0.f, 0.f};
    L = 0.f;
#pragma unroll
    for (int u = 0; u < SUBS; ++u) {
        const float wgt = ml[u].x > -INFINITY ? fast_exp2(ml[u].x - top) : 0.f;
        L += ml[u].y * wgt;
        y += red[u][sub][lane] * wgt;
    }
    __syncthreads();                                       // (before the next item's)
    if (rho0 + r32 >= rows) continue;
    const int64_t rho = rho0 + r32, qi = (uint32_t)rho / (uint32_t)G, hd = kvh * (int64_t)G + (rho - qi * G);
    const int64_t q0 = a.q_starts ? a.q_starts[s] : 0, pad = a.q_starts ? 0 : s;
    y *= L != 0.f ? 1.0f / L : 0.f;
    unsigned char* dst = a.out.data + (pad * a.out.seq + (q0 + qi) * a.out.row + hd * a.out.head + 32 * i + 8 * sub + 4 * g) * Elem<T>::bytes;
    if constexpr (C::F32) *reinterpret_cast<f32x4*>(dst) = y;
    else *reinterpret_cast<__attribute__((ext_vector_type(4))) __bf16*>(dst) = __builtin_convertvector(y, __attribute__((ext_vector_type(4))) __bf16);
    if (a.lse && i == 0 && sub == 0 && g == 0)
        a.lse[(a.q_starts ? hd * a.n_hat + q0 : ((int64_t)s * a.Hq + hd) * a.n_hat) + qi] = L != 0.f ? (log2f(L) + top) * 0.69314718055994531f : -INFINITY;
    }
}

int64_t packed_items(int B, int64_t n_hat, int Hkv, int G, bool packed) {
    if (packed) return Hkv * ((n_hat * G + PACKED_ROWS - 1) / PACKED_ROWS + B);
    return (int64_t)B * Hkv * ((n_hat * G + PACKED_ROWS - 1) / PACKED_ROWS);
}
static int packed_resident(int dtype, int d) { return 256 * (dtype == 1 ? 2 : d == 64 ? 4 : 3); }
PackedCut packed_cut(int B, bool packed, int64_t keys, int64_t queries, int Hkv, int G, int dtype, int d, int64_t room) {
    const int64_t items = packed_items(B, queries, Hkv, G, packed);
    const int resident = packed_resident(dtype, d);
    PackedCut c{0, dtype == 1 ? 1 : 8, dtype == 1 ? 1 << 20 : 12, (dtype == 1 ? 4.f : 0.65f) * (d == 64 ? 0.5f : 1.f)};
    const int64_t units = (room < resident ? room : resident) / 8 * 8;
    if (units <= items || B > PACKED_SORTED) return c;
    c.units = (int)units;
    // Where the host sees that nothing will be cut, there is no launch that looks for parts (an empty one is 2.6 us): of equal sequences what the device finds, of others the least that it may find
    const PackedSeq s{(int)keys, (int)queries};
    const int blocks = packed_blocks(s.queries, G), longest = packed_steps(s, G, blocks - 1);
    const bool whole = !packed || B == 1 ? packed_length(c, Hkv, packed_work(s, G) * (float)B, blocks * B, longest) == 1 << 28
                                         : packed_time(c, (float)((keys + PACKED_KEYS - 1) / PACKED_KEYS), (float)items) < packed_time(c, (float)c.least, 1.f) + 7.f;
    if (whole) c.units = 0;
    return c;
}

template <typename T, int D>
static hipError_t run_packed_t(PackedArgs a, hipStream_t st) {
    constexpr int dtype = PackCfg<T, D>::F32 ? 1 : 0;
    const int64_t items = packed_items(a.B, a.n_hat, a.Hkv, a.G, a.q_starts != nullptr);
    a.sorted = a.B <= PACKED_SORTED && items > packed_resident(dtype, D) ? packed_resident(dtype, D) : 0;
    // the ranks of a KV head's items, rounded up to what the XCDs share
    int64_t groups = a.cut.units ? a.cut.units : (items + 7) / 8 * 8;
    if (!a.cut.units && 8 % a.Hkv != 0 && a.Hkv % 8 != 0) groups = items;
    hipLaunchKernelGGL((packed_kernel<T, D>), dim3((uint32_t)groups), dim3(PK_THREADS), (PackCfg<T, D>::LDS), st, a);
    if (a.cut.units) hipLaunchKernelGGL((packed_join_kernel<T, D>), dim3((uint32_t)std::min<int64_t>(items * 4 * PackCfg<T, D>::DBLK, PK_JOIN_GROUPS)), dim3(256), 0, st, a);
    return hipGetLastError();
}
hipError_t init_packed_kernels() {
    hipError_t e;
    if ((e = allow_full_lds(&packed_kernel<bf16_t, 128>)) != hipSuccess || (e = allow_full_lds(&packed_kernel<bf16_t, 64>)) != hipSuccess) return e;
    if ((e = allow_full_lds(&packed_kernel<float, 128>)) != hipSuccess) return e;
    return allow_full_lds(&packed_kernel<float, 64>);
}
hipError_t run_packed(const PackedArgs& a, int dtype, int d, hipStream_t st) {
    if (dtype == 0) return d == 128 ? run_packed_t<bf16_t, 128>(a, st) : run_packed_t<bf16_t, 64>(a, st);
    return d == 128 ? run_packed_t<float, 128>(a, st) : run_packed_t<float, 64>(a, st);
}

}  // namespace ls
