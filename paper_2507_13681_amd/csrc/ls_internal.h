// Host-side argument blocks and launchers shared by the translation units of libloopserve.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace ls {

struct ScoreArgs {
    const void* q;            // [B,Hq,w,d]
    const void* k;            // [B,Hkv,n,d]
    const int64_t* q_pos;     // [w] or null
    int64_t n;
    int w, G, Hq, Hkv, B, BH, nkb;
    float scale_log2e;
    float* part;              // [B*Hkv][nkb][G*w][2] per key block max / sum of every row; later the shares of the totals
    float* rowstat;           // [BH*w][2]        row max, 1 / row sum
    float* spart;             // [2][BH][n][2]    mode 0: diagonal partial sum / max by key-block parity, or what neighbouring key blocks leave each other (edge, edge_share, edge_done)
    float *vert, *slash, *vmax, *smax, *total;
    float* gscore;            // [B*Hkv][n]       group-summed column sums (retention score)
    float* a_win;             // [BH][w][n]       the window matrix (mode 3), or [heads from bh_first on][t1 - t0][n] a band of it (mode 1)
    int64_t win_rows;         // mode 1: how many rows of a KV head's G heads the buffer takes, at least one
    // set by run_score for each launch
    bool retain;              // mode 2: all rows in LDS
    int parts, stat_chunks;   // ranges of keys whose row statistics lie in `part`; chunks of rows of a workgroup of range_stats_kernel, at most
    bool join;                // mode 0: lines_kernel joins the key blocks' results itself
    int shares;               // mode 0: workgroups that share a KV head's query heads
    int bk0, bh_first;        // first KV head / query head
    int t0, t1;               // window rows whose matrix is written out
    int sums;                 // mode 1: the column sums of the chunks are added here (not on a chunk's later bands)
    uint32_t* done;           // [BH] workgroups of lines_kernel or finish_kernel that are done, of a head (the first of a share), cleared by stats_kernel or range_stats_kernel (null: not used)
};

// Where range x of `ranges` begins among `count` tiles or blocks of keys: floor(count * x / ranges).  That product passes 2^32 in ls_score, which has up to 768
// ranges and takes up to 2^31 keys (2^24 blocks); these do not, with at most 2^16 ranges.
__host__ __device__ inline uint32_t range_begin(uint32_t count, uint32_t ranges, uint32_t x) {
    const uint32_t each = count / ranges, rest = count % ranges;
    return each * x + rest * x / ranges;
}
// What of the scoring passes serves a call.
struct ScoreRoute {
    int ranges, unit;         // range_stats_kernel: ranges of keys, cut at multiples of `unit` keys; 0: stats_kernel
    int chunks;               // of 32 query rows, a workgroup of range_stats_kernel at most
    int shares;               // workgroups of stats_kernel that share a KV head's query heads
    bool folds;               // no merge_kernel: lines_kernel merges the row statistics
    bool joins;               // no finish_kernel: lines_kernel joins the key blocks' results
    bool streams;             // retention: all query rows stay in LDS while the keys come by
    int band_heads, band_rows, band_shares;        // mode 1: KV heads and window rows of a band of the matrix, workgroups of the first that share a KV head's query heads
};
ScoreRoute score_route(ScoreArgs& a, bool bf16, int d, int mode);

constexpr int SELECT_RANGES = 128;         // most ranges that a list is put in order by
constexpr int SELECT_HEAD_LINES = 1024;   // lines at the front of each sorted list whose weight and maximum are stored in order at least

// (The order decides which of its pointers walk_exact_kernel keeps in vector registers; with `w` last and `spin_limit` between the
// pointers it takes 73.9 instead of 69.6 us for 16 heads of 907 lines, 51.2 instead of 49.7 for 32 of 8192.)
struct SelectArgs {
    int64_t n, n_hat;
    int BH;
    float alpha;
    int spin_limit;           // bound of every wait between the waves of walk_kernel
    int w;                    // rows of a_win
    const float *vert, *slash, *vmax, *smax, *total;
    int32_t* sidx;            // [2][BH][n] line indices in sorted order
    int64_t kept;             // of each sorted list, the first lines whose weight and largest entry are there in order: n, or SELECT_HEAD_LINES
    float *sorted_w, *sorted_m;            // [2][BH][kept] (sorted_m: null where nobody wants it)
    int32_t* info;            // [2][BH][SELECT_RANGES] of a range of the list: 0: in order, 1: and one of its largest entries is negative or no number, -1 - k: left out, and k of the
                              // lines before it are in order (only with `open`); null: nobody has looked
    int32_t* open;            // [BH] ranges that were left out, of heads whose walk came to the end of what is in order (else 0), [BH] workgroups that have put their share of the rest in order; null: all of it is
    int ranges;               // of a list
    bool sorted;              // kept == n, and a block of lines may be read past the lists' ends
    int32_t *v_idx, *v_cnt, *s_idx, *s_cnt;
    int cap_v, cap_s;
    float* accounted;         // may be null
    int32_t* status;          // device status word of the context (bits LS_STAT_*), OR-ed into
    // exact-overlap variant (run_select_exact) only
    const float* a_win;       // [BH][w][n] window matrix
    const int64_t* q_pos;     // [w] positions of the scored rows, or null (the last w)
};

constexpr int64_t TOPB_MAX_LEN = 262144;   // longest score row run_topb takes

struct TopbArgs {
    const float* score;       // [BK][len]
    int64_t len;              // <= TOPB_MAX_LEN
    int budget;
    int32_t *keep_idx, *keep_cnt;
    // filled in by run_topb from its scratch block
    int chunks;
    uint32_t *hist, *state, *cnt;
};

constexpr uint32_t CUT_ON = 1u << 30;     // in a cut's tile word: the piece ends inside the item in which it begins

struct PlanArgs {
    int64_t n;
    int words, tab_len;
    const int32_t *v_idx, *v_cnt, *s_idx, *s_cnt;
    int cap_v, cap_s;
    uint32_t* obits;          // [BH][4 + words], four zero words first
    uint8_t* tab;             // [BH][tab_len]
    int nqb;                  // row blocks of the turn
    int64_t pos0;             // position of the first
    int dtype;
    uint16_t* elist;          // [BH][tab_len + 1] the table entries with a selected diagonal, ascending
    uint32_t* rec;            // [BH][nqb] of each row block: key blocks it visits | columns it gathers << 13
    uint32_t* upto;           // [BH][nqb] work of the head's row blocks up to and including this one (null: not wanted)
    uint32_t* arrived;        // [BH][nqb] cleared here for the parts of items (wanted with `upto`)
    uint32_t* head_work;      // [BH] work of all of them
    int32_t* split_count;     // [2] cleared here for sched_kernel
    int32_t* status;          // device status word of the context (bits LS_STAT_*), OR-ed into
};

// Work queues of the sparse attention kernel: one list per XCD of (head, row block) items or parts of them.
struct SchedArgs {
    int BH, G, Hq, Hkv, nqb;
    const uint32_t* rec;      // [BH][nqb], as plan_kernel left them
    const uint32_t* head_work;
    uint4* queue;             // [items + slots] entries, one queue behind the other: {item, part | parts << 8 | first slot << 16, key blocks, columns}
    int32_t* qlen;            // [8]
    int32_t* qbase;           // [8] first entry of each queue
    int32_t* qhead;           // [8] next entry to hand out (the first ones go by workgroup number)
    int grid;                 // workgroups of the attention kernel
    int slots;                // results of parts that the workspace holds (0: no item is split)
    uint2* split;             // [slots] split items: {item, parts | first slot << 16}
    int32_t* split_count;     // [2] slots in use, split items; cleared by plan_kernel
};

struct PrefillArgs {
    const void *q, *k, *v;
    void* out;
    float* lse;
    int64_t n, n_hat, pos0;
    int Hq, Hkv, G, BH, nqb, words, tab_len, dtype;
    float scale_log2e;
    const uint32_t* obits;
    const uint8_t* tab;
    const int32_t* v_idx;
    int cap_v;
    const uint16_t* elist;    // as plan_kernel left them
    int grid;                 // workgroups
    int slots;                // results of parts that may be kept
    // pieces (ls_prefill.hip): at most `grid`
    const uint32_t* rec;
    const uint32_t *upto, *head_work;
    int2* cuts;               // [1 + pieces] their number, and where each piece begins {item, tile | CUT_ON (that flag with `arrived` only)}
    uint32_t* arrived;        // [BH][nqb] tiles of the item's parts that are done, cleared by plan_kernel; null: combine_kernel puts the parts together
    // or work queues built by sched_kernel
    const uint4* queue;       // null: pieces
    const int32_t *qlen, *qbase;
    int32_t* qhead;
    const uint2* split;
    const int32_t* split_count;
    float *part_o, *part_ml;  // [slots][128][d] accumulators in lane order, [slots][128][2] reference and normaliser
};

struct DecodeArgs {
    const void *q;            // [B][Hq][d]
    const void *kc, *vc;      // [B][Hkv][cap][d] retained entries (first cnt rows valid)
    const void *kt, *vt;      // [B][Hkv][T][d] tokens since the retention
    const int32_t* cnt;       // [B][Hkv] or NULL (all cap rows)
    void* out;                // [B][Hq][d]
    float* lse;               // [B][Hq] or NULL
    float* part;              // [B*Hkv][nsplit][G][d + 4] per-split output, reference, normaliser
    uint32_t* done;           // [B*Hkv] splits finished; zero between calls
    uint32_t* done_clear;     // [clear_heads] the counters of the call after the next, cleared here; clear_heads >= B*Hkv
    int clear_heads;
    int B, Hq, Hkv, G, cap, T, nsplit, chunk;
    float scale_log2e;
};

// A paged cache (ls_cache)
struct CacheArgs {
    unsigned char *k, *v;     // [pages][Hkv][page][d] bf16 or e4m3
    uint8_t *kx, *vx;         // [pages][Hkv][page] e4m3: exponents
    const int32_t* table;     // [B][max_pages]
    int max_pages;
    uint32_t pages;
    int Hkv, page_log;        // a page holds 2^page_log positions
};
// Rows of a caller's tensor (ls_rows)
struct RowArgs {
    unsigned char* data;
    int64_t seq, row, head;   // strides, elements
};
// The page of position p of sequence b as the table has it, or -1: that position is nowhere.
__host__ __device__ inline int page_of(const CacheArgs& c, int b, int64_t p) {
    const int64_t at = p >> c.page_log;
    if (p < 0 || at >= c.max_pages) return -1;
    const int32_t id = c.table[(int64_t)b * c.max_pages + at];
    return (uint32_t)id < c.pages ? id : -1;
}
// Rows a .. e - 1 of `rows`, as a sequence's starts say: whether they are any
__host__ __device__ inline bool starts_ok(int32_t a, int32_t e, int64_t rows) { return a >= 0 && e >= a && e <= rows; }

struct MoveArgs {
    CacheArgs cache;
    RowArgs k, v;
    const int32_t *starts, *count, *pos;       // as ls_cache_write has them
    int B, n_hat;
    int heads;                // KV heads of a workgroup
    int64_t group0;           // first group of rows of this launch
    bool once;                // pages that are read are not read again soon
    int32_t* status;
};

// ls_paged_attend.  A unit of work is a part of the 32-key tiles of one KV head of one sequence, and a workgroup has one.  Which one follows from the lengths, which only the device
// knows.
constexpr int PAGED_TILE = 32;               // keys
// Few heads go in as many parts as there are compute units, which have a workgroup each; more heads, whose lengths may differ, in twice as many at most, two workgroups to a unit: what is
// left over at the ends is shorter then, but a part more is a result more to put together.  256 parts / 512, us: four caches of 16384, 8 KV heads, e4m3 31.1 / 33.6, one of 131072, bf16 96.7 / 102.2; 13 caches of
// 1 to 67000 113.7 / 106.2, 24 of 0 to 31000 96 / 56.6.  Parts are as short as lets all of them run at once.
constexpr int PAGED_ALONE = 64;              // heads up to which a workgroup has its compute unit for itself
__host__ __device__ inline int paged_slots(int64_t heads) { return heads <= PAGED_ALONE ? 256 : 512; }
__host__ __device__ inline bool paged_at_once(int64_t heads) { return heads * 4 <= paged_slots(heads) * 3; }
// Tiles that a head is not cut for, two a wave.  Whole / in parts, us: 32 tiles 14.3 / 8.9, 17 tiles 9.8 / 8.7, 10 tiles 7.1 / 8.3, 16 tiles of 32 sequences 10.6 / 14.0
constexpr int PAGED_WHOLE = 16;
constexpr int PAGED_SHORTEST = 4, PAGED_SHORTEST_MANY = 32;                          // tiles of a part at least; of that many heads
__host__ __device__ inline int paged_cuts(int tiles, int length) { return tiles <= PAGED_WHOLE ? 1 : (int)(((uint32_t)tiles + (uint32_t)length - 1) / (uint32_t)length); }
// Tiles of a part of a call, of so many tiles in all: what `length` makes of them is counted until it is accepted, four times at most, and then `enough` is taken.  (24 ragged caches of 3212 tiles: 51, 57, 60
// and 63 tiles are too many parts, 65 would do, 81 are taken.)
struct PagedLength {
    int length, enough, slots, tries;        // enough: it will do, whatever the sequences are
    bool sorts;                              // not all parts run at once: the longest first
    __host__ __device__ PagedLength(int64_t tiles, int64_t heads) : slots(paged_slots(heads)), tries(0) {
        const bool at_once = paged_at_once(heads);
        sorts = !at_once;
        auto least = [&](int64_t parts) {
            const int64_t each = (tiles + parts - 1) / parts, from = at_once ? PAGED_SHORTEST : PAGED_SHORTEST_MANY;
            return each < from ? (int)from : each < 1 << 30 ? (int)each : 1 << 30;
        };
        length = least(slots);
        enough = at_once ? least(slots - heads) : length;      // (a part begun in each head)
    }
    __host__ __device__ bool accepts(int64_t units) {
        if (units <= slots || length >= enough) return true;
        const int64_t more = length * (units - slots) / slots / 2;
        length += more > 1 ? (int)more : 1;
        if (length > enough || ++tries == 4) length = enough;
        return false;
    }
};
struct PagedArgs {
    CacheArgs cache;
    const void* q;            // [B][Hq][d]
    const int32_t* len;       // [B]
    void* out;                // [B][Hq][d]
    float* lse;               // [B][Hq] or NULL
    float* part;              // [units][G][d + 4] output, reference, normaliser of each part of a head
    uint32_t* done;           // [B*Hkv] parts finished; zero between calls.  Null: paged_join_kernel puts the parts together
    uint32_t* done_clear;     // [clear_heads] the counters of the call after the next, cleared here
    int clear_heads;
    int B, Hq, Hkv, G;
    int64_t most;             // no sequence is longer
    float scale_log2e;
    int32_t* status;
};

// ls_packed_prefill.  An item is a block of 128 rows of one KV head of one sequence, where a "row" is one of the G query heads of one query: row r is head r % G of query
// r / G.  Items go by how many 32-key steps they take; where there are few of them they are cut into parts.  (Keys, and queries times G, are less than 2^31: 32-bit divisions,
// which take a tenth of the instructions that 64-bit ones do.)
constexpr int PACKED_ROWS = 128, PACKED_KEYS = 32;
struct PackedSeq { int keys, queries; };
__host__ __device__ inline int packed_blocks(int queries, int G) { return (int)(((uint32_t)queries * (uint32_t)G + (PACKED_ROWS - 1)) / PACKED_ROWS); }
// steps that block j of a sequence takes: those up to the last key that its last row sees
__host__ __device__ inline int packed_steps(const PackedSeq& s, int G, int j) {
    const uint32_t rows = (uint32_t)s.queries * (uint32_t)G, behind = (uint32_t)PACKED_ROWS * (uint32_t)(j + 1), end = behind < rows ? behind : rows;
    const int seen = s.keys - s.queries + (int)((end - 1) / (uint32_t)G) + 1;
    return seen > 0 ? (int)(((uint32_t)seen + (PACKED_KEYS - 1)) / PACKED_KEYS) : 0;
}
// blocks of a sequence that take more than x steps: its last ones.  (The last row sees query y or one after it, y = 32 x - keys + queries, if
// the block ends behind row y G.)
__host__ __device__ inline int packed_longer(const PackedSeq& s, int G, int x) {
    const int blocks = packed_blocks(s.queries, G);
    if (x < 0) return blocks;
    const int64_t y = (int64_t)PACKED_KEYS * x - s.keys + s.queries;
    if (y >= s.queries) return 0;
    return y <= 0 ? blocks : blocks - (int)((uint32_t)y * (uint32_t)G / PACKED_ROWS);
}
// no less than the steps of all its blocks together (each less than 4 above what is linear in j)
__host__ __device__ inline float packed_work(const PackedSeq& s, int G) {
    const float blocks = (float)packed_blocks(s.queries, G), before = s.keys > s.queries ? (float)((s.keys - s.queries) / PACKED_KEYS) : 0.f;
    return blocks * (before + 4.f) + 0.5f * PACKED_ROWS / PACKED_KEYS * blocks * (blocks + 1.f) / (float)G;
}
constexpr int64_t PACKED_MOST_ITEMS = (1 << 24) - 8;   // (of a grid of 2^32 threads HIP runs what is left modulo 2^32, without an error)
// With more sequences items go by sequence, whole: a wave's lanes have a sequence each, once.  64 / 65 sequences, us: one new row of each on 20000 keys, 4 query heads of one KV head 154 / 458, one of 20000
// among ones of 300, a new row each, 8 KV heads 68 / 332; where the rows fill the chip there is nothing to cut: prompts of 300 and one of 8192 589 / 582.
constexpr int PACKED_SORTED = 64;
// How a call cuts its items.  Parts are no more than the workgroups that are resident, so that they run at once (fp32 at d = 128 twice as many: one and two rounds, us, 1024 positions 51.6 / 47.0,
// 300 and 40 new rows behind 2700 and none 103.5 / 76.6).  Whole / cut, us: follow-ups of 1 to 200 rows on 2900 to 20000 keys 460 / 83, 61 new rows of 12347 216 / 37, fp32 1024 positions of 8 heads of 128 149 / 47.
struct PackedCut {
    int units;                // parts that there is room for; 0: items are whole
    int least, some;          // steps of a part at least; up to this many, as many as leave a part to a compute unit
    float step;               // what a step takes where a workgroup has its compute unit for itself, us
};
// What `steps` steps of `groups` workgroups take, us: where compute units have more than one, each takes longer.
__host__ __device__ inline float packed_time(const PackedCut& c, float steps, float groups) {
    return c.step * steps * (groups > 256.f ? 0.67f + 0.33f / 256.f * groups : 1.f);
}
// Steps of a part, of so much work, so many items and the longest of them (all of one of the Hkv KV heads); items and parts are no more than units / Hkv then.  Where whole items
// take no longer than parts and what it takes to put them together (7 us, and 3 for a hundred parts), they stay whole.
__host__ __device__ inline int packed_length(const PackedCut& c, int Hkv, float work, int items, int longest) {
    const float each = work / (float)(c.units / Hkv - items) * 1.00001f, even = work * (float)Hkv / 256.f;
    float l = even < (float)c.some ? even : (float)c.some;
    l = l > (float)c.least ? l : (float)c.least;
    l = l > each ? l : each;
    if (!(l < (float)longest)) return 1 << 28;
    const float parts = (float)Hkv * ((float)items + work / l);
    if (packed_time(c, (float)longest, (float)items * (float)Hkv) < packed_time(c, l, parts) + 7.f + 0.03f * parts) return 1 << 28;
    return (int)l + ((float)(int)l < l ? 1 : 0);
}
struct PackedArgs {
    RowArgs q, k, v, out;
    const int32_t *q_starts, *k_starts;
    float* lse;
    int B, Hq, Hkv, G;
    int n, n_hat;
    float scale_log2e;
    PackedCut cut;
    int sorted;               // more items than workgroups are resident: how many are, and those of the longest sequences may go first; else 0
    float *part_o, *part_ml;  // [units][128][d] accumulators in lane order, [units][128][2] reference and normaliser
    int32_t* status;
};

// status bits (mirrors of LS_STAT_* in loopserve.h)
constexpr int STAT_WALK_TIMEOUT = 1, STAT_S_TRUNCATED = 2, STAT_V_TRUNCATED = 4, STAT_S_RANGE = 8, STAT_V_INVALID = 16,
              STAT_MERGE_RANGE = 32, STAT_PAGE_RANGE = 64, STAT_STARTS = 128;
constexpr int WALK_SPIN_DEFAULT = 1 << 22;   // never reached in practice (about a second of polling)

// Lets a kernel use all of a compute unit's LDS (160 KB, less what the kernel declares statically) as
// dynamic LDS; the launches then only have to name the size they need.
template <typename K>
inline hipError_t allow_full_lds(K kernel) {
    hipFuncAttributes fa;
    hipError_t e = hipFuncGetAttributes(&fa, reinterpret_cast<const void*>(kernel));
    if (e != hipSuccess) return e;
    return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                               160 * 1024 - (int)fa.sharedSizeBytes);
}

// Once per device, with that device current: lets every kernel that asks for dynamic LDS use the whole 160 KB.
hipError_t init_score_kernels();
hipError_t init_select_kernels();
hipError_t init_prefill_kernels();
hipError_t init_decode_kernels();

hipError_t init_paged_kernels();

hipError_t init_packed_kernels();
hipError_t run_packed(const PackedArgs& a, int dtype, int d, hipStream_t st);
PackedCut packed_cut(int B, bool packed, int64_t keys, int64_t queries, int Hkv, int G, int dtype, int d, int64_t room);           // with room for so many parts' results
int64_t packed_items(int B, int64_t n_hat, int Hkv, int G, bool packed);       // no fewer than there are
hipError_t run_move(const MoveArgs& a, bool write, int dtype, int type, int d, hipStream_t st);
hipError_t run_paged(const PagedArgs& a, int type, int d, int units, hipStream_t st);
int paged_units(int B, int Hkv, int64_t most);                       // workgroups that sequences of up to so many keys take
bool paged_joins(int B, int Hkv, int G, int64_t most);                      // the kernel puts parts together itself
int paged_most_cuts(int B, int Hkv, int64_t most);                   // ... and parts of a head
hipError_t run_score(const ScoreArgs& a, int dtype, int d, int mode, hipStream_t st);
hipError_t run_decode(const DecodeArgs& a, int d, hipStream_t st);
size_t decode_smem_bytes(int d, int G, int nsplit);
size_t decode_part_floats(int d);                                   // floats of one partial result
void decode_split(int BK, int cap, int T, int limit, int* nsplit, int* chunk);   // at most `limit` splits; chunk: 32-key tiles per workgroup
constexpr int DECODE_MAX_SPLITS = 128;
// Union of two selections per head (the accumulated line set of Alg. 1): lists a and b in, ascending unique list out.
struct MergeArgs {
    int64_t n;
    int BH;
    const int32_t *idx_a[2], *cnt_a[2], *idx_b[2], *cnt_b[2];   // [0] diagonals, [1] columns
    int cap_a[2], cap_b[2];
    int32_t *idx[2], *cnt[2];
    int cap[2];
    int32_t* status;
};
hipError_t run_merge_lines(const MergeArgs& a, hipStream_t st);
hipError_t run_select(const SelectArgs& a, hipStream_t st);
int select_ranges_left_out(const SelectArgs& a);                      // ranges of each list of a call that may leave some of them out; else 0
hipError_t run_select_exact(const SelectArgs& a, hipStream_t st);   // a_win, q_pos, w set; vmax / smax unused
hipError_t run_topb(const TopbArgs& a, int BK, uint32_t* scratch, hipStream_t st);   // scratch: topb_scratch_words(BK, len) words
size_t topb_scratch_words(int BK, int64_t len);
hipError_t run_gather_rows(const void* const* src, void* const* dst, int tensors, const int32_t* keep_idx, const int32_t* keep_cnt,
                           int BK, int64_t len, int budget, int row_bytes, hipStream_t st);      // one or two tensors
hipError_t launch_plan(const PlanArgs& a, int BH, hipStream_t st);
hipError_t launch_sched(const SchedArgs& a, hipStream_t st);
// ev (null or four events): the start and stop time of the attention kernel's own dispatch, and, where a.slots > 0, of combine_kernel's
hipError_t launch_prefill(const PrefillArgs& a, int dtype, int d, hipStream_t st, const hipEvent_t* ev = nullptr);
size_t prefill_smem_bytes(int dtype, int d, int tab_len);
int prefill_block_rows();
bool prefill_in_pieces(int BH, int64_t n, int nqb, int dtype, int d);               // the work is shared out in pieces, or by queues
int prefill_grid(int dtype, int d, int64_t n, int64_t items, bool pieces);
int prefill_split_slots(int64_t items, int grid, bool pieces);      // parts' results that a call with so many (head, row block) items may use
size_t prefill_slot_bytes(int d);
int prefill_pieces_for(int64_t items, int grid, int slots);              // workgroups of a call in pieces with room for so many parts' results (0: queues)
bool prefill_joins(int dtype, int64_t items, int grid);               // pieces: whether the attention kernel puts the parts together itself
int prefill_piece_xcd(int p, int pieces);                                // XCD whose workgroup takes piece p

}  // namespace ls
