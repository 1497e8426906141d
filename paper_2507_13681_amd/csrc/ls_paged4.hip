// ls_paged_attend over e2m1 pages: the instances of paged_kernel (ls_paged.h) for them.
//
// A row of 128 values is 64 bytes of codes and 4 of exponents, one for 32 values: 0.53 bytes a value are read, and so the steps between loads count where for the other types the loads do.
//   K: the 8 codes that a lane has of a fragment are 4 bytes; eight become bf16 with their group's power of two in four instructions, exactly (a code has 2 bits).
//   V: lanes hold a row's 32 values, make them bf16 with their power and put them into the LDS copy that the other types fill by transfers, from which the transposed fragments are read.
//   Products of both halves of a tile take turns, V's fragments are asked for four at a time, and the largest logit goes through registers: a wave's tiles are bound by that chain, about 1.2 us for one
//   of each wave.  One wave finds the workgroup's part and hands it to the others, which would only take its turns at the instructions.
// 8 KV heads of 128, caches not on the chip, us: one of 131072 34.5 (143 MB, 4.1 TB/s; while rows come 6.1), four of 16384, 64 query heads, 19.5 (3.7 TB/s), one of 519 8.4.  Of these about 11, 8 and 8 are there at any
// length: the part is found after 1.8, the first rows are there after 4, waves are merged in 1.1, counted in 1 to 3, parts put together in 3 to 5.
#include "ls_paged.h"

namespace ls {

hipError_t init_paged4_kernels() {
    const hipError_t e = init_paged_t<128, CACHE_E2M1>();
    return e != hipSuccess ? e : init_paged_t<64, CACHE_E2M1>();
}
hipError_t run_paged4(const PagedArgs& a, int d, int units, hipStream_t st) {
    return d == 128 ? run_paged_d<128, CACHE_E2M1>(a, units, st) : run_paged_d<64, CACHE_E2M1>(a, units, st);
}

}  // namespace ls
