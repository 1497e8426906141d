// ls_paged_attend over e2m1 pages: the instances of paged_kernel (ls_paged.h) for them.
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
