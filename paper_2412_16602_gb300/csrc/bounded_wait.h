// bounded_wait.h - a wait that gives up after a time, for kernels (and, with a clock of its own, for a program on the host).
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define VMB_WAIT_FN __device__ __forceinline__
#else
#define VMB_WAIT_FN inline
#endif

namespace vmb {

// True once test() is, false when `limit` of clock() has passed without that.  What passes may be time in which nothing ran: a context that was
// switched out between a test and the look at the clock comes back late.  So the limit is two halves, whose second begins at the clock as
// it is found then, and a test ends it: work that was done meanwhile counts, and work that was held up as well has half of the limit to go on.
template <typename Test, typename Clock> VMB_WAIT_FN bool bounded_wait(Test test, Clock clock, uint64_t limit) {
    if (test()) return true;
    for (int half = 0; half < 2; ++half) {
        const uint64_t t0 = clock();
        do {
            if (test()) return true;
        } while (clock() - t0 <= limit / 2);
    }
    return test();
}

}  // namespace vmb
