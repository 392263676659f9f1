// Sums that the blocks of one launch leave in scratch memory which nothing has
// set up: which block is the last to come, and so adds them.
//
// A block writes its part, then a mark that only this call has, and then looks
// at the marks of all.  Between the two stands a sequentially consistent fence:
// of two blocks at least one sees the other's mark, so the last one sees all of
// them.  No block waits for another, whatever is resident and however late a
// block comes.  Blocks that come at the same time may each see all marks; they
// then add the same parts in the same order and write the same values.  Who has
// seen all takes them away, so that a captured call, whose mark is the same at
// every replay, finds none of its own.
#pragma once

#include <cuda_runtime.h>

namespace aloco {

// By the thread that has written the block's part (or behind a barrier that
// others of the block have written theirs before).
__device__ __forceinline__ void leave_mark(unsigned long long *p, unsigned long long mark) {
    __threadfence();  // the part is there before the mark is
    asm volatile("st.relaxed.gpu.global.u64 [%0], %1;" ::"l"(p), "l"(mark) : "memory");
    __threadfence();  // and the mark before the block looks at the others
}

// Whether this thread's share of n marks, `stride` bytes apart, is there: tid
// and every THREADS-th after it.  Behind a barrier after leave_mark; a block
// may read the parts when all its threads have said yes at another barrier.
template <int THREADS>
__device__ __forceinline__ bool marks_here(const char *first, int stride, int n,
                                           unsigned long long mark, int tid) {
    constexpr int kAtOnce = 4;
    for (int c = tid; c < n; c += kAtOnce * THREADS) {
        unsigned long long m[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            m[k] = mark;
            if (c + k * THREADS < n)
                asm volatile("ld.relaxed.gpu.global.u64 %0, [%1];"
                             : "=l"(m[k])
                             : "l"(first + (size_t)(c + k * THREADS) * stride)
                             : "memory");
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
            if (m[k] != mark) return false;
    }
    __threadfence();  // the marks before the parts
    return true;
}

template <int THREADS>
__device__ __forceinline__ void take_marks(char *first, int stride, int n, int tid) {
    for (int c = tid; c < n; c += THREADS)
        asm volatile("st.relaxed.gpu.global.u64 [%0], %1;" ::"l"(first + (size_t)c * stride),
                     "l"(0ull)
                     : "memory");
}

}  // namespace aloco
