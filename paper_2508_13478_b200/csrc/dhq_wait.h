// A wait that ends: what a kernel does while something has not come yet.  No CUDA in it, so that it runs on a host as well.
#pragma once

#ifdef __CUDACC__
#define DHQ_ANYWHERE __host__ __device__ __forceinline__
#else
#define DHQ_ANYWHERE inline
#endif

namespace dhq {

// Until attempt() is true, or another wait has given up (*failed), or `limit` ns of now() have passed since this wait's own first attempt came back
// without success: then *failed is set.  (Not since the block began: a block that the GPU puts aside, or one with much to do, is no reason to give up.)
template <class Attempt, class Now> DHQ_ANYWHERE bool wait_bounded(Attempt attempt, Now now, unsigned long long limit, volatile int *failed)
{
    unsigned long long begun = 0;
    while (!attempt()) {
        if (*failed) return false;
        const unsigned long long t = now();
        if (begun == 0) begun = t;
        if (t - begun > limit) *failed = 1;
    }
    return true;
}

} // namespace dhq
