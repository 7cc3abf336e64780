// What the kernels of attention over a cache's rows (span_attn.hip, attn.hip) share.
#pragma once

#include "vitcop_internal.h"

namespace vitcop {

// The sample that a workgroup takes as the `nth`, where samples have lengths of their own: the longest first, so that no long
// one is left over at the end, and every other `layer` of samples (what one workgroup on each CU takes; 0: no layers) backwards,
// so that a CU that starts with a long one goes on with a short one.  Sorted in groups of 64, by every wavefront for itself.
// (16 conversations of up to 2000 rows x 32 heads, 25 drafts: 79 us in the order given, 65 so.)
__device__ __forceinline__ int span_sample(const SpanArgs& A, int nth, int layer) {
    const int lane = threadIdx.x & 63, first = nth & ~63, n = min(64, A.B - first);
    int at = nth - first;
    if (layer > 0 && layer < 64) {
        const int l = at / layer, size = min(layer, n - l * layer);
        if (l & 1) at = l * layer + size - 1 - (at - l * layer);
    }
    int work = -1;
    if (lane < n) {
        const int tok = A.counts ? min(max(A.counts[first + lane], 0), A.T) : A.T;
        const int start = A.starts ? min(max(A.starts[first + lane], 0), A.start) : A.start;
        work = tok == 0 ? 0 : tok + (A.window ? min(start, A.window + A.sinks) : start);
    }
    int rank = 0;
    for (int i = 0; i < n; ++i) {
        const int other = __builtin_amdgcn_readlane(work, i);
        rank += other > work || (other == work && i < lane) ? 1 : 0;
    }
    return first + __builtin_ctzll(__builtin_amdgcn_ballot_w64(lane < n && rank == at));
}

}  // namespace vitcop
