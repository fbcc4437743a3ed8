// The line of keys that persistent blocks share out (attention over four-bit caches).
//
// The keys of all (layer, sequence) pairs, layer-major and the sequences' lengths one after
// another, form one line of n = layers * sum keys; block group g takes keys
// [g * per, (g + 1) * per).  Each block finds its place from the lengths alone, in one scan by
// the whole block (every thread adds up a run of sequences), so no launch and no counter comes
// before the kernel.
#pragma once

#include "sonic_dev.cuh"

namespace sonic {

struct LineShared {
    long long warp_sum[32];
    long long sum;
    int seq, off;
};

// Sum of len(b) over the sequences and the place of key `x(sum)` (of one layer: x < sum) in
// them; len(b) >= 0.  Called by the whole block; sh is written and the block synchronised.
template <int kThreads, typename Len, typename Key>
__device__ __forceinline__ void line_find(int B, Len len, Key key, LineShared &sh) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int run = (B + kThreads - 1) / kThreads;
    const int b0 = min(B, tid * run), b1 = min(B, b0 + run);
    long long mine = 0;
    for (int b = b0; b < b1; ++b) mine += len(b);
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += u;
    }
    if (lane == 31) sh.warp_sum[warp] = incl;
    if (tid == 0) {
        sh.seq = B;
        sh.off = 0;
    }
    __syncthreads();
    long long before = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        const long long v = sh.warp_sum[w];
        if (w < warp) before += v;
        sum += v;
    }
    const long long x = key(sum);
    long long at = before + incl - mine;
    if (x >= at && x < at + mine) {  // one thread
        for (int b = b0; b < b1; ++b) {
            const int n = len(b);
            if (x < at + n) {
                sh.seq = b;
                sh.off = (int)(x - at);
                break;
            }
            at += n;
        }
    }
    if (tid == 0) sh.sum = sum;
    __syncthreads();
}

}  // namespace sonic
