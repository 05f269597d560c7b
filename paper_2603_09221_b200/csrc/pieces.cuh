// Packed sequences cut into pieces of equal length, whose blocks find what they work on in a table.
#pragma once

#include "block_common.cuh"

namespace ttc {
namespace blk {

// Pieces of packed sequences: seq_first [batch + 1], and {sequence, first token} of each; every sequence has at least `at_least`
// pieces (one in the forward pass, so that its last state is written).  Offsets that do decrease could ask for more than the `bound`
// pieces that there is room for, and for more than 32 bits hold: counts and sums stop at the bound (below 2^31, so the sum of two
// fits), the pieces behind it are left out.  One block.
static __global__ void __launch_bounds__(1024) piece_map_kernel(Seqs s, long long piece, int at_least, long long bound, int2* map, int* seq_first)
{
    wait_for_previous();
    __shared__ unsigned sum[1024];
    __shared__ unsigned base;
    const unsigned most = static_cast<unsigned>(bound);
    if (threadIdx.x == 0)
        base = 0;
    __syncthreads();
    for (long long b0 = 0; b0 < s.batch; b0 += 1024) {
        const long long b = b0 + threadIdx.x;
        unsigned count = 0;
        if (b < s.batch) {
            const long long c = (span_of(s, b).len + piece - 1) / piece;
            count = static_cast<unsigned>(min(max(c, (long long)at_least), bound));
        }
        sum[threadIdx.x] = count;
        __syncthreads();
        for (int o = 1; o < 1024; o *= 2) {
            const unsigned v = threadIdx.x >= o ? sum[threadIdx.x - o] : 0;
            __syncthreads();
            sum[threadIdx.x] = min(sum[threadIdx.x] + v, most);
            __syncthreads();
        }
        if (b < s.batch)
            seq_first[b] = static_cast<int>(min(base + (threadIdx.x ? sum[threadIdx.x - 1] : 0), most));
        __syncthreads();
        if (threadIdx.x == 1023)
            base = min(base + sum[1023], most);
        __syncthreads();
    }
    if (threadIdx.x == 0)
        seq_first[s.batch] = static_cast<int>(base);
    __syncthreads();
    for (long long i = threadIdx.x; i < bound; i += 1024) {
        long long lo = 0, hi = s.batch;                              // the last sequence that does not begin behind piece i
        while (hi - lo > 1) {
            const long long mid = (lo + hi) / 2;
            if (seq_first[mid] <= i)
                lo = mid;
            else
                hi = mid;
        }
        map[i] = i < (long long)base ? make_int2(static_cast<int>(lo), static_cast<int>((i - seq_first[lo]) * piece)) : make_int2(-1, 0);
    }
}

} // namespace blk
} // namespace ttc
