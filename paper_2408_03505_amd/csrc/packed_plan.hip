// Work list of a packed batch: its sequences cut into tiles of kPackedRows
// tokens, the longest sequence first, so that an attention launch starts its
// longest workgroups first and ends with short ones.  Built on the GPU from the
// sequences' offsets, once per batch, and read by every attention launch on it.
//
// Bound by latency.  Every sequence counts the tiles that precede its own (of
// sequences with more tiles, or as many and a lower index), so no sort, atomic
// or second launch is needed and the list is the same every time; that is
// seqs^2 comparisons, 256 sequences to a workgroup.  5 us for 40 sequences.
#include "common.hpp"
#include "kernels.hpp"

namespace optimus {

namespace {

// First token and token count of sequence i, kept inside [0, tokens) whatever
// the offsets hold.
__device__ __forceinline__ void sequence(const int *cu, int i, int tokens, int &first, int &len) {
  first = min(max(cu[i], 0), tokens);
  len = min(max(cu[i + 1], first), tokens) - first;
}

__global__ __launch_bounds__(256) void packed_plan_kernel(int tokens, int seqs, int cap, const int *__restrict__ cu,
                                                          PackedPlan *__restrict__ plan) {
  __shared__ int tiles[256];
  const int tid = threadIdx.x, mine = blockIdx.x * 256 + tid;
  int first = 0, len = 0;
  if (mine < seqs) sequence(cu, mine, tokens, first, len);
  const int t = packed_tiles(len);
  long before = 0, total = 0;
  for (int j0 = 0; j0 < seqs; j0 += 256) {
    int f, l = 0;
    if (j0 + tid < seqs) sequence(cu, j0 + tid, tokens, f, l);
    __syncthreads();
    tiles[tid] = packed_tiles(l);
    __syncthreads();
    const int n = min(256, seqs - j0);  // (the others of the 256 have no tiles)
    for (int j = 0; j < n; j += 8)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int o = tiles[j + e];
        total += o;
        if (o > t || (o == t && j0 + j + e < mine)) before += o;
      }
  }
  // the last tile first: with causal attention it is the longest (offsets that
  // go backwards could ask for more items than there is room for)
  for (int k = 0; k < t && before + k < cap; ++k)
    plan->item[before + k] = PackedItem{first, len, (t - 1 - k) * kPackedRows, 0};
  // empty items behind the list's end
  if (blockIdx.x == 0) {
    for (long k = total + tid; k < cap; k += 256) plan->item[k] = PackedItem{0, 0, 0, 0};
    if (tid == 0) plan->count = static_cast<int>(min(total, static_cast<long>(cap)));
  }
}

}  // namespace

bool launch_packed_plan(int tokens, int seqs, const int *cu, PackedPlan *plan, hipStream_t s) {
  hipLaunchKernelGGL(packed_plan_kernel, dim3((seqs + 255) / 256), dim3(256), 0, s, tokens, seqs,
                     packed_slots(tokens, seqs), cu, plan);
  return true;
}

}  // namespace optimus
