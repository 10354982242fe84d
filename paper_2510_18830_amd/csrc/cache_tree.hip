// Masks and positions of drafted trees.
//
// Node t of a sequence's tree has a parent among the nodes before it, or none (the child of the
// context's last token).  Its position is lens + the number of its ancestors; it sees itself and
// those ancestors that the window or the sinks leave visible.  A thread walks one node's
// ancestors, which descend, and writes its words from the last to the first as it passes them: no
// word is held or read back.  Bound by latency: the walk's LDS reads, one after the other.
#include "cache.h"
#include "trace.h"

namespace msparse {

namespace {

constexpr int kThreads = 256;

__global__ void __launch_bounds__(kThreads) tree_mask_kernel(TreeMaskArgs a) {
    __shared__ int16_t up[kMaxNodes];
    const int b = blockIdx.x;
    const int first = min(max(ldc(a.lens, b), 0), kMaxLength);
    const int nodes = a.counts ? min(max(ldc(a.counts, b), 0), a.T) : a.T;
    for (int t = threadIdx.x; t < a.T; t += kThreads) {
        const int p = a.parents[int64_t(b) * a.T + t];
        up[t] = int16_t(p >= 0 && p < t ? p : -1);
    }
    __syncthreads();
    for (int t = threadIdx.x; t < a.T; t += kThreads) {
        const bool live = t < nodes;
        int depth = 0;
        if (live)
            for (int u = up[t]; u >= 0; u = up[u]) ++depth;
        int32_t* row = a.seen + (int64_t(b) * a.T + t) * a.words;
        int word = a.words - 1;
        uint32_t bits = 0;
        if (live) {
            int u = t;
            for (int k = 0; k <= depth; ++k) {   // the ancestor k steps up, at position first + depth - k
                while (word > u >> 5) {
                    row[word--] = int32_t(bits);
                    bits = 0;
                }
                if (k < a.W || int64_t(first) + depth - k < a.S) bits |= 1u << (u & 31);
                u = up[u];
            }
        }
        while (word >= 0) {
            row[word--] = int32_t(bits);
            bits = 0;
        }
        a.at[int64_t(b) * a.T + t] = int32_t(min(int64_t(first) + depth, int64_t(INT32_MAX)));
    }
}

}  // namespace

hipError_t launch_tree_mask(const TreeMaskArgs& a, hipStream_t s) {
    TraceScope _t("tree_mask", s);
    hipLaunchKernelGGL(tree_mask_kernel, dim3(unsigned(a.B)), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace msparse
