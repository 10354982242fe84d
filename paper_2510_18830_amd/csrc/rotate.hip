// Rotation of queries and keys by positions on several axes, and its transpose for
// their gradients.
//
// Columns (i, i + d/2) turn by the angle p[axis[i]] freq[i] of their token: x1' = x1 cos -
// x2 sin, x2' = x2 cos + x1 sin.  The map is orthogonal, so the gradient of its input is
// the gradient of its output turned back (the sine negated).  Angles are formed in 64 bits
// for positions of any size and rounded to 32 once, products and sums are in 32 bits, and
// the result is rounded once.
//
// Bound by memory.  A workgroup takes up to 64 tokens and a share of the heads of q and k,
// forms the tokens' angles once for all of them in LDS, and passes the heads' rows by the
// caches: they are read and written once.  131072 tokens, 32 + 8 heads of 128: bf16 530 us, 5.1 TB/s;
// fp32 1105 us, 4.9 TB/s.  777 tokens, 4 + 2 heads of 64: 5.5 us, a launch and a round of each.
#include "rotate.h"
#include "trace.h"

namespace msparse {

namespace {

constexpr int kThreads = 256;

template <class T>
struct Row8;   // eight columns of a row in memory
template <>
struct Row8<uint16_t> {
    u32x4 w;
    __device__ __forceinline__ void load(const uint16_t* p) {
        w = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    }
    __device__ __forceinline__ void store(uint16_t* p) const {
        __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(p));
    }
};
template <>
struct Row8<float> {
    f32x4 w[2];
    __device__ __forceinline__ void load(const float* p) {
        w[0] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p));
        w[1] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p + 4));
    }
    __device__ __forceinline__ void store(float* p) const {
        __builtin_nontemporal_store(w[0], reinterpret_cast<f32x4*>(p));
        __builtin_nontemporal_store(w[1], reinterpret_cast<f32x4*>(p + 4));
    }
};
__device__ __forceinline__ void turn(Row8<uint16_t>& r1, Row8<uint16_t>& r2, const float* c, const float* s) {
    rotate8<true>(r1.w, r2.w, c, s);
}
__device__ __forceinline__ void turn(Row8<float>& r1, Row8<float>& r2, const float* c, const float* s) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float x1 = r1.w[j >> 2][j & 3], x2 = r2.w[j >> 2][j & 3];
        rotate(x1, x2, c[j], s[j]);
        if (!stays(s[j])) {
            r1.w[j >> 2][j & 3] = x1;
            r2.w[j >> 2][j & 3] = x2;
        }
    }
}

template <int D, class T>
__global__ void __launch_bounds__(kThreads) rotate_kernel(RotateArgs a) {
    constexpr int H2 = D / 2, C = D / 16;   // chunks of eight pairs of a row
    __shared__ __attribute__((aligned(16))) float cosv[kRotateTokens * H2], sinv[kRotateTokens * H2];
    const int share = blockIdx.x % a.shares;
    const int blk = blockIdx.x / a.shares % a.blocks, b = blockIdx.x / a.shares / a.blocks;
    const int t0 = blk * kRotateTokens, m = min(a.T - t0, kRotateTokens);
    for (int x = threadIdx.x; x < m * H2; x += kThreads) {
        const Turn z = turn_at(a.pos, x % H2, int64_t(b) * a.T + t0 + x / H2);
        cosv[x] = float(z.c);
        sinv[x] = a.inverse ? -float(z.s) : float(z.s);
    }
    __syncthreads();
    // the share's heads, every shares-th of q's and then k's; items are (head, token, chunk)
    const int heads = (a.Hq + a.Hkv - share + a.shares - 1) / a.shares, each = m * C;
    const T* q = static_cast<const T*>(a.q);
    const T* k = static_cast<const T*>(a.k);
    T* qo = static_cast<T*>(a.qout);
    T* ko = static_cast<T*>(a.kout);
    constexpr int U = sizeof(T) == 2 ? 4 : 2;   // items in flight
    for (int x0 = threadIdx.x; x0 < heads * each; x0 += U * kThreads) {
        Row8<T> r1[U], r2[U];
        T* to[U];
        int at[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int x = x0 + u * kThreads;
            to[u] = nullptr;
            if (x >= heads * each) continue;
            const int h = share + x / each * a.shares, y = x % each, t = y / C, c = y % C;
            const bool isq = h < a.Hq;
            const T* from = isq ? q + b * a.qs[0] + h * a.qs[1] + (t0 + t) * a.qs[2]
                                : k + b * a.ks[0] + (h - a.Hq) * a.ks[1] + (t0 + t) * a.ks[2];
            to[u] = (isq ? qo + b * a.qos[0] + h * a.qos[1] + (t0 + t) * a.qos[2]
                         : ko + b * a.kos[0] + (h - a.Hq) * a.kos[1] + (t0 + t) * a.kos[2]) + 8 * c;
            at[u] = t * H2 + 8 * c;
            r1[u].load(from + 8 * c);
            r2[u].load(from + 8 * c + H2);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!to[u]) continue;
            turn(r1[u], r2[u], cosv + at[u], sinv + at[u]);
            r1[u].store(to[u]);
            r2[u].store(to[u] + H2);
        }
    }
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& a, hipStream_t s) {
    TraceScope _t("rotate", s);
    const dim3 g(unsigned(int64_t(a.B) * a.blocks * a.shares)), t(kThreads);
    if (a.f32) {
        if (a.d == 128) hipLaunchKernelGGL((rotate_kernel<128, float>), g, t, 0, s, a);
        else hipLaunchKernelGGL((rotate_kernel<64, float>), g, t, 0, s, a);
    } else {
        if (a.d == 128) hipLaunchKernelGGL((rotate_kernel<128, uint16_t>), g, t, 0, s, a);
        else hipLaunchKernelGGL((rotate_kernel<64, uint16_t>), g, t, 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace msparse
