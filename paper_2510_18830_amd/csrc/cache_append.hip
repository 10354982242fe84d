// Appends keys and values to the paged 8-bit cache: rotation, quantisation and
// the writes in one pass; the new tokens' queries are rotated on the way.
//
// Token t of sequence b gets the position lens[b] + t.  Rotation pairs columns
// (i, i + d/2): x1' = x1 cos - x2 sin, x2' = x2 cos + x1 sin at the angle
// position * freq[i].  A page's scale is the smallest power of two s with
// max |x| <= 448 s over its tokens of the head, so moving codes to a larger scale
// when later tokens need one is exact but for values that fall below e4m3's
// normal range.  One workgroup per (sequence, page, share of the heads): it owns
// the page's codes and scales of its heads, and the angles are computed once for
// all of them.  Bound by memory at long T (q read and written dominates), by
// latency at one token.
#include "cache.h"
#include "trace.h"

namespace msparse {

namespace {

constexpr int kThreads = 256;

// cos and sin of pos * freq, good to fp32 for any position: the angle in
// revolutions as a sum of two doubles, reduced to an eighth of a revolution, then
// the Taylor series (their first missing terms are below 1e-12).
__device__ __forceinline__ void cos_sin(int pos, float freq, float& c, float& s) {
    constexpr double kInv = 0.15915494309189535, kInvLo = -9.839338337591243e-18;   // 1 / (2 pi) in two parts
    const double x = double(pos) * double(freq);
    const double hi = x * kInv;
    const double lo = __builtin_fma(x, kInv, -hi) + x * kInvLo;
    const double r = (hi - __builtin_rint(hi)) + lo;        // revolutions in [-1/2, 1/2]
    const double quarter = __builtin_rint(4.0 * r);
    const double y = (r - 0.25 * quarter) * 6.283185307179586;   // [-pi/4, pi/4]
    const double y2 = y * y;
    double ps = 1.0 / 6227020800.0, pc = 1.0 / 479001600.0;
    ps = __builtin_fma(ps, y2, -1.0 / 39916800.0);
    pc = __builtin_fma(pc, y2, -1.0 / 3628800.0);
    ps = __builtin_fma(ps, y2, 1.0 / 362880.0);
    pc = __builtin_fma(pc, y2, 1.0 / 40320.0);
    ps = __builtin_fma(ps, y2, -1.0 / 5040.0);
    pc = __builtin_fma(pc, y2, -1.0 / 720.0);
    ps = __builtin_fma(ps, y2, 1.0 / 120.0);
    pc = __builtin_fma(pc, y2, 1.0 / 24.0);
    ps = __builtin_fma(ps, y2, -1.0 / 6.0);
    pc = __builtin_fma(pc, y2, -0.5);
    const float fs = float(__builtin_fma(ps * y2, y, y)), fc = float(__builtin_fma(pc, y2, 1.0));
    const int n = int(quarter) & 3;
    const float a = (n & 1) ? fs : fc, b = (n & 1) ? fc : fs;
    c = (n == 1 || n == 2) ? -a : a;
    s = (n & 2) ? -b : b;
}

// x1 c - x2 s and x2 c + x1 s, every product rounded: the same values whichever
// of the two a fused form would leave unrounded
__device__ __forceinline__ void rotate(float& x1, float& x2, float c, float s) {
#pragma clang fp contract(off)
    const float a = x1 * c, b = x2 * s, e = x2 * c, f = x1 * s;
    x1 = a - b;
    x2 = e + f;
}

__device__ __forceinline__ void unpack8(const u32x4& w, float* x) {
    const uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = bf16_lo(a[j]);
        x[2 * j + 1] = bf16_hi(a[j]);
    }
}

// smallest power of two s >= 2^-126 with amax <= 448 s (448 = 0.875 * 2^9)
__device__ __forceinline__ float code_scale(float amax) {
    int e;
    const float m = frexpf(amax, &e);
    e = m <= 0.875f ? e - 9 : e - 8;
    return amax > 0.f ? ldexpf(1.f, max(e, -126)) : 0x1p-126f;
}
__device__ __forceinline__ float finite_abs(float x) {
    const float a = fabsf(x);
    return a < INFINITY ? a : 0.f;
}
// e4m3 of x * inv, to nearest even; what is not finite becomes NaN
__device__ __forceinline__ float code_input(float x, float inv) {
    return fabsf(x) < INFINITY ? x * inv : __builtin_nanf("");
}
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(code_input(a, inv), code_input(b, inv), 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(code_input(c, inv), code_input(d, inv), w, true);
    return uint32_t(w);
}
// codes moved to a scale 1 / ratio times larger
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float ratio) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_cvt_f32_fp8(w, 0) * ratio,
                                            __builtin_amdgcn_cvt_f32_fp8(w, 1) * ratio, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_cvt_f32_fp8(w, 2) * ratio,
                                        __builtin_amdgcn_cvt_f32_fp8(w, 3) * ratio, r, true);
    return uint32_t(r);
}

// A head's new tokens of one page, 64 x d values over 256 threads: thread u takes
// chunk u % C of the tokens u / C, u / C + R, ... (C chunks of 8 columns a row).
template <int D>
struct Split {
    static constexpr int C = D / 8, R = kThreads / C, N = kPage / R;
};

template <int D>
__global__ void __launch_bounds__(kThreads) cache_append_kernel(AppendArgs a) {
    constexpr int H2 = D / 2, C = Split<D>::C, R = Split<D>::R, N = Split<D>::N;
    constexpr int kPad = 16;                       // V tile rows: 64 codes + pad
    __shared__ __attribute__((aligned(16))) float cosv[kPage * H2], sinv[kPage * H2];
    __shared__ __attribute__((aligned(16))) uint8_t vt[D * (kPage + kPad)];
    __shared__ float red[2][kThreads / 64];
    const int tid = threadIdx.x;
    const int share = blockIdx.x % a.split;
    const int p = blockIdx.x / a.split % a.P;
    const int b = blockIdx.x / (a.split * a.P);
    const int len = max(ldc(a.c.lens, b), 0);
    const int cnt = a.counts ? min(max(ldc(a.counts, b), 0), a.T) : a.T;
    const int lp = len / kPage + p;                // page of the sequence
    const int64_t base = int64_t(lp) * kPage;
    const int s0 = int(max(int64_t(len) - base, int64_t(0)));                  // slots [s0, s1) are new
    const int s1 = int(min(int64_t(len) + cnt - base, int64_t(kPage)));
    const int m = s1 - s0;
    const int t0 = int(base + s0 - len);           // their first token of the call
    // queries are rotated for all T tokens, the count's and those behind it alike
    const int mq = a.q ? int(min(int64_t(len) + a.T - base, int64_t(kPage))) - s0 : 0;
    if (max(m, mq) <= 0) return;
    const int page = m > 0 ? cache_page(a.c, b, lp) : -1;
    if (a.freq) {
        for (int x = tid; x < max(m, mq) * H2; x += kThreads) {
            const int t = x / H2, i = x % H2;
            float c, s;
            cos_sin(int(base + s0 + t), a.freq[i], c, s);
            cosv[t * H2 + i] = c;
            sinv[t * H2 + i] = s;
        }
        __syncthreads();
    }
    // ---- K and V of this share's heads
    if (page >= 0)
        for (int hk = share; hk < a.c.Hkv; hk += a.split) {
            const uint16_t* kp = a.k + b * a.ks[0] + hk * a.ks[1];
            const uint16_t* vp = a.v + b * a.vs[0] + hk * a.vs[1];
            const int64_t at = int64_t(page) * a.c.Hkv + hk;
            uint8_t* kc = a.c.k + at * (kPage * D);
            uint8_t* vc = a.c.v + at * (kPage * D);
            const float kwas = s0 > 0 ? a.c.ks[at] : 0.f, vwas = s0 > 0 ? a.c.vs[at] : 0.f;
            // K: columns 4 c .. 4 c + 3 of either half; V: columns 8 c .. 8 c + 7
            const int c = tid % C, r0 = tid / C;
            float kx[N][8], vx[N][8];
            float km = 0.f, vm = 0.f;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int t = r0 + n * R;
                if (t < m) {
                    const uint16_t* kr = kp + (t0 + t) * a.ks[2];
                    const u32x2 lo = *reinterpret_cast<const u32x2*>(kr + 4 * c);
                    const u32x2 hi = *reinterpret_cast<const u32x2*>(kr + H2 + 4 * c);
                    unpack8(u32x4{lo.x, lo.y, hi.x, hi.y}, kx[n]);
                    unpack8(*reinterpret_cast<const u32x4*>(vp + (t0 + t) * a.vs[2] + 8 * c), vx[n]);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) kx[n][j] = vx[n][j] = 0.f;
                }
            }
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int t = r0 + n * R;
                if (t < m && a.freq) {
                    const f32x4 cs = *reinterpret_cast<const f32x4*>(cosv + t * H2 + 4 * c);
                    const f32x4 sn = *reinterpret_cast<const f32x4*>(sinv + t * H2 + 4 * c);
#pragma unroll
                    for (int j = 0; j < 4; ++j) rotate(kx[n][j], kx[n][4 + j], cs[j], sn[j]);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    km = fmaxf(km, finite_abs(kx[n][j]));
                    vm = fmaxf(vm, finite_abs(vx[n][j]));
                }
            }
            km = wave_max(km);
            vm = wave_max(vm);
            __syncthreads();   // the last head's readers of red and vt are done
            if ((tid & 63) == 0) {
                red[0][tid >> 6] = km;
                red[1][tid >> 6] = vm;
            }
            __syncthreads();
            km = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
            vm = fmaxf(fmaxf(red[1][0], red[1][1]), fmaxf(red[1][2], red[1][3]));
            const float ksc = fmaxf(code_scale(km), kwas), vsc = fmaxf(code_scale(vm), vwas);
            const float ki = 1.f / ksc, vi = 1.f / vsc;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int t = r0 + n * R;
                if (t < m) {
                    uint8_t* row = kc + (s0 + t) * D;
                    *reinterpret_cast<uint32_t*>(row + 4 * c) = codes4(kx[n][0], kx[n][1], kx[n][2], kx[n][3], ki);
                    *reinterpret_cast<uint32_t*>(row + H2 + 4 * c) = codes4(kx[n][4], kx[n][5], kx[n][6], kx[n][7], ki);
                    const uint32_t w[2] = {codes4(vx[n][0], vx[n][1], vx[n][2], vx[n][3], vi),
                                           codes4(vx[n][4], vx[n][5], vx[n][6], vx[n][7], vi)};
#pragma unroll
                    for (int j = 0; j < 8; ++j) vt[(8 * c + j) * (kPage + kPad) + s0 + t] = uint8_t(w[j >> 2] >> (8 * (j & 3)));
                }
            }
            if (s0 > 0 && ksc > kwas) {   // older tokens move to the larger scale
                const float ratio = kwas * ki;
                for (int x = tid; x < s0 * (D / 4); x += kThreads) {
                    uint32_t* word = reinterpret_cast<uint32_t*>(kc) + x;
                    *word = rescale4(*word, ratio);
                }
            }
            if (tid == 0) {
                a.c.ks[at] = ksc;
                a.c.vs[at] = vsc;
            }
            __syncthreads();
            // V rows from the tile, 16 codes (slots 16 g ..) at a time; codes of other slots stay
            const bool vmove = s0 > 0 && vsc > vwas;
            const float vratio = vwas * vi;
            const int g0 = vmove ? 0 : s0 / 16, g1 = (s1 + 15) / 16;
            for (int x = tid; x < D * (g1 - g0); x += kThreads) {
                const int row = x / (g1 - g0), g = g0 + x % (g1 - g0);
                u32x4* dst = reinterpret_cast<u32x4*>(vc + row * kPage + 16 * g);
                u32x4 w = *reinterpret_cast<const u32x4*>(vt + row * (kPage + kPad) + 16 * g);
                if (16 * g < s0 || 16 * g + 16 > s1) {
                    const u32x4 held = *dst;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int s = 16 * g + 4 * j;   // this word's first slot
                        const uint32_t old = vmove ? rescale4(held[j], vratio) : held[j];
                        uint32_t r = 0;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t byte = 0xffu << (8 * e);
                            const uint32_t src = s + e < s0 ? old : s + e < s1 ? w[j] : held[j];
                            r |= src & byte;
                        }
                        w[j] = r;
                    }
                }
                *dst = w;
            }
        }
    // ---- the queries of this share's heads
    if (mq <= 0) return;
    constexpr int QC = D / 16;                     // chunks of 8 pairs of columns
    const int heads = (a.Hq - share + a.split - 1) / a.split;
    for (int x = tid; x < heads * mq * QC; x += kThreads) {
        const int c = x % QC, t = x / QC % mq, h = share + a.split * (x / (QC * mq));
        const uint16_t* src = a.q + b * a.qs[0] + h * a.qs[1] + (t0 + t) * a.qs[2] + 8 * c;
        uint16_t* dst = a.qout + b * a.qos[0] + h * a.qos[1] + (t0 + t) * a.qos[2] + 8 * c;
        u32x4 lo = *reinterpret_cast<const u32x4*>(src), hi = *reinterpret_cast<const u32x4*>(src + H2);
        if (a.freq) {
            float x1[8], x2[8];
            unpack8(lo, x1);
            unpack8(hi, x2);
            const float* cs = cosv + t * H2 + 8 * c;
            const float* sn = sinv + t * H2 + 8 * c;
#pragma unroll
            for (int j = 0; j < 8; ++j) rotate(x1[j], x2[j], cs[j], sn[j]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                lo[j] = pack_bf16x2(x1[2 * j], x1[2 * j + 1]);
                hi[j] = pack_bf16x2(x2[2 * j], x2[2 * j + 1]);
            }
        }
        *reinterpret_cast<u32x4*>(dst) = lo;
        *reinterpret_cast<u32x4*>(dst + H2) = hi;
    }
}

}  // namespace

hipError_t launch_cache_append(const AppendArgs& a, hipStream_t s) {
    TraceScope _t("cache_append", s);
    const dim3 g(unsigned(int64_t(a.c.B) * a.P * a.split)), t(kThreads);
    if (a.c.d == 128) hipLaunchKernelGGL(cache_append_kernel<128>, g, t, 0, s, a);
    else hipLaunchKernelGGL(cache_append_kernel<64>, g, t, 0, s, a);
    return hipGetLastError();
}

}  // namespace msparse
