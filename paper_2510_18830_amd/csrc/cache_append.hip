// Appends keys and values to the paged 8-bit cache: rotation, quantisation and
// the writes in one pass; the new tokens' queries are rotated on the way.
//
// Token t of sequence b gets the position lens[b] + t.  Rotation pairs columns
// (i, i + d/2): x1' = x1 cos - x2 sin, x2' = x2 cos + x1 sin at the angle
// position * freq[i].  A page's scale is the smallest power of two s with
// max |x| <= 448 s over its tokens of the head, so moving codes to a larger scale
// when later tokens need one is exact but for values that fall below e4m3's
// normal range.  A workgroup per (sequence, page, share of the KV heads) owns the
// page's codes and scales of its heads, others turn shares of the query heads; each
// computes the page's angles once for all of its heads.  Bound by memory at long T, where
// q read and written dominates: 128K tokens of 28 over 4 heads, 2.28 GB, take 427 us (a
// copy of q alone 358); q passes by the caches (465 us through them).  Bound by latency
// at one token.
#include "cache.h"
#include "codes.h"
#include "rotary.h"
#include "trace.h"

namespace msparse {

namespace {

constexpr int kThreads = kAppendThreads;

// A head's new tokens of one page, 64 x d values over 256 threads: thread u takes
// chunk u % C of the tokens u / C, u / C + R, ... (C chunks of 8 columns a row).
template <int D>
struct Split {
    static constexpr int C = D / 8, R = kThreads / C, N = kPage / R;
};

// AT: the tokens' positions are given, so that every angle is formed by itself (2 x 20011 tokens, 28 over 4 heads of
// 128: 138 us, 114 where it follows from the one before).
template <int D, bool AT>
__global__ void __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(3, D == 128 ? 3 : 4)))
cache_append_kernel(AppendArgs a) {
    constexpr int H2 = D / 2, C = Split<D>::C, R = Split<D>::R, N = Split<D>::N;
    constexpr int kPad = 16;                       // V tile rows: 64 codes + pad
    __shared__ __attribute__((aligned(16))) float cosv[kPage * H2], sinv[kPage * H2];
    __shared__ __attribute__((aligned(16))) uint8_t vt[D * (kPage + kPad)];
    __shared__ float red[2][kThreads / 64];
    const int tid = threadIdx.x, shares = a.kv_shares + a.q_shares;
    const int share = blockIdx.x % shares;
    const int p = blockIdx.x / shares % a.P;
    const int b = blockIdx.x / (shares * a.P);
    const int len = max(ldc(a.c.lens, b), 0);
    const int lp = len / kPage + p;                // page of the sequence
    const int64_t base = int64_t(lp) * kPage;
    const int s0 = int(max(int64_t(len) - base, int64_t(0)));   // the page's first new slot
    const int t0 = int(base + s0 - len);           // its token of the call
    // The angles of the page's new tokens: a thread has one frequency and every
    // STEP-th token, each turned on from the one before by a product in 64 bits (AT: each
    // from its own position).
    auto angles = [&](int tokens) {
        if constexpr (AT) {
            for (int x = tid; x < tokens * H2; x += kThreads) {
                const Turn z = turn_at(a.pos, x % H2, int64_t(b) * a.T + t0 + x / H2);
                cosv[x] = float(z.c);
                sinv[x] = float(z.s);
            }
            __syncthreads();
            return;
        }
        if (a.freq) {
            constexpr int STEP = kThreads / H2;
            const int t = tid / H2;
            if (t < tokens) {
                const float f = a.freq[tid % H2];
                Turn z = turn_by(double(base + s0 + t), f), d{1.0, 0.0};
                if (t + STEP < tokens) d = turn_by(double(STEP), f);
                for (int x = tid; x < tokens * H2; x += kThreads) {
                    cosv[x] = float(z.c);
                    sinv[x] = float(z.s);
                    z = Turn{z.c * d.c - z.s * d.s, z.s * d.c + z.c * d.s};
                }
            }
        }
        __syncthreads();
    };
    // The queries of every shares-th head: all T tokens, the count's and those behind
    // it alike.  A thread has 8 pairs of columns of a token (of QN tokens at head dim
    // 128) and walks the heads, the next one's loads in flight; `par` heads go side by
    // side where the tokens are few.
    const int mq = a.q ? int(min(int64_t(len) + a.T - base, int64_t(kPage))) - s0 : 0;
    auto queries = [&](int share, int shares) {
        const int m = mq;
        if (m <= 0) return;
        constexpr int QC = query_chunks(D), QN = kPage * QC / kThreads;
        const int combos = m * QC, par = heads_aside(m, D);
        const int heads = (a.Hq - share + shares - 1) / shares;
        const int h0 = par > 1 ? tid / combos : 0, x0 = par > 1 ? tid % combos : tid;
        const int c = x0 % QC;                     // (kThreads is a multiple of QC)
        const uint16_t* src = a.q + b * a.qs[0] + 8 * c;
        uint16_t* dst = a.qout + b * a.qos[0] + 8 * c;
        bool mine[QN];
        int64_t from[QN], to[QN];
#pragma unroll
        for (int u = 0; u < QN; ++u) {
            const int x = x0 + u * kThreads;
            mine[u] = x < combos && h0 < par;
            from[u] = (t0 + x / QC) * a.qs[2];
            to[u] = (t0 + x / QC) * a.qos[2];
        }
        u32x4 lo[QN], hi[QN];
        auto load = [&](int k) {
#pragma unroll
            for (int u = 0; u < QN; ++u)
                if (mine[u] && k < heads) {
                    const uint16_t* r = src + (share + shares * k) * a.qs[1] + from[u];
                    lo[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(r));
                    hi[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(r + H2));
                }
        };
        load(h0);
        angles(m);
        for (int k = h0; k < heads; k += par) {
            u32x4 l[QN], r[QN];
#pragma unroll
            for (int u = 0; u < QN; ++u) {
                l[u] = lo[u];
                r[u] = hi[u];
            }
            load(k + par);
#pragma unroll
            for (int u = 0; u < QN; ++u)
                if (mine[u]) {
                    if (AT || a.freq) {
                        const int at = (x0 + u * kThreads) / QC * H2 + 8 * c;
                        rotate8<AT>(l[u], r[u], cosv + at, sinv + at);
                    }
                    uint16_t* w = dst + (share + shares * k) * a.qos[1] + to[u];
                    __builtin_nontemporal_store(l[u], reinterpret_cast<u32x4*>(w));
                    __builtin_nontemporal_store(r[u], reinterpret_cast<u32x4*>(w + H2));
                }
        }
    };
    if (share >= a.kv_shares) return queries(share - a.kv_shares, a.q_shares);
    // ---- K and V of this share's heads
    const int cnt = a.counts ? min(max(ldc(a.counts, b), 0), a.T) : a.T;
    const int s1 = int(min(int64_t(len) + cnt - base, int64_t(kPage)));   // slots [s0, s1) are new
    const int m = s1 - s0;
    const int page = m > 0 ? cache_page(a.c, b, lp) : -1;
    if (page < 0) return;
    // K: columns 4 c .. 4 c + 3 of either half; V: columns 8 c .. 8 c + 7
    const int c = tid % C, r0 = tid / C;
    u32x2 klo[N], khi[N];
    u32x4 vraw[N];
    auto load = [&](int hk) {
        const uint16_t* kp = a.k + b * a.ks[0] + hk * a.ks[1];
        const uint16_t* vp = a.v + b * a.vs[0] + hk * a.vs[1];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int t = r0 + n * R;
            klo[n] = khi[n] = u32x2{};
            vraw[n] = u32x4{};
            if (t < m) {
                const uint16_t* kr = kp + (t0 + t) * a.ks[2] + 4 * c;
                klo[n] = *reinterpret_cast<const u32x2*>(kr);
                khi[n] = *reinterpret_cast<const u32x2*>(kr + H2);
                vraw[n] = *reinterpret_cast<const u32x4*>(vp + (t0 + t) * a.vs[2] + 8 * c);
            }
        }
    };
    load(share);
    angles(m);
    for (int hk = share; hk < a.c.Hkv; hk += a.kv_shares) {
        const int64_t at = int64_t(page) * a.c.Hkv + hk;
        uint8_t* kc = a.c.k + at * (kPage * D);
        uint8_t* vc = a.c.v + at * (kPage * D);
        const float kwas = s0 > 0 ? a.c.ks[at] : 0.f, vwas = s0 > 0 ? a.c.vs[at] : 0.f;
        // V rows are written 16 codes (slots 16 g ..) at a time; where slots of other
        // tokens lie among them they are read first, and the first of a thread's reads
        // is made here, so that one token does not wait for it at the end
        const int g1 = (s1 + 15) / 16, f0 = s0 / 16;
        u32x4 early = u32x4{};
        if (tid < D * (g1 - f0))
            early = *reinterpret_cast<const u32x4*>(vc + tid / (g1 - f0) * kPage + 16 * (f0 + tid % (g1 - f0)));
        float kx[N][8], vx[N][8];
        float km = 0.f, vm = 0.f;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int t = min(r0 + n * R, m - 1);   // (past the last: zeros)
            unpack8(u32x4{klo[n].x, klo[n].y, khi[n].x, khi[n].y}, kx[n]);
            unpack8(vraw[n], vx[n]);
            if (AT || a.freq) {
                const f32x4 cs = *reinterpret_cast<const f32x4*>(cosv + t * H2 + 4 * c);
                const f32x4 sn = *reinterpret_cast<const f32x4*>(sinv + t * H2 + 4 * c);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float x1 = kx[n][j], x2 = kx[n][4 + j];
                    rotate(x1, x2, cs[j], sn[j]);
                    if (AT && stays(sn[j])) continue;
                    kx[n][j] = x1;
                    kx[n][4 + j] = x2;
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                km = fmaxf(km, finite_abs(kx[n][j]));
                vm = fmaxf(vm, finite_abs(vx[n][j]));
            }
        }
        if (hk + a.kv_shares < a.c.Hkv) load(hk + a.kv_shares);
        km = wave_max(km);
        vm = wave_max(vm);
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
                for (int j = 0; j < 8; ++j)
                    vt[(8 * c + j) * (kPage + kPad) + s0 + t] = uint8_t(w[j >> 2] >> (8 * (j & 3)));
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
        // V rows from the tile; codes of other slots stay
        const bool vmove = s0 > 0 && vsc > vwas;
        const float vratio = vwas * vi;
        const int g0 = vmove ? 0 : f0;
        for (int x = tid; x < D * (g1 - g0); x += kThreads) {
            const int row = x / (g1 - g0), g = g0 + x % (g1 - g0);
            u32x4* dst = reinterpret_cast<u32x4*>(vc + row * kPage + 16 * g);
            u32x4 w = *reinterpret_cast<const u32x4*>(vt + row * (kPage + kPad) + 16 * g);
            if (16 * g < s0 || 16 * g + 16 > s1) {
                const u32x4 held = x == tid && !vmove ? early : *dst;
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
        __syncthreads();   // vt and red are read
    }
}

}  // namespace

hipError_t launch_cache_append(const AppendArgs& a, hipStream_t s) {
    TraceScope _t("cache_append", s);
    const dim3 g(unsigned(int64_t(a.c.B) * a.P * (a.kv_shares + a.q_shares))), t(kThreads);
    if (a.pos.at) {
        if (a.c.d == 128) hipLaunchKernelGGL((cache_append_kernel<128, true>), g, t, 0, s, a);
        else hipLaunchKernelGGL((cache_append_kernel<64, true>), g, t, 0, s, a);
    } else {
        if (a.c.d == 128) hipLaunchKernelGGL((cache_append_kernel<128, false>), g, t, 0, s, a);
        else hipLaunchKernelGGL((cache_append_kernel<64, false>), g, t, 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace msparse
