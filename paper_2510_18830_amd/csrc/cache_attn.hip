// Attention of a sequence's newest tokens over the paged 8-bit cache.
//
// The T G rows of a KV head (row r: token r / G, head r % G of the group) are cut
// into tiles; a wave takes 16 or 32 rows through one page of 64 tokens at a time:
//   S^T = K Q^T      (16x16x32 bf16: A = 16 tokens' codes, B = the rows' queries)
//   online softmax   (a lane owns a row and 16 of the page's tokens)
//   O^T += V^T P^T   (A = 16 columns' codes, B = P straight from the S^T registers)
// e4m3 codes convert to bf16 exactly; a page's K scale is folded into the logits'
// factor and its V scale into P, in fp32.  The order in which tokens and columns
// enter the products is free as long as both operands share it, and is chosen so
// that every operand is 16 contiguous bytes of a page: lane (quarter g, m) reads
// key token 16 (m / 4) + 4 a + m % 4 for the S^T tile a, so its accumulators hold
// the tokens 16 g .. 16 g + 15, and those are the bytes of V's row it reads.  No
// LDS, no barrier, no exchange inside the walk but the row maximum's.
//
// One token per sequence is bound by the cache's bytes: waves walk pages with the
// next page's loads in flight, and long contexts are cut into chunks of equal
// length whatever the batch's raggedness, joined by a second launch.  Many rows
// are bound by the products and the conversions: four waves take rows of their
// own over the same pages.
#include "cache.h"
#include "trace.h"

#include <algorithm>

namespace msparse {

namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// D(16x16) += A(16x32) B(32x16), bf16: lane l supplies A[l % 16][8 (l / 16) ..] and
// B[8 (l / 16) ..][l % 16]; accumulator r of lane l is D[4 (l / 16) + r][l % 16].
__device__ __forceinline__ f32x4 mfma16(const u32x4& a, const u32x4& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                  0, 0);
}
// eight codes as bf16
__device__ __forceinline__ u32x4 codes_to_bf16(uint32_t lo, uint32_t hi) {
    u32x4 r;
    r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false));
    r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true));
    r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false));
    r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true));
    return r;
}
// x combined over the four lanes of a row (l, l ^ 16, l ^ 32, l ^ 48)
__device__ __forceinline__ float row_max(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return half_swap_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float row_sum(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return half_swap_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// The pages that the rows at the positions p0 .. p1 (p1 >= 0) see: the sinks'
// pages, then those of the window.
struct PageList {
    int32_t sinks, lo, count;
    __device__ __forceinline__ int32_t page(int x) const { return x < sinks ? x : lo + x - sinks; }
};
__device__ __forceinline__ PageList page_list(int p0, int p1, int W, int S, int width) {
    PageList l{0, 0, 0};
    if (p1 < 0) return l;
    const int end = min((p1 >> 6) + 1, width);
    l.lo = min(max(max(p0, 0) - W + 1, 0) >> 6, end);
    l.sinks = min(min(int((int64_t(S) + 63) >> 6), l.lo), end);
    l.count = l.sinks + end - l.lo;
    return l;
}
// positions of the first and last row of tile `tile` of sequence b
struct TileRows {
    int32_t r0, len, p0, p1;
};
__device__ __forceinline__ TileRows tile_rows(const CacheAttnArgs& a, int b, int tile, int rows) {
    TileRows t;
    const int G = a.Hq / a.c.Hkv;
    t.len = min(max(ldc(a.c.lens, b), 0), a.c.width * kPage);
    t.r0 = tile * rows;
    t.p0 = t.len - a.T + t.r0 / G;
    t.p1 = t.len - a.T + min(t.r0 + rows, a.T * G) / G - (min(t.r0 + rows, a.T * G) % G == 0);
    return t;
}

// Which tile and which of its chunks workgroup `item` takes: chunk = the pages a
// chunk holds, from the pages of all tiles and the chunks aimed at; first = the
// number of the tile's first chunk.  False past the last one.
struct Chunk {
    int32_t e, first, count, index, pages;
};
__device__ bool find_chunk(const CacheAttnArgs& a, int rows, int item, Chunk& out) {
    __shared__ int64_t sum[kThreads / 64];
    __shared__ int32_t sh[kThreads / 64];
    __shared__ Chunk found;
    const int tid = threadIdx.x, E = a.c.B * a.tiles;
    auto pages_of = [&](int e) {
        const TileRows t = tile_rows(a, e / a.tiles, e % a.tiles, rows);
        return page_list(t.p0, t.p1, a.W, a.S, a.c.width).count;
    };
    int64_t mine = 0;
    for (int e = tid; e < E; e += kThreads) mine += pages_of(e);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mine += __shfl_xor(mine, o);
    if ((tid & 63) == 0) sum[tid >> 6] = mine;
    if (tid == 0) found.count = 0;
    __syncthreads();
    const int64_t total = sum[0] + sum[1] + sum[2] + sum[3];
    const int chunk = int(max((total + a.items - 1) / a.items, int64_t(4)));
    int base = 0;
    for (int e0 = 0; e0 < E && base <= item; e0 += kThreads) {
        const int e = e0 + tid;
        const int np = e < E ? pages_of(e) : 0;
        const int n = e < E ? max((np + chunk - 1) / chunk, 1) : 0;
        int x = n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(x, o);
            if ((tid & 63) >= o) x += y;
        }
        if ((tid & 63) == 63) sh[tid >> 6] = x;
        __syncthreads();
        int before = base;
        for (int w = 0; w < (tid >> 6); ++w) before += sh[w];
        const int first = before + x - n;
        if (n > 0 && item >= first && item < first + n) found = Chunk{e, first, n, item - first, chunk};
        base += sh[0] + sh[1] + sh[2] + sh[3];
        __syncthreads();
    }
    out = found;
    return found.count > 0;
}

// RT tiles of 16 rows per wave; WR = 4: the waves take rows of their own, 1: they
// share the rows and take pages in turn.
template <int D, int RT, int WR>
__global__ void __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, RT == 1 ? 3 : 2)))
cache_attn_kernel(CacheAttnArgs a) {
    constexpr int KS = D / 32;      // k-steps of S^T
    constexpr int KL = D / 64;      // 16-byte loads of a token's key per lane
    constexpr int ND = D / 16;      // column tiles of O^T
    constexpr int ROWS = 16 * RT * WR;
    const int tid = threadIdx.x, lane = tid & 63, g4 = lane >> 4, m = lane & 15;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int G = a.Hq / a.c.Hkv, R = a.T * G;
    const int hk = blockIdx.x % a.c.Hkv;
    Chunk ch{};
    if (a.items > 0) {
        if (!find_chunk(a, ROWS, blockIdx.x / a.c.Hkv, ch)) return;
        ch.e = __builtin_amdgcn_readfirstlane(ch.e);
        ch.first = __builtin_amdgcn_readfirstlane(ch.first);
        ch.count = __builtin_amdgcn_readfirstlane(ch.count);
        ch.index = __builtin_amdgcn_readfirstlane(ch.index);
        ch.pages = __builtin_amdgcn_readfirstlane(ch.pages);
    } else {
        ch.e = blockIdx.x / a.c.Hkv;
        ch.count = 1;
        ch.pages = INT32_MAX;
    }
    const int b = ch.e / a.tiles;
    const TileRows tr = tile_rows(a, b, ch.e % a.tiles, ROWS);
    const PageList pl = page_list(tr.p0, tr.p1, a.W, a.S, a.c.width);
    const int c0 = int(min(int64_t(ch.index) * ch.pages, int64_t(pl.count)));
    const int c1 = int(min(int64_t(c0) + ch.pages, int64_t(pl.count)));
    if (a.items > 0 && hk == 0 && ch.index == 0 && tid == 0) {
        a.info[2 * ch.e] = ch.first;
        a.info[2 * ch.e + 1] = ch.count;
    }
    // this wave's rows
    const int wr0 = tr.r0 + (WR > 1 ? 16 * RT * w : 0);
    int pos[RT];
    u32x4 q[RT][KS];
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        const int r = min(wr0 + 16 * x + m, R - 1);
        pos[x] = tr.len - a.T + r / G;
        const uint16_t* qp = a.q + b * a.qs[0] + (hk * G + r % G) * a.qs[1] + (r / G) * a.qs[2];
#pragma unroll
        for (int s = 0; s < KS; ++s)
            q[x][s] = *reinterpret_cast<const u32x4*>(qp + 64 * (s >> 1) + 16 * g4 + 8 * (s & 1));
    }
    const int wp0 = tr.len - a.T + min(wr0, R - 1) / G;       // below 0: rows before the sequence, which see nothing
    const int wp1 = tr.len - a.T + min(wr0 + 16 * RT - 1, R - 1) / G;
    f32x4 o[RT][ND];
    float mx[RT], l[RT];
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        mx[x] = -INFINITY;
        l[x] = 0.f;
#pragma unroll
        for (int y = 0; y < ND; ++y) o[x][y] = f32x4{};
    }
    const float c2 = a.scale * kLog2e;
    u32x4 kr[4][KL], vr[ND];
    auto load_k = [&](int page) {
        const uint8_t* p = a.c.k + (int64_t(page) * a.c.Hkv + hk) * (kPage * D) + (16 * (m >> 2) + (m & 3)) * D + 16 * g4;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int j = 0; j < KL; ++j) kr[t][j] = *reinterpret_cast<const u32x4*>(p + 4 * t * D + 64 * j);
    };
    auto load_v = [&](int page) {
        const uint8_t* p = a.c.v + (int64_t(page) * a.c.Hkv + hk) * (kPage * D) + m * kPage + 16 * g4;
#pragma unroll
        for (int y = 0; y < ND; ++y) vr[y] = *reinterpret_cast<const u32x4*>(p + 16 * y * kPage);
    };
    const int far = max(wp0, 0) - a.W;   // the last position that the window of no row reaches
    constexpr int STEP = WR > 1 ? 1 : kThreads / 64;
    // the next page's codes are requested as soon as this one's are used up
    int page = -1;
    int x0 = c0 + (WR > 1 ? 0 : w);
    if (x0 < c1) {
        page = cache_page(a.c, b, pl.page(x0));
        load_k(max(page, 0));
        load_v(max(page, 0));
    }
    for (; x0 < c1; x0 += STEP) {
        // a page that the table does not have lies beyond every row
        const int t0 = page < 0 ? kMaxWidth * kPage : 64 * pl.page(x0);
        const bool more = x0 + STEP < c1;
        const int next = more ? cache_page(a.c, b, pl.page(x0 + STEP)) : -1;
        const bool part = !(t0 <= wp0 - 63 && (t0 > wp1 - a.W || t0 < a.S - 63));
        const int64_t at = int64_t(max(page, 0)) * a.c.Hkv + hk;
        // (kept above 0: a masked logit times 0 would be NaN)
        const float kscale = fmaxf(ldc(a.c.ks, at) * c2, 0x1p-126f), vscale = ldc(a.c.vs, at);
        // ---- S^T
        f32x4 s[RT][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int x = 0; x < RT; ++x) s[x][t] = f32x4{};
#pragma unroll
            for (int j = 0; j < KL; ++j) {
                const uint32_t k0 = kr[t][j].x, k1 = kr[t][j].y, k2 = kr[t][j].z, k3 = kr[t][j].w;
                const u32x4 lo = codes_to_bf16(k0, k1), hi = codes_to_bf16(k2, k3);
#pragma unroll
                for (int x = 0; x < RT; ++x) {
                    s[x][t] = mfma16(lo, q[x][2 * j], s[x][t]);
                    s[x][t] = mfma16(hi, q[x][2 * j + 1], s[x][t]);
                }
            }
            __builtin_amdgcn_sched_barrier(0);   // one token tile's operands at a time
        }
        if (more) load_k(max(next, 0));
        __builtin_amdgcn_sched_barrier(0);
        if (part) {
            keep_branch();
#pragma unroll
            for (int x = 0; x < RT; ++x) {
                const int lim = min(a.S - 1, pos[x]);
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int j = t0 + 16 * g4 + 4 * t + r;
                        if (!(uint32_t(pos[x] - j) < uint32_t(a.W) || j <= lim)) s[x][t][r] = -INFINITY;
                    }
            }
            // codes of tokens that no row sees (free slots, pages reused) may stand
            // for anything, NaN among it, which a weight of 0 would not remove
            u32x4 keep;
            const int lim = min(a.S - 1, wp1);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t byte = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int k = t0 + 16 * g4 + 4 * j + e;
                    if (k <= wp1 && (k > far || k <= lim)) byte |= 0xffu << (8 * e);
                }
                keep[j] = byte;
            }
#pragma unroll
            for (int y = 0; y < ND; ++y) vr[y] &= keep;
        }
        // ---- softmax
        u32x4 pb[RT][2];
#pragma unroll
        for (int x = 0; x < RT; ++x) {
            float top = -INFINITY;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) top = fmaxf(top, s[x][t][r]);
            top = fmaxf(row_max(top) * kscale, mx[x]);
            if (__any(top > mx[x])) {
                const float alpha = mx[x] == -INFINITY ? 0.f : fast_exp2(mx[x] - top);
                l[x] *= alpha;
#pragma unroll
                for (int y = 0; y < ND; ++y) o[x][y] *= alpha;
                mx[x] = top;
            }
            const float use = top == -INFINITY ? 0.f : top;
            float sum = 0.f;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                float p[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    p[r] = fast_exp2(__builtin_fmaf(s[x][t][r], kscale, -use));
                    sum += p[r];
                }
                pb[x][t >> 1][2 * (t & 1)] = pack_bf16x2(p[0] * vscale, p[1] * vscale);
                pb[x][t >> 1][2 * (t & 1) + 1] = pack_bf16x2(p[2] * vscale, p[3] * vscale);
            }
            l[x] += sum;
        }
        // ---- O^T
#pragma unroll
        for (int y = 0; y < ND; ++y) {
            const uint32_t v0 = vr[y].x, v1 = vr[y].y, v2 = vr[y].z, v3 = vr[y].w;
            const u32x4 lo = codes_to_bf16(v0, v1), hi = codes_to_bf16(v2, v3);
#pragma unroll
            for (int x = 0; x < RT; ++x) {
                o[x][y] = mfma16(lo, pb[x][0], o[x][y]);
                o[x][y] = mfma16(hi, pb[x][1], o[x][y]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (more) load_v(max(next, 0));
        page = next;
    }
#pragma unroll
    for (int x = 0; x < RT; ++x) l[x] = row_sum(l[x]);
    // ---- join the waves of a shared row tile: a fixed order, by halves
    if constexpr (WR == 1) {
        __shared__ __attribute__((aligned(16))) float so[2][RT * ND * 4 * 64];
        __shared__ float sml[2][RT][2][64];
#pragma unroll
        for (int half = 2; half >= 1; half >>= 1) {
            if (w >= half && w < 2 * half) {
#pragma unroll
                for (int x = 0; x < RT; ++x) {
                    sml[w - half][x][0][lane] = mx[x];
                    sml[w - half][x][1][lane] = l[x];
#pragma unroll
                    for (int y = 0; y < ND; ++y)
                        *reinterpret_cast<f32x4*>(&so[w - half][((x * ND + y) * 64 + lane) * 4]) = o[x][y];
                }
            }
            __syncthreads();
            if (w < half) {
#pragma unroll
                for (int x = 0; x < RT; ++x) {
                    const float m1 = sml[w][x][0][lane], l1 = sml[w][x][1][lane];
                    const float top = fmaxf(mx[x], m1);
                    const float a0 = mx[x] == -INFINITY ? 0.f : fast_exp2(mx[x] - top);
                    const float a1 = m1 == -INFINITY ? 0.f : fast_exp2(m1 - top);
                    mx[x] = top;
                    l[x] = l[x] * a0 + l1 * a1;
#pragma unroll
                    for (int y = 0; y < ND; ++y)
                        o[x][y] = o[x][y] * a0 + *reinterpret_cast<const f32x4*>(&so[w][((x * ND + y) * 64 + lane) * 4]) * a1;
                }
            }
            __syncthreads();
        }
        if (w != 0) return;
    }
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        const int r = wr0 + 16 * x + m;
        if (r >= R) continue;
        if (ch.count > 1) {
            const int64_t row = (int64_t(ch.first + ch.index) * a.c.Hkv + hk) * ROWS + (r - tr.r0);
            float* po = a.po + row * D + 4 * g4;
#pragma unroll
            for (int y = 0; y < ND; ++y) *reinterpret_cast<f32x4*>(po + 16 * y) = o[x][y];
            if (g4 == 0) {
                a.pml[2 * row] = mx[x];
                a.pml[2 * row + 1] = l[x];
            }
            continue;
        }
        const int t = r / G, h = hk * G + r % G;
        const bool empty = mx[x] == -INFINITY;
        const float inv = empty ? 0.f : 1.f / l[x];
        uint16_t* op = a.out + b * a.os[0] + h * a.os[1] + t * a.os[2] + 4 * g4;
#pragma unroll
        for (int y = 0; y < ND; ++y) {
            u32x2 pk;
            pk.x = pack_bf16x2(o[x][y].x * inv, o[x][y].y * inv);
            pk.y = pack_bf16x2(o[x][y].z * inv, o[x][y].w * inv);
            *reinterpret_cast<u32x2*>(op + 16 * y) = pk;
        }
        if (a.lse && g4 == 0)
            a.lse[(int64_t(b) * a.Hq + h) * a.T + t] = empty ? -INFINITY : (mx[x] + fast_log2(l[x])) * kLn2;
    }
}

// Joins the chunks of one row, in order: groups of D / 4 lanes take chunks in turn.
template <int D>
__global__ void __launch_bounds__(kThreads) cache_join_kernel(CacheAttnArgs a, int rows) {
    constexpr int C = D / 4, N = kThreads / C;
    __shared__ __attribute__((aligned(16))) float so[N][D];
    __shared__ float sm[N], sl[N];
    const int G = a.Hq / a.c.Hkv, R = a.T * G;
    const int r = blockIdx.x % R, hk = blockIdx.x / R % a.c.Hkv, b = blockIdx.x / (R * a.c.Hkv);
    const int e = b * a.tiles + r / rows;
    const int first = a.info[2 * e], count = a.info[2 * e + 1];
    if (count <= 1) return;
    const int c = threadIdx.x % C, n = threadIdx.x / C;
    float mx = -INFINITY, l = 0.f;
    f32x4 o = f32x4{};
    for (int s = n; s < count; s += N) {
        const int64_t row = (int64_t(first + s) * a.c.Hkv + hk) * rows + r % rows;
        const float m1 = a.pml[2 * row], l1 = a.pml[2 * row + 1];
        const f32x4 x = *reinterpret_cast<const f32x4*>(a.po + row * D + 4 * c);
        const float top = fmaxf(mx, m1);
        if (top == -INFINITY) continue;
        const float a0 = fast_exp2(mx - top), a1 = fast_exp2(m1 - top);
        mx = top;
        l = l * a0 + l1 * a1;
        o = o * a0 + x * a1;
    }
    *reinterpret_cast<f32x4*>(&so[n][4 * c]) = o;
    if (c == 0) {
        sm[n] = mx;
        sl[n] = l;
    }
    __syncthreads();
    if (n > 0) return;
    float top = -INFINITY;
#pragma unroll
    for (int s = 0; s < N; ++s) top = fmaxf(top, sm[s]);
    float sum = 0.f;
    o = f32x4{};
    if (top != -INFINITY)
#pragma unroll
        for (int s = 0; s < N; ++s) {
            const float f = fast_exp2(sm[s] - top);
            sum += sl[s] * f;
            o += *reinterpret_cast<const f32x4*>(&so[s][4 * c]) * f;
        }
    const bool empty = top == -INFINITY;
    const float inv = empty ? 0.f : 1.f / sum;
    const int t = r / G, h = hk * G + r % G;
    u32x2 pk;
    pk.x = pack_bf16x2(o.x * inv, o.y * inv);
    pk.y = pack_bf16x2(o.z * inv, o.w * inv);
    *reinterpret_cast<u32x2*>(a.out + b * a.os[0] + h * a.os[1] + t * a.os[2] + 4 * c) = pk;
    if (a.lse && c == 0) a.lse[(int64_t(b) * a.Hq + h) * a.T + t] = empty ? -INFINITY : (top + fast_log2(sum)) * kLn2;
}

template <int D>
void launch(const CacheAttnArgs& a, const CacheAttnPlan& p, hipStream_t s) {
    const int64_t wgs = (p.items > 0 ? int64_t(p.slots) : int64_t(a.c.B) * p.tiles) * a.c.Hkv;
    const dim3 g(static_cast<unsigned>(wgs)), t(kThreads);
    {
        TraceScope _t("cache_attn", s);
        if (p.wr == 4) hipLaunchKernelGGL((cache_attn_kernel<D, 2, 4>), g, t, 0, s, a);
        else if (p.rt == 2) hipLaunchKernelGGL((cache_attn_kernel<D, 2, 1>), g, t, 0, s, a);
        else hipLaunchKernelGGL((cache_attn_kernel<D, 1, 1>), g, t, 0, s, a);
    }
    if (p.items > 0) {
        TraceScope _t("cache_join", s);
        const dim3 gj(unsigned(int64_t(a.c.B) * a.Hq * a.T));
        hipLaunchKernelGGL((cache_join_kernel<D>), gj, t, 0, s, a, p.rows);
    }
}

}  // namespace

CacheAttnPlan cache_attn_plan(int64_t B, int64_t Hq, int64_t Hkv, int64_t T, int64_t width) {
    CacheAttnPlan p{};
    const int64_t rows = Hq / Hkv * T;
    p.rt = rows <= 16 ? 1 : 2;
    p.wr = rows <= 32 ? 1 : 4;
    p.rows = 16 * p.rt * p.wr;
    p.tiles = int32_t((rows + p.rows - 1) / p.rows);
    const int64_t e = B * p.tiles;
    constexpr int64_t kItems = 768;
    if (width > 4 && e * Hkv < 2 * kItems) {
        p.items = int32_t(std::max<int64_t>(1, kItems / Hkv));
        p.slots = int32_t(std::min(p.items + e, e * ((width + 3) / 4)));
    }
    return p;
}

hipError_t launch_cache_attn(const CacheAttnArgs& a, const CacheAttnPlan& p, hipStream_t s) {
    if (a.c.d == 128) launch<128>(a, p, s);
    else launch<64>(a, p, s);
    return hipGetLastError();
}

}  // namespace msparse
