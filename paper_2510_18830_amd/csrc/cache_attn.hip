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
// length whatever the batch's raggedness, joined by a second launch: 8 contexts of
// 13K to 128K tokens x 8 heads (1.32 GB) take 208 us, 6.4 TB/s; the join 5 us.  Many
// rows are bound by the products and exponentials: four waves take 32 rows each over
// the same pages, whose codes are converted once for all of them (4 x 200 tokens of 16
// over 2 heads in a window of 4096: 62 us, 7 of them the join's).
#include "cache_walk.h"
#include "tiles.h"
#include "trace.h"

#include <algorithm>

namespace msparse {

namespace {

constexpr int kThreads = 256;
constexpr int64_t kManyRows = 2048;  // rows from which the join takes one per group of lanes
constexpr int kWideWaves = 16;       // of a wide workgroup: four a SIMD, what the registers of head dim 64 allow
// workgroups of the kernel for many rows that run at once: two or three a CU
constexpr int64_t kRowsResident(int d) { return d == 128 ? 512 : 768; }
constexpr int64_t kLongTile = 128;   // pages that many workgroups take without a cut

// Up to 32 rows: the WAVES waves share them and take pages in turn, straight from
// memory to registers.  A page is read by one wave alone, once, hence past the
// caches (a plain read reaches 7.0 TB/s that way against 6.1).
constexpr int per_simd(int RT, int waves) { return waves == kWideWaves ? 4 : RT == 1 ? 3 : 2; }
template <int D, int RT, int WAVES, bool TREE>
__global__ void __launch_bounds__(64 * WAVES)
    __attribute__((amdgpu_waves_per_eu(per_simd(RT, WAVES), per_simd(RT, WAVES)))) cache_attn_kernel(CacheAttnArgs a) {
    constexpr int KL = CacheRows<D, RT>::KL, ND = CacheRows<D, RT>::ND, ROWS = 16 * RT;
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    __shared__ __attribute__((aligned(16))) float so[WAVES / 2][RT * ND * 4 * 64];
    __shared__ float sml[WAVES / 2][RT][2][64];
    Walk k;
    if (!open_walk<false, TREE>(a, ROWS, lane, k)) return;
    CacheRows<D, RT> st;
    open_rows<D, RT, TREE>(a, st, k.b, k.hk, k.tr, k.tr.r0, lane);
    u32x4 kr[4][KL], vr[ND];
    auto load_k = [&](int page) {
        const uint8_t* p = a.c.k + (int64_t(max(page, 0)) * a.c.Hkv + k.hk) * (kPage * D) + key_offset(0, 0, lane, D);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int j = 0; j < KL; ++j)
                kr[t][j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + 4 * t * D + 64 * j));
    };
    auto load_v = [&](int page) {
        const uint8_t* p = a.c.v + (int64_t(max(page, 0)) * a.c.Hkv + k.hk) * (kPage * D) + value_offset(0, lane);
#pragma unroll
        for (int y = 0; y < ND; ++y)
            vr[y] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + 16 * y * kPage));
    };
    // the next page's codes are requested as soon as this one's are used up
    constexpr int STEP = WAVES;
    for (int x0 = k.c0 + w; x0 < k.c1; x0 += 64 * STEP) {
        const Pages pages = look_up(a, k, x0, STEP, lane);
        const int n = min((k.c1 - x0 + STEP - 1) / STEP, 64);
        load_k(page_at(pages, 0));
        load_v(page_at(pages, 0));
        for (int i = 0; i < n; ++i) {
            const int next = page_at(pages, min(i + 1, 63));
            page_step<D, RT, RT == 1 ? 2 : 1, RT == 1 ? 4 : 2, 1, TREE>(
                a, st, page_start(page_at(pages, i), k.pl.page(x0 + i * STEP)), lane_value(pages.ks, i),
                lane_value(pages.vs, i), a.W, a.S, lane, [&](int t, int j, int) { return kr[t][j]; },
                [&](int y, int) { return vr[y]; },
                [&] {
                    if (i + 1 < n) load_k(next);
                },
                [&](int t0, uint32_t seen) {
                    const u32x4 keep = TREE ? bytes_of(seen) : seen_bytes(t0, st.wp1, st.far, a.S, lane);
#pragma unroll
                    for (int y = 0; y < ND; ++y) vr[y] &= keep;
                });
            if (i + 1 < n) load_v(next);
        }
    }
    // join the waves, by halves in a fixed order
#pragma unroll
    for (int x = 0; x < RT; ++x) st.l[x] = row_sum(st.l[x]);
#pragma unroll
    for (int half = WAVES / 2; half >= 1; half >>= 1) {
        if (w >= half && w < 2 * half) {
#pragma unroll
            for (int x = 0; x < RT; ++x) {
                sml[w - half][x][0][lane] = st.mx[x];
                sml[w - half][x][1][lane] = st.l[x];
#pragma unroll
                for (int y = 0; y < ND; ++y)
                    *reinterpret_cast<f32x4*>(&so[w - half][((x * ND + y) * 64 + lane) * 4]) = st.o[x][y];
            }
        }
        __syncthreads();
        if (w < half) {
#pragma unroll
            for (int x = 0; x < RT; ++x) {
                const float m1 = sml[w][x][0][lane], l1 = sml[w][x][1][lane];
                const float top = fmaxf(st.mx[x], m1);
                const float a0 = st.mx[x] == -INFINITY ? 0.f : fast_exp2(st.mx[x] - top);
                const float a1 = m1 == -INFINITY ? 0.f : fast_exp2(m1 - top);
                st.mx[x] = top;
                st.l[x] = st.l[x] * a0 + l1 * a1;
#pragma unroll
                for (int y = 0; y < ND; ++y)
                    st.o[x][y] = st.o[x][y] * a0 +
                                 *reinterpret_cast<const f32x4*>(&so[w][((x * ND + y) * 64 + lane) * 4]) * a1;
            }
        }
        __syncthreads();
    }
    if (w == 0) close_rows<D, RT, TREE>(a, st, k, k.tr.r0, ROWS, lane);
}

// More rows: each of the four waves takes 32 of its own through all pages of the
// chunk.  A page is read and converted once for the workgroup, a quarter a wave: from
// memory to registers two pages ahead, to bf16 operands in LDS one ahead.  (Codes staged
// in LDS and converted by every wave, which leaves room for three workgroups a CU: 14 x
// 127 tokens of 32 over 8 heads at 4551 270 us, so 194; 4 x 200 in a window 67, 62; 1 x
// 4096 at 8192 526, 499; 3 x 500 of 64 heads at 8192 534, 568; 1 x 16384 at 20480 3.52
// ms, 3.63.)
template <int D>
__global__ void __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(D == 128 ? 2 : 3, D == 128 ? 2 : 3)))
cache_attn_rows_kernel(CacheAttnArgs a) {
    constexpr int RT = 2, KL = CacheRows<D, RT>::KL, ND = CacheRows<D, RT>::ND, ROWS = 16 * RT * 4;
    constexpr int kOps = 4 * KL + ND, NV = ND / 4;   // operands of a page, 2 KB of bf16 each
    __shared__ __attribute__((aligned(16))) u32x4 buf[2][kOps][2][64];   // [page][operand][half][lane]
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Walk k;
    if (!open_walk<true, false>(a, ROWS, lane, k)) return;
    const int wr0 = k.tr.r0 + 16 * RT * w;
    CacheRows<D, RT> st;
    open_rows<D, RT, false>(a, st, k.b, k.hk, k.tr, wr0, lane);
    const bool live = wr0 < a.T * (a.Hq / a.c.Hkv);
    u32x4 kr[KL], vr[NV];   // this wave's codes of a page: the keys of the token tile w, the columns w, w + 4, ..
    auto load = [&](int page) {
        const int64_t at = (int64_t(max(page, 0)) * a.c.Hkv + k.hk) * (kPage * D);
        const uint8_t* kp = a.c.k + at + key_offset(w, 0, lane, D);
#pragma unroll
        for (int j = 0; j < KL; ++j) kr[j] = *reinterpret_cast<const u32x4*>(kp + 64 * j);
        const uint8_t* vp = a.c.v + at + value_offset(w, lane);
#pragma unroll
        for (int y = 0; y < NV; ++y) vr[y] = *reinterpret_cast<const u32x4*>(vp + 64 * y * kPage);
    };
    auto convert = [&](u32x4 (*b)[2][64], int t0) {
        if (partly(t0, k.tr.p0, k.tr.p1, a.W, a.S)) {
            keep_branch();
            const u32x4 keep = seen_bytes(t0, k.tr.p1, max(k.tr.p0, 0) - a.W, a.S, lane);
#pragma unroll
            for (int y = 0; y < NV; ++y) vr[y] &= keep;
        }
#pragma unroll
        for (int p = 0; p < 2; ++p) {
#pragma unroll
            for (int j = 0; j < KL; ++j) b[w * KL + j][p][lane] = operand<1>(&kr[j], p);
#pragma unroll
            for (int y = 0; y < NV; ++y) b[4 * KL + w + 4 * y][p][lane] = operand<1>(&vr[y], p);
        }
    };
    for (int x0 = k.c0; x0 < k.c1; x0 += 64) {
        const Pages pages = look_up(a, k, x0, 1, lane);
        const int n = min(k.c1 - x0, 64);
        auto start = [&](int i) { return page_start(page_at(pages, i), k.pl.page(x0 + i)); };
        // every page of the 64 before has been read: its last step ended with a barrier
        load(page_at(pages, 0));
        convert(buf[0], start(0));
        if (n > 1) load(page_at(pages, 1));
        __syncthreads();
        for (int i = 0; i < n; ++i) {
            if (i + 1 < n) convert(buf[(i + 1) & 1], start(i + 1));
            if (i + 2 < n) load(page_at(pages, i + 2));
            __builtin_amdgcn_sched_barrier(0);
            const u32x4 (*cur)[2][64] = buf[i & 1];
            const int t0 = start(i);
            if (live && t0 <= st.wp1 && (t0 + 63 > st.far || t0 < a.S))
                page_step<D, RT, 1, 2, 2, false>(
                    a, st, t0, lane_value(pages.ks, i), lane_value(pages.vs, i), a.W, a.S, lane,
                    [&](int t, int j, int p) { return cur[t * KL + j][p][lane]; },
                    [&](int y, int p) { return cur[4 * KL + y][p][lane]; }, [] {}, [](int, uint32_t) {});
            __builtin_amdgcn_sched_barrier(0);
            __syncthreads();
        }
    }
#pragma unroll
    for (int x = 0; x < RT; ++x) st.l[x] = row_sum(st.l[x]);
    if (live) close_rows<D, RT, false>(a, st, k, wr0, ROWS, lane);
}

// Joins a row's chunks.  D / 4 lanes hold a row; the kThreads / (D / 4) groups of a
// workgroup take a row each (MANY), or the chunks of one row in turn, so that a
// long context's hundreds of chunks are not one walk.  Both orders are fixed.
template <int D, bool MANY>
__global__ void __launch_bounds__(kThreads) cache_join_kernel(CacheAttnArgs a, int rows) {
    constexpr int C = D / 4, N = kThreads / C;
    __shared__ __attribute__((aligned(16))) float so[MANY ? 1 : N][D];
    __shared__ float sm[N], sl[N];
    const int G = a.Hq / a.c.Hkv, R = a.T * G;
    const int c = threadIdx.x % C, n = threadIdx.x / C;
    const int64_t at = MANY ? int64_t(blockIdx.x) * N + n : blockIdx.x;   // row of (sequence, KV head, row)
    if (at >= int64_t(a.c.B) * a.c.Hkv * R) return;
    const int r = int(at % R), hk = int(at / R % a.c.Hkv), b = int(at / R / a.c.Hkv);
    const int e = b * a.tiles + r / rows;
    const int first = a.info[2 * e], count = a.info[2 * e + 1];   // slots of the tile's chunks
    if (count <= 1) return;   // (the same for every thread unless MANY, which has no barrier)
    float mx = -INFINITY, l = 0.f;
    f32x4 o = f32x4{};
#pragma unroll 4
    for (int s = MANY ? 0 : n; s < count; s += MANY ? 1 : N) {
        const int64_t row = (int64_t(first + s) * a.c.Hkv + hk) * rows + r % rows;
        const float m1 = a.pml[2 * row], l1 = a.pml[2 * row + 1];
        const f32x4 x = *reinterpret_cast<const f32x4*>(a.po + row * D + 4 * c);
        const float top = fmaxf(mx, m1), use = top == -INFINITY ? 0.f : top;
        const float a0 = fast_exp2(mx - use), a1 = fast_exp2(m1 - use);
        mx = top;
        l = l * a0 + l1 * a1;
        o = o * a0 + x * a1;
    }
    if constexpr (!MANY) {
        *reinterpret_cast<f32x4*>(&so[n][4 * c]) = o;
        if (c == 0) {
            sm[n] = mx;
            sl[n] = l;
        }
        __syncthreads();
        if (n > 0) return;
        mx = -INFINITY;
#pragma unroll
        for (int s = 0; s < N; ++s) mx = fmaxf(mx, sm[s]);
        const float use = mx == -INFINITY ? 0.f : mx;
        l = 0.f;
        o = f32x4{};
#pragma unroll
        for (int s = 0; s < N; ++s) {
            const float f = fast_exp2(sm[s] - use);
            l += sl[s] * f;
            o += *reinterpret_cast<const f32x4*>(&so[s][4 * c]) * f;
        }
    }
    const bool empty = no_key(mx, l);
    const float inv = empty ? 0.f : 1.f / l;
    const int t = r / G, h = hk * G + r % G;
    u32x2 pk;
    pk.x = pack_bf16x2(o.x * inv, o.y * inv);
    pk.y = pack_bf16x2(o.z * inv, o.w * inv);
    *reinterpret_cast<u32x2*>(a.out + b * a.os[0] + h * a.os[1] + t * a.os[2] + 4 * c) = pk;
    if (a.lse && c == 0) a.lse[(int64_t(b) * a.Hq + h) * a.T + t] = empty ? -INFINITY : (mx + fast_log2(l)) * kLn2;
}

template <int D, bool TREE>
void launch_wide(const CacheAttnArgs& a, dim3 g, hipStream_t s) {
    if constexpr (D == 64)
        hipLaunchKernelGGL((cache_attn_kernel<64, 1, kWideWaves, TREE>), g, dim3(64 * kWideWaves), 0, s, a);
}

template <int D, bool TREE>
void launch(const CacheAttnArgs& a, const CacheAttnPlan& p, hipStream_t s) {
    const int64_t wgs = cache_attn_groups(p, a.c.B) * a.c.Hkv;
    const dim3 g(static_cast<unsigned>(wgs)), t(kThreads);
    {
        TraceScope _t(TREE ? "cache_tree_attn" : "cache_attn", s);
        if (p.wr == 4) {
            if constexpr (TREE) launch_tree_rows(a, p.rows, g, s);
            else hipLaunchKernelGGL((cache_attn_rows_kernel<D>), g, t, 0, s, a);
        }
        else if (p.wide) launch_wide<D, TREE>(a, g, s);
        else if (p.rt == 2) hipLaunchKernelGGL((cache_attn_kernel<D, 2, 4, TREE>), g, t, 0, s, a);
        else hipLaunchKernelGGL((cache_attn_kernel<D, 1, 4, TREE>), g, t, 0, s, a);
    }
    if (p.slots > 0) {
        TraceScope _t("cache_join", s);
        const int64_t rows = int64_t(a.c.B) * a.Hq * a.T;
        constexpr int N = kThreads / (D / 4);
        if (rows >= kManyRows)
            hipLaunchKernelGGL((cache_join_kernel<D, true>), dim3(unsigned((rows + N - 1) / N)), t, 0, s, a, p.rows);
        else
            hipLaunchKernelGGL((cache_join_kernel<D, false>), dim3(unsigned(rows)), t, 0, s, a, p.rows);
    }
}

}  // namespace

CacheAttnPlan cache_attn_plan(int64_t B, int64_t Hq, int64_t Hkv, int64_t T, int64_t width, int d, int64_t W,
                              int64_t S, bool tree) {
    CacheAttnPlan p{};
    const int64_t rows = Hq / Hkv * T;
    p.rt = rows <= 16 ? 1 : 2;
    // From 33 rows on one tile over four waves, also where some stay without rows (us, tiles
    // of 32 rows that walk the pages each -> this: 32 contexts of up to 16K, 28 over 4 heads,
    // 5 to 9 tokens 146-150 -> 112-116; 16 of up to 8K, 32 over 8, head dim 64, 9 to 16
    // tokens 46-49 -> 39-40; 4 of up to 8K, 16 over 2, 5 to 8 tokens 17.5-18.7 -> 17.9-19.4;
    // 64 of up to 2K, 32 over 4, head dim 64, 6 to 8 tokens 24.4 -> 29.6)
    // Trees take 64 at most in tiles of their own (as above 93-95 us, in tiles of 128 102-104).
    p.wr = rows <= 32 ? 1 : 4;
    p.rows = tree && p.wr == 4 && rows <= 64 ? 64 : 16 * p.rt * p.wr;
    p.tiles = int32_t((rows + p.rows - 1) / p.rows);
    // the most pages that a tile sees: the window of its tokens (of a tree's nodes: of any), the sinks' (what a plan
    // needs grows with them, so that one without a window has room for all)
    const int64_t span = tree ? T : std::min(T, p.rows / (Hq / Hkv) + 2);
    width = std::min(width, (W + span + 61) / kPage + 1 + (S + kPage - 1) / kPage);
    const int64_t e = B * p.tiles, groups = e * Hkv;
    // One chunk per row tile, where a cut would cost a short context more than it saves
    // (a join and half the walk: 64 contexts of 512 tokens, one KV head: 10.7 -> 8.7 us)
    p.per_tile = 1;
    p.chunk = INT32_MAX;
    if (width <= (p.wr == 4 ? kMinChunk : 2 * kMinChunk)) return p;
    // Or one workgroup of many waves, up to one a CU, which joins its pages by itself
    // (head dim 64, one to 16 rows; both in us, equal chunks -> this): one tile of 16 pages 9.2 ->
    // 8.0, 32 9.1 -> 9.7, 64 9.2 -> 13.4; 128 tiles of 32 16.2 -> 12.1, 64 21.5 -> 18.1,
    // 125 29.9 -> 29.7; 240 tiles (four waves each) of 32 14.4 -> 13.4, 64 27.4 -> 23.7.
    // With eight waves at head dim 128, or of 32 rows, it loses from 16 pages on.
    p.wide = d == 64 && p.rt == 1 && groups <= 256 && width <= (groups < 112 ? 2 * kWideWaves : kLongTile);
    if (p.wide) return p;
    if (groups < (p.wr == 4 ? 512 : width <= kLongTile ? 192 : 560)) {
        // Few tiles: equal chunks whatever the raggedness (find_chunk).  Where rows bound
        // the work, as many as run at once (512, 768, 1024 of them: 63, 72, 70 us for 4 x
        // 200 tokens of 16 over 2 heads in a window of 4096), where memory does, two
        // rounds of them (512, 768, 1024, 1536, 2048: 255, 236, 224, 211, 211 us for 8
        // contexts of up to 128K x 8 heads), each tile one more than its share at most.
        const int64_t aim = (p.wr == 4 ? kRowsResident(d) : p.rt == 1 ? 1536 : 768) / Hkv;
        p.even = tree && p.wr == 4;
        p.items = int32_t(std::max(p.wr == 4 ? aim : aim - e, p.even ? 1 : e));
        const int64_t most = p.wr == 4 ? 2 * int64_t(p.items) : p.items + e;
        p.slots = int32_t(p.even ? p.items + e : std::min(most, e * ((width + kMinChunk - 1) / kMinChunk)));
        while (e * ((width >> p.unit) + 1) > INT32_MAX / (p.even ? 2 : 1)) ++p.unit;   // (even: a run's end past all)
        return p;
    }
    // Many tiles fill the card by themselves; every wave's search for its chunk among
    // them, and the join, would cost more than even shares give (both in us, equal chunks
    // -> these): one token, 8 KV heads: 256 ragged contexts of up to 512 tokens 60 -> 37,
    // 1024 of 4096 952 -> 788, 4096 of 512 4207 -> 535, 64 of 4096 63 -> 69 (all of one
    // length 100 -> 90); of 16K: 52: 180 -> 213 (302 -> 325), 72: 245 -> 259 (466 -> 417),
    // 90: 330 -> 335 (736 -> 506).  Of 128 rows, from about a workgroup for every place on.
    // Contexts longer than kLongTile pages are still cut, at even lengths from the
    // table's width, so that one long context among short ones is not a walk of one
    // workgroup's; the slots of their chunks take about 1/2 GB at most.
    const int64_t most = p.wr == 4 ? std::min<int64_t>(16, 8192 / groups) : std::min<int64_t>(8, 32768 / groups);
    if (width > kLongTile && most > 1) {
        const int64_t least = p.wr == 4 ? kLongTile / 2 : kLongTile;
        p.chunk = int32_t(std::max(least, (width + most - 1) / most));
        p.per_tile = int32_t((width + p.chunk - 1) / p.chunk);
        p.slots = int32_t(e * p.per_tile);
    }
    return p;
}

hipError_t launch_cache_attn(const CacheAttnArgs& a, const CacheAttnPlan& p, hipStream_t s) {
    const bool tree = a.seen != nullptr;
    if (a.c.d == 128) tree ? launch<128, true>(a, p, s) : launch<128, false>(a, p, s);
    else tree ? launch<64, true>(a, p, s) : launch<64, false>(a, p, s);
    return hipGetLastError();
}

}  // namespace msparse
