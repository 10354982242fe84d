// Attention over the paged cache, what its kernels share: the walk of a workgroup
// (its rows, the pages that they see, its chunk of them), a wave's rows, and the step
// of 16 or 32 rows over a page.  TREE: the rows are the nodes of a drafted tree, whose
// masks among each other come from words of bits.
#pragma once

#include "cache.h"

namespace msparse {

namespace {

constexpr int kMinChunk = 4;         // pages: one for each wave
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// D(16x16) += A(16x32) B(32x16), bf16: lane l supplies A[l % 16][8 (l / 16) ..] and
// B[8 (l / 16) ..][l % 16]; accumulator r of lane l is D[4 (l / 16) + r][l % 16].
__device__ __forceinline__ f32x4 mfma16(const u32x4& a, const u32x4& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                  0, 0);
}
// eight codes as bf16, times a power of two
__device__ __forceinline__ u32x4 codes_to_bf16(uint32_t lo, uint32_t hi, float power = 1.f) {
    u32x4 r;
    r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, power, false));
    r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, power, true));
    r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, power, false));
    r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, power, true));
    return r;
}
// 16 bits as bytes: 0xff where a bit is set
__device__ __forceinline__ u32x4 bytes_of(uint32_t bits) {
    u32x4 r;
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = (((bits >> (4 * j)) & 15) * 0x00204081u & 0x01010101u) * 0xffu;
    return r;
}
// x or-ed over the 16 lanes of a quarter of the wave
__device__ __forceinline__ uint32_t quarter_or(uint32_t x) {
    x |= __builtin_amdgcn_update_dpp(0, x, 0x121, 0xf, 0xf, false);   // the lane 1, 2, 4, 8 before, around
    x |= __builtin_amdgcn_update_dpp(0, x, 0x122, 0xf, 0xf, false);
    x |= __builtin_amdgcn_update_dpp(0, x, 0x124, 0xf, 0xf, false);
    x |= __builtin_amdgcn_update_dpp(0, x, 0x128, 0xf, 0xf, false);
    return x;
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

// Whether a row with this maximum and sum of weights saw no key.  (Logits that are all
// NaN leave the maximum at -inf too, but a sum that is NaN, as out and lse then are.)
__device__ __forceinline__ bool no_key(float mx, float l) { return mx == -INFINITY && l == 0.f; }

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
// tokens of sequence b, past the table too (page_list ends with the table)
__device__ __forceinline__ int32_t length_of(const CacheAttnArgs& a, int b) {
    return min(max(ldc(a.c.lens, b), 0), kMaxLength);
}
// positions of the first and last row of tile `tile` of a sequence of `len` tokens.  TREE:
// the rows' positions lie between that of the first node, `base`, and the last slot's, in any
// order; a tile without nodes has no pages.
struct TileRows {
    int32_t r0, len, p0, p1, base;
};
// nodes of sequence b's tree, the last of its len tokens
__device__ __forceinline__ int32_t nodes_of(const CacheAttnArgs& a, int b, int32_t len) {
    return min(a.counts ? min(max(ldc(a.counts, b), 0), a.T) : a.T, len);
}
template <bool TREE>
__device__ __forceinline__ TileRows tile_rows(const CacheAttnArgs& a, int b, int32_t len, int tile, int rows) {
    TileRows t;
    const int G = a.Hq / a.c.Hkv;
    t.len = len;
    t.r0 = tile * rows;
    if constexpr (TREE) {
        const int32_t nodes = nodes_of(a, b, len);
        t.base = len - nodes;
        const bool some = t.r0 < nodes * G;
        t.p0 = some ? t.base : -1;
        t.p1 = some ? len - 1 : -1;
        return t;
    }
    t.base = 0;
    t.p0 = t.len - a.T + t.r0 / G;
    t.p1 = t.len - a.T + min(t.r0 + rows, a.T * G) / G - (min(t.r0 + rows, a.T * G) % G == 0);
    return t;
}

// Inclusive sum over the wave's lanes, in registers (a sum through LDS permutes
// takes a microsecond of a workgroup's start).
__device__ __forceinline__ int32_t wave_scan(int32_t x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // the lane 1, 2, 4, 8 before, within 16
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // lane 15 of the 16 before, to rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // lane 31, to rows 2 and 3
    return x;
}
__device__ __forceinline__ PageList tile_pages(const CacheAttnArgs& a, const TileRows& t) {
    return page_list(t.p0, t.p1, a.W, a.S, a.c.width);
}
// A workgroup's chunk: `index` of the `count` of tile e, `pages` each, `first` being the
// slot of that tile's first; a tile without pages has one chunk too.
struct Chunk {
    int32_t e, first, count, index, pages;
};
// With few tiles their pages are cut into chunks of one length, so that whatever the
// raggedness the workgroups take as long: from the sum over all tiles and the number of
// chunks aimed at, a tile having one more at most.  FIT: the smallest length found that
// makes no more than `items` chunks, which run at once, or twice as many in two rounds,
// where one leaves many places empty (5 x 200 tokens of 32 over 4 heads at 8192, 65 tiles
// for 128 places: 324 -> 252 us).  False past the last chunk.  Every wave finds its own.
constexpr uint32_t kStartPages = 3;   // what a workgroup's start costs, in pages
template <bool FIT, bool TREE>
__device__ __forceinline__ bool find_chunk(const CacheAttnArgs& a, int rows, int item, int lane, Chunk& out) {
    const int E = a.c.B * a.tiles;
    auto pages_of = [&](int e) {
        return e < E ? tile_pages(a, tile_rows<TREE>(a, e / a.tiles, length_of(a, e / a.tiles), e % a.tiles, rows)).count : 0;
    };
    // the sum counts units of 2^unit pages, a tile's rounded up, so that it stays below 2^31
    auto units = [&](int np) { return int((uint32_t(np) + (1u << a.unit) - 1) >> a.unit); };
    const int own = pages_of(lane);   // the first 64 tiles are looked up once
    int sum = units(own);
    for (int e = 64 + lane; e < E; e += 64) sum += units(pages_of(e));
    const uint32_t total = __builtin_amdgcn_readlane(wave_scan(sum), 63);
    auto share = [&](int chunks) { return max(((total + chunks - 1) / chunks) << a.unit, uint32_t(kMinChunk)); };
    uint32_t pages = share(a.items);
    auto chunks_of = [&](int e0) {
        const uint32_t np = e0 == 0 ? own : pages_of(e0 + lane);
        return e0 + lane < E ? max(int((np + pages - 1) / pages), 1) : 0;
    };
    if constexpr (FIT) {
        auto fit = [&](int most) {   // (E <= most: one chunk each in the end)
            for (pages = share(most);; pages += max(pages / 16, 1u)) {
                int n = 0;
                for (int e0 = 0; e0 < E; e0 += 64) n += chunks_of(e0);
                if (__builtin_amdgcn_readlane(wave_scan(n), 63) <= most) return;
            }
        };
        fit(a.items);
        if (10 * pages > 13 * ((total / a.items) << a.unit)) {
            const uint32_t one = pages;
            fit(2 * a.items);
            if (2 * (pages + kStartPages) > one) pages = one;
        }
    }
    int base = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {
        const int n = chunks_of(e0);
        const int last = base + wave_scan(n);   // chunks up to this tile's end
        const uint64_t beyond = __ballot(item < last);
        if (beyond) {
            const int l = __builtin_ctzll(beyond);
            const int first = __builtin_amdgcn_readlane(last - n, l);
            out = Chunk{e0 + l, first, __builtin_amdgcn_readlane(n, l), item - first, int32_t(pages)};
            return true;
        }
        base = __builtin_amdgcn_readlane(last, 63);
    }
    return false;
}

// ---------------------------------------------------------------- one wave's rows
// RT tiles of 16 rows of a (sequence, KV head); lane (quarter g, m) owns row m of each.
template <int D, int RT>
struct CacheRows {
    static constexpr int KS = D / 32;      // k-steps of S^T
    static constexpr int KL = D / 64;      // 16-byte pieces of a token's key per lane
    static constexpr int ND = D / 16;      // column tiles of O^T
    u32x4 q[RT][KS];
    f32x4 o[RT][ND];
    float mx[RT], l[RT];
    int pos[RT];
    int wp0, wp1;   // positions of the first and last row; below 0: rows before the sequence, which see nothing
    int far;        // the last position that the window of no row reaches
    int b, r0;      // TREE: the sequence, the first row
};

// A value that the compiler does not know to be the same every time: what a rare branch computes from it is not
// computed ahead of the loop and held in registers.
__device__ __forceinline__ int opaque(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// rows from wr0 on (past the last: that one again) of R = T G
template <int D, int RT, bool TREE>
__device__ __forceinline__ void open_rows(const CacheAttnArgs& a, CacheRows<D, RT>& st, int b, int hk,
                                          const TileRows& tr, int wr0, int lane) {
    const int len = tr.len;
    const int g4 = lane >> 4, m = lane & 15, G = a.Hq / a.c.Hkv, R = a.T * G;
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        const int r = min(wr0 + 16 * x + m, R - 1);
        // (a row before the sequence: no difference to a key overflows)
        if constexpr (!TREE) st.pos[x] = max(len - a.T + r / G, -1);
        const uint16_t* qp = a.q + b * a.qs[0] + (hk * G + r % G) * a.qs[1] + (r / G) * a.qs[2];
#pragma unroll
        for (int s = 0; s < CacheRows<D, RT>::KS; ++s)
            st.q[x][s] = *reinterpret_cast<const u32x4*>(qp + 64 * (s >> 1) + 16 * g4 + 8 * (s & 1));
        st.mx[x] = -INFINITY;
        st.l[x] = 0.f;
#pragma unroll
        for (int y = 0; y < CacheRows<D, RT>::ND; ++y) st.o[x][y] = f32x4{};
    }
    if constexpr (TREE) {   // what all rows see in full ends before the first node
        st.wp0 = tr.base - 1;
        st.wp1 = len - 1;
        st.far = tr.base - a.W;
        st.b = b;
        st.r0 = wr0;
        return;
    }
    st.wp0 = len - a.T + min(wr0, R - 1) / G;
    st.wp1 = len - a.T + min(wr0 + 16 * RT - 1, R - 1) / G;
    st.far = max(st.wp0, 0) - a.W;
}

// Which of the 16 tokens from slot j on row r of sequence b's tree sees: of the context, which ends at `base`, what its
// position does (without a window that says nothing but that the row is behind it), of the nodes behind it (up to slot
// len) those of its bits.  A row behind the nodes sees nothing.
__device__ __forceinline__ uint32_t below(int n) { return n >= 16 ? 0xffffu : (1u << max(n, 0)) - 1; }
__device__ __forceinline__ uint32_t node_sees(const CacheAttnArgs& a, int b, int r, int j, int base, int len, int W, int S) {
    const int t = r / (a.Hq / a.c.Hkv), node = b * a.T + t;
    if (t >= len - base) return 0;
    const int pos = max(min(a.at ? a.at[node] : base, len - 1), base);
    uint32_t bits = 0;
    if (j < len && j + 15 >= base) {
        const int u = j - base, w = u >> 5;   // (u > -16: the word before the first is empty)
        const int32_t* row = a.seen + int64_t(node) * a.words;
        const uint32_t lo = w >= 0 && w < a.words ? uint32_t(row[w]) : 0;
        const uint32_t hi = w + 1 < a.words ? uint32_t(row[w + 1]) : 0;
        bits = uint32_t(((uint64_t(hi) << 32) | lo) >> (u & 31)) & below(len - j);
    }
    const uint32_t context = below(base - j);
    return (bits & ~context) | (context & (~below(max(pos - W + 1, 0) - j) | below(min(S - 1, pos) + 1 - j)));
}

// byte offsets of this lane's 16-byte operands in a page's codes of one head
__device__ __forceinline__ int key_offset(int t, int j, int lane, int D) {
    const int g4 = lane >> 4, m = lane & 15;
    return (16 * (m >> 2) + 4 * t + (m & 3)) * D + 64 * j + 16 * g4;
}
__device__ __forceinline__ int value_offset(int y, int lane) {
    return (16 * y + (lane & 15)) * kPage + 16 * (lane >> 4);
}

// Which of this lane's 16 tokens of a page at t0 some of the rows wp0 .. wp1 see, a
// byte each.  (Codes of free slots and of pages used before may stand for anything,
// NaN among it, which a weight of 0 would not remove.)
__device__ __forceinline__ u32x4 seen_bytes(int t0, int wp1, int far, int S, int lane) {
    u32x4 keep;
    const int lim = min(S - 1, wp1);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t byte = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int k = t0 + 16 * (lane >> 4) + 4 * j + e;
            if (k <= wp1 && (k > far || k <= lim)) byte |= 0xffu << (8 * e);
        }
        keep[j] = byte;
    }
    return keep;
}
// whether some of the rows wp0 .. wp1 do not see all of the page at t0
__device__ __forceinline__ bool partly(int t0, int wp0, int wp1, int W, int S) {
    return !(t0 <= wp0 - 63 && (t0 > wp1 - W || t0 < S - 63));
}

// Half p of a 16-token or 16-column operand: its codes converted, or read as bf16.
template <int PARTS>
__device__ __forceinline__ u32x4 operand(const u32x4* x, int p) {
    if constexpr (PARTS == 2) return x[p];
    const uint32_t lo = x[0][2 * p], hi = x[0][2 * p + 1];
    return codes_to_bf16(lo, hi);
}

// One page, its first token at position t0: key(t, j, p) and value(y, p) give this lane's
// operands, 16 codes (PARTS 1) or their halves as bf16 (2); keys_done() runs once the
// keys are used up, and clear(t0, seen) before the values of a page are that some row does not
// see in full: it clears the codes of the tokens that no row sees (TREE: this lane's 16 are
// given as bits; else they follow from t0).
template <int D, int RT, int TS, int YS, int PARTS, bool TREE, class Key, class Value, class Done, class Clear>
__device__ __forceinline__ void page_step(const CacheAttnArgs& a, CacheRows<D, RT>& st, int t0, float kscale,
                                          float vscale, int W, int S, int lane, Key key, Value value, Done keys_done,
                                          Clear clear) {
    constexpr int KL = CacheRows<D, RT>::KL, ND = CacheRows<D, RT>::ND;
    const int g4 = lane >> 4;
    const bool part = partly(t0, st.wp0, st.wp1, W, S);
    // ---- S^T, TS token tiles at a time: their operands are read a group ahead, and
    // the accumulators of a group take turns, as an MFMA that adds to the one before
    // it waits for it
    f32x4 s[RT][4];
    u32x4 kb[2][TS][KL][PARTS];
    auto read_k = [&](int set, int t) {
#pragma unroll
        for (int i = 0; i < TS; ++i)
#pragma unroll
            for (int j = 0; j < KL; ++j)
#pragma unroll
                for (int p = 0; p < PARTS; ++p) kb[set][i][j][p] = key(t + i, j, p);
    };
    read_k(0, 0);
#pragma unroll
    for (int t = 0; t < 4; t += TS) {
        const int set = (t / TS) & 1;
        if (t + TS < 4) read_k(set ^ 1, t + TS);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < TS; ++i)
#pragma unroll
            for (int x = 0; x < RT; ++x) s[x][t + i] = f32x4{};
#pragma unroll
        for (int j = 0; j < KL; ++j)
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int i = 0; i < TS; ++i) {
                    const u32x4 k = operand<PARTS>(kb[set][i][j], p);
#pragma unroll
                    for (int x = 0; x < RT; ++x) s[x][t + i] = mfma16(k, st.q[x][2 * j + p], s[x][t + i]);
                }
        __builtin_amdgcn_sched_barrier(0);
    }
    keys_done();
    __builtin_amdgcn_sched_barrier(0);
    if (part) {
        keep_branch();
        uint32_t some = 0;
#pragma unroll
        for (int x = 0; x < RT; ++x) {
            if constexpr (TREE) {
                const int l = opaque(lane);
                const uint32_t sees = node_sees(a, st.b, st.r0 + 16 * x + (l & 15), t0 + 16 * (l >> 4), st.wp0 + 1,
                                                st.wp1 + 1, W, S);
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (!((sees >> e) & 1)) s[x][e >> 2][e & 3] = -INFINITY;
                some |= sees;
                continue;
            }
            const int lim = min(S - 1, st.pos[x]);
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int j = t0 + 16 * g4 + 4 * t + r;
                    if (!(uint32_t(st.pos[x] - j) < uint32_t(W) || j <= lim)) s[x][t][r] = -INFINITY;
                }
        }
        if constexpr (TREE) {
            some = quarter_or(some);
            if (!__any(some)) vscale = 0.f;   // (a page that no row sees a token of: its scale may be anything too)
        }
        clear(t0, some);
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
        top = fmaxf(row_max(top) * kscale, st.mx[x]);
        if (__any(top > st.mx[x])) {
            const float alpha = st.mx[x] == -INFINITY ? 0.f : fast_exp2(st.mx[x] - top);
            st.l[x] *= alpha;
#pragma unroll
            for (int y = 0; y < ND; ++y) st.o[x][y] *= alpha;
            st.mx[x] = top;
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
        st.l[x] += sum;
    }
    // ---- O^T, YS column tiles at a time, likewise
    u32x4 vb[2][YS][PARTS];
    auto read_v = [&](int set, int y) {
#pragma unroll
        for (int i = 0; i < YS; ++i)
#pragma unroll
            for (int p = 0; p < PARTS; ++p) vb[set][i][p] = value(y + i, p);
    };
    read_v(0, 0);
#pragma unroll
    for (int y = 0; y < ND; y += YS) {
        const int set = (y / YS) & 1;
        if (y + YS < ND) read_v(set ^ 1, y + YS);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int i = 0; i < YS; ++i) {
                const u32x4 v = operand<PARTS>(vb[set][i], p);
#pragma unroll
                for (int x = 0; x < RT; ++x) st.o[x][y + i] = mfma16(v, pb[x][p], st.o[x][y + i]);
            }
        __builtin_amdgcn_sched_barrier(0);
    }
}

// What a workgroup walks: the entries [c0, c1) of its tile's pages.
struct Walk {
    Chunk ch;
    TileRows tr;
    PageList pl;
    int32_t b, hk, c0, c1;
};
// The rows' results: to out and lse, or, of a tile with several chunks, to this
// chunk's slot.  wr0: the wave's first row.
template <int D, int RT, bool TREE>
__device__ __forceinline__ void close_rows(const CacheAttnArgs& a, CacheRows<D, RT>& st, const Walk& k, int wr0,
                                           int rows, int lane) {
    constexpr int ND = CacheRows<D, RT>::ND;
    const int g4 = lane >> 4, m = lane & 15, G = a.Hq / a.c.Hkv, R = a.T * G;
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        const int r = wr0 + 16 * x + m;
        if (r >= R) continue;
        if (TREE && r / G >= k.tr.len - k.tr.base) {   // (pages without a mask have been added to it too)
            st.mx[x] = -INFINITY;
            st.l[x] = 0.f;
#pragma unroll
            for (int y = 0; y < ND; ++y) st.o[x][y] = f32x4{};
        }
        if (k.ch.count > 1) {
            const int64_t row = (int64_t(k.ch.first + k.ch.index) * a.c.Hkv + k.hk) * rows + (r - k.tr.r0);
            float* po = a.po + row * D + 4 * g4;
#pragma unroll
            for (int y = 0; y < ND; ++y) *reinterpret_cast<f32x4*>(po + 16 * y) = st.o[x][y];
            if (g4 == 0) {
                a.pml[2 * row] = st.mx[x];
                a.pml[2 * row + 1] = st.l[x];
            }
            continue;
        }
        const int t = r / G, h = k.hk * G + r % G;
        const bool empty = no_key(st.mx[x], st.l[x]);
        const float inv = empty ? 0.f : 1.f / st.l[x];
        uint16_t* op = a.out + k.b * a.os[0] + h * a.os[1] + t * a.os[2] + 4 * g4;
#pragma unroll
        for (int y = 0; y < ND; ++y) {
            u32x2 pk;
            pk.x = pack_bf16x2(st.o[x][y].x * inv, st.o[x][y].y * inv);
            pk.y = pack_bf16x2(st.o[x][y].z * inv, st.o[x][y].w * inv);
            *reinterpret_cast<u32x2*>(op + 16 * y) = pk;
        }
        if (a.lse && g4 == 0)
            a.lse[(int64_t(k.b) * a.Hq + h) * a.T + t] = empty ? -INFINITY : (st.mx[x] + fast_log2(st.l[x])) * kLn2;
    }
}

template <bool FIT, bool TREE>
__device__ __forceinline__ bool open_walk(const CacheAttnArgs& a, int rows, int lane, Walk& k) {
    k.hk = blockIdx.x % a.c.Hkv;
    const int item = blockIdx.x / a.c.Hkv, E = a.c.B * a.tiles;
    if (a.items > 0) {
        if (!find_chunk<FIT, TREE>(a, rows, item, lane, k.ch)) return false;
    } else {   // the tiles' first chunks, then their second ones, ..
        k.ch = Chunk{item % E, item % E * a.per_tile, 1, item / E, a.chunk};
    }
    k.b = k.ch.e / a.tiles;
    // (the clamp is a vector instruction; left in a vector register, the length takes the
    // positions that follow from it along, and they spill: 8 x 128K 210 us, so 226)
    k.tr = tile_rows<TREE>(a, k.b, __builtin_amdgcn_readfirstlane(length_of(a, k.b)), k.ch.e % a.tiles, rows);
    k.pl = tile_pages(a, k.tr);
    if (a.items == 0) {
        k.ch.count = max(int((int64_t(k.pl.count) + a.chunk - 1) / a.chunk), 1);
        if (k.ch.index >= k.ch.count) return false;
    }
    k.c0 = int(min(int64_t(k.ch.index) * k.ch.pages, int64_t(k.pl.count)));
    k.c1 = int(min(int64_t(k.c0) + k.ch.pages, int64_t(k.pl.count)));
    if (a.slots > 0 && k.hk == 0 && k.ch.index == 0 && threadIdx.x == 0) {
        a.info[2 * k.ch.e] = k.ch.first;
        a.info[2 * k.ch.e + 1] = k.ch.count;
    }
    return true;
}
// Pages and scales of the next 64 entries x, x + step, .. of a walk, one per lane:
// looked up together, then read lane by lane.  A lookup for each page on its way
// would put two dependent memory latencies into every step.
struct Pages {
    int32_t page;     // -1: the table has none
    float ks, vs;     // scales of the logits (in log2 units) and of the values
};
__device__ __forceinline__ Pages look_up(const CacheAttnArgs& a, const Walk& k, int x, int step, int lane) {
    const int e = x + step * lane;
    int32_t page = -1;
    if (e < k.c1) {
        const int index = k.pl.page(e);
        if (index < a.c.width) page = a.c.table[int64_t(k.b) * a.c.width + index];
        if (uint32_t(page) >= uint32_t(a.c.pages)) page = -1;
    }
    const int64_t at = int64_t(max(page, 0)) * a.c.Hkv + k.hk;
    // (The first stays above 0, as a masked logit times 0 would be NaN.  A missing page's
    // values weigh 0, whatever scale stands where it reads one; masked by its sign, as a
    // selection becomes a branch around the load: 8 x 128K 225 us, 209 so.)
    const float vs = __uint_as_float(__float_as_uint(a.c.vs[at]) & ~uint32_t(page >> 31));
    return Pages{page, fmaxf(a.c.ks[at] * (a.scale * kLog2e), 0x1p-126f), vs};
}
__device__ __forceinline__ int32_t page_at(const Pages& p, int i) { return __builtin_amdgcn_readlane(p.page, i); }
__device__ __forceinline__ float lane_value(float x, int i) {
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), i));
}
// position of a page's first token; a page that the table does not have lies beyond every row
__device__ __forceinline__ int page_start(int page, int index) { return page < 0 ? kMaxLength : kPage * index; }

}  // namespace

}  // namespace msparse
