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
#include "cache.h"
#include "tiles.h"
#include "trace.h"

#include <algorithm>

namespace msparse {

namespace {

constexpr int kThreads = 256;
constexpr int64_t kManyRows = 2048;  // rows from which the join takes one per group of lanes
constexpr int kMinChunk = 4;         // pages: one for each wave
constexpr int kWideWaves = 16;       // of a wide workgroup: four a SIMD, what the registers of head dim 64 allow
// workgroups of the kernel for many rows that run at once: two or three a CU
constexpr int64_t kRowsResident(int d) { return d == 128 ? 512 : 768; }
constexpr int64_t kLongTile = 128;   // pages that many workgroups take without a cut
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
// positions of the first and last row of tile `tile` of a sequence of `len` tokens
struct TileRows {
    int32_t r0, len, p0, p1;
};
__device__ __forceinline__ TileRows tile_rows(const CacheAttnArgs& a, int32_t len, int tile, int rows) {
    TileRows t;
    const int G = a.Hq / a.c.Hkv;
    t.len = len;
    t.r0 = tile * rows;
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
template <bool FIT>
__device__ __forceinline__ bool find_chunk(const CacheAttnArgs& a, int rows, int item, int lane, Chunk& out) {
    const int E = a.c.B * a.tiles;
    auto pages_of = [&](int e) {
        return e < E ? tile_pages(a, tile_rows(a, length_of(a, e / a.tiles), e % a.tiles, rows)).count : 0;
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
};

// rows from wr0 on (past the last: that one again) of R = T G
template <int D, int RT>
__device__ __forceinline__ void open_rows(const CacheAttnArgs& a, CacheRows<D, RT>& st, int b, int hk, int len, int wr0,
                                          int lane) {
    const int g4 = lane >> 4, m = lane & 15, G = a.Hq / a.c.Hkv, R = a.T * G;
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        const int r = min(wr0 + 16 * x + m, R - 1);
        st.pos[x] = max(len - a.T + r / G, -1);   // (a row before the sequence: no difference to a key overflows)
        const uint16_t* qp = a.q + b * a.qs[0] + (hk * G + r % G) * a.qs[1] + (r / G) * a.qs[2];
#pragma unroll
        for (int s = 0; s < CacheRows<D, RT>::KS; ++s)
            st.q[x][s] = *reinterpret_cast<const u32x4*>(qp + 64 * (s >> 1) + 16 * g4 + 8 * (s & 1));
        st.mx[x] = -INFINITY;
        st.l[x] = 0.f;
#pragma unroll
        for (int y = 0; y < CacheRows<D, RT>::ND; ++y) st.o[x][y] = f32x4{};
    }
    st.wp0 = len - a.T + min(wr0, R - 1) / G;
    st.wp1 = len - a.T + min(wr0 + 16 * RT - 1, R - 1) / G;
    st.far = max(st.wp0, 0) - a.W;
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
// keys are used up, and clear(t0) before the values of a page are that some row does not
// see in full: it clears the codes of the tokens that no row sees.
template <int D, int RT, int TS, int YS, int PARTS, class Key, class Value, class Done, class Clear>
__device__ __forceinline__ void page_step(CacheRows<D, RT>& st, int t0, float kscale, float vscale, int W, int S,
                                          int lane, Key key, Value value, Done keys_done, Clear clear) {
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
#pragma unroll
        for (int x = 0; x < RT; ++x) {
            const int lim = min(S - 1, st.pos[x]);
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int j = t0 + 16 * g4 + 4 * t + r;
                    if (!(uint32_t(st.pos[x] - j) < uint32_t(W) || j <= lim)) s[x][t][r] = -INFINITY;
                }
        }
        clear(t0);
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
template <int D, int RT>
__device__ __forceinline__ void close_rows(const CacheAttnArgs& a, const CacheRows<D, RT>& st, const Walk& k, int wr0,
                                           int rows, int lane) {
    constexpr int ND = CacheRows<D, RT>::ND;
    const int g4 = lane >> 4, m = lane & 15, G = a.Hq / a.c.Hkv, R = a.T * G;
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        const int r = wr0 + 16 * x + m;
        if (r >= R) continue;
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

template <bool FIT>
__device__ __forceinline__ bool open_walk(const CacheAttnArgs& a, int rows, int lane, Walk& k) {
    k.hk = blockIdx.x % a.c.Hkv;
    const int item = blockIdx.x / a.c.Hkv, E = a.c.B * a.tiles;
    if (a.items > 0) {
        if (!find_chunk<FIT>(a, rows, item, lane, k.ch)) return false;
    } else {   // the tiles' first chunks, then their second ones, ..
        k.ch = Chunk{item % E, item % E * a.per_tile, 1, item / E, a.chunk};
    }
    k.b = k.ch.e / a.tiles;
    // (the clamp is a vector instruction; left in a vector register, the length takes the
    // positions that follow from it along, and they spill: 8 x 128K 210 us, so 226)
    k.tr = tile_rows(a, __builtin_amdgcn_readfirstlane(length_of(a, k.b)), k.ch.e % a.tiles, rows);
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

// Up to 32 rows: the WAVES waves share them and take pages in turn, straight from
// memory to registers.  A page is read by one wave alone, once, hence past the
// caches (a plain read reaches 7.0 TB/s that way against 6.1).
constexpr int per_simd(int RT, int waves) { return waves == kWideWaves ? 4 : RT == 1 ? 3 : 2; }
template <int D, int RT, int WAVES>
__global__ void __launch_bounds__(64 * WAVES)
    __attribute__((amdgpu_waves_per_eu(per_simd(RT, WAVES), per_simd(RT, WAVES)))) cache_attn_kernel(CacheAttnArgs a) {
    constexpr int KL = CacheRows<D, RT>::KL, ND = CacheRows<D, RT>::ND, ROWS = 16 * RT;
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    __shared__ __attribute__((aligned(16))) float so[WAVES / 2][RT * ND * 4 * 64];
    __shared__ float sml[WAVES / 2][RT][2][64];
    Walk k;
    if (!open_walk<false>(a, ROWS, lane, k)) return;
    CacheRows<D, RT> st;
    open_rows(a, st, k.b, k.hk, k.tr.len, k.tr.r0, lane);
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
            page_step<D, RT, RT == 1 ? 2 : 1, RT == 1 ? 4 : 2, 1>(
                st, page_start(page_at(pages, i), k.pl.page(x0 + i * STEP)), lane_value(pages.ks, i),
                lane_value(pages.vs, i), a.W, a.S, lane, [&](int t, int j, int) { return kr[t][j]; },
                [&](int y, int) { return vr[y]; },
                [&] {
                    if (i + 1 < n) load_k(next);
                },
                [&](int t0) {
                    const u32x4 keep = seen_bytes(t0, st.wp1, st.far, a.S, lane);
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
    if (w == 0) close_rows(a, st, k, k.tr.r0, ROWS, lane);
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
    if (!open_walk<true>(a, ROWS, lane, k)) return;
    const int wr0 = k.tr.r0 + 16 * RT * w;
    CacheRows<D, RT> st;
    open_rows(a, st, k.b, k.hk, k.tr.len, wr0, lane);
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
                page_step<D, RT, 1, 2, 2>(
                    st, t0, lane_value(pages.ks, i), lane_value(pages.vs, i), a.W, a.S, lane,
                    [&](int t, int j, int p) { return cur[t * KL + j][p][lane]; },
                    [&](int y, int p) { return cur[4 * KL + y][p][lane]; }, [] {}, [](int) {});
            __builtin_amdgcn_sched_barrier(0);
            __syncthreads();
        }
    }
#pragma unroll
    for (int x = 0; x < RT; ++x) st.l[x] = row_sum(st.l[x]);
    if (live) close_rows(a, st, k, wr0, ROWS, lane);
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

template <int D>
void launch_wide(const CacheAttnArgs& a, dim3 g, hipStream_t s) {
    if constexpr (D == 64)
        hipLaunchKernelGGL((cache_attn_kernel<64, 1, kWideWaves>), g, dim3(64 * kWideWaves), 0, s, a);
}

template <int D>
void launch(const CacheAttnArgs& a, const CacheAttnPlan& p, hipStream_t s) {
    const int64_t wgs = cache_attn_groups(p, a.c.B) * a.c.Hkv;
    const dim3 g(static_cast<unsigned>(wgs)), t(kThreads);
    {
        TraceScope _t("cache_attn", s);
        if (p.wr == 4) hipLaunchKernelGGL((cache_attn_rows_kernel<D>), g, t, 0, s, a);
        else if (p.wide) launch_wide<D>(a, g, s);
        else if (p.rt == 2) hipLaunchKernelGGL((cache_attn_kernel<D, 2, 4>), g, t, 0, s, a);
        else hipLaunchKernelGGL((cache_attn_kernel<D, 1, 4>), g, t, 0, s, a);
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
                              int64_t S) {
    CacheAttnPlan p{};
    const int64_t rows = Hq / Hkv * T;
    p.rt = rows <= 16 ? 1 : 2;
    // From 33 rows on one tile over four waves, also where some stay without rows (us, tiles
    // of 32 rows that walk the pages each -> this: 32 contexts of up to 16K, 28 over 4 heads,
    // 5 to 9 tokens 146-150 -> 112-116; 16 of up to 8K, 32 over 8, head dim 64, 9 to 16
    // tokens 46-49 -> 39-40; 4 of up to 8K, 16 over 2, 5 to 8 tokens 17.5-18.7 -> 17.9-19.4;
    // 64 of up to 2K, 32 over 4, head dim 64, 6 to 8 tokens 24.4 -> 29.6)
    p.wr = rows <= 32 ? 1 : 4;
    p.rows = 16 * p.rt * p.wr;
    p.tiles = int32_t((rows + p.rows - 1) / p.rows);
    // the most pages that a tile sees: the window of its tokens, the sinks' (what a plan
    // needs grows with them, so that one without a window has room for all)
    const int64_t span = std::min(T, p.rows / (Hq / Hkv) + 2);
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
        p.items = int32_t(std::max(p.wr == 4 ? aim : aim - e, e));
        const int64_t most = p.wr == 4 ? 2 * int64_t(p.items) : p.items + e;
        p.slots = int32_t(std::min(most, e * ((width + kMinChunk - 1) / kMinChunk)));
        while (e * ((width >> p.unit) + 1) > INT32_MAX) ++p.unit;
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
    if (a.c.d == 128) launch<128>(a, p, s);
    else launch<64>(a, p, s);
    return hipGetLastError();
}

}  // namespace msparse
