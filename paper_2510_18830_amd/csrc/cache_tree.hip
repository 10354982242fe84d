// Drafted trees over the paged 8-bit cache: masks and positions, and the attention of
// calls with many rows.
//
// ---- Masks.  Node t of a sequence's tree has a parent among the nodes before it, or none (the child of the
// context's last token).  Its position is lens + the number of its ancestors; it sees itself and
// those ancestors that the window or the sinks leave visible.  A thread walks one node's
// ancestors, which descend, and writes its words from the last to the first as it passes them: no
// word is held or read back.  Bound by latency: the walk's LDS reads, one after the other (64 trees
// of 16 nodes 3.4 us).
//
// ---- Attention.  The T G rows of a KV head (row r: node r / G, head r % G of the group) are cut into tiles of 128, 32
// a wave, that walk the pages they see together; up to 64 rows, two waves share 32, and each takes half of every page's
// tokens:
//   S^T = K Q^T      (32x32x16 bf16: A = 32 tokens, B = the queries)
//   online softmax   (a lane owns a row and half of the tokens)
//   O^T += V^T P^T   (A = 32 columns, B = P from the S^T registers)
// Codes go to LDS as they lie in memory, some pages ahead and past the registers, and every wave converts its operands to
// bf16 between the products.  A page's K scale enters the logits' factor, its V scale the conversion.  (Products of 8
// bits, which would take keys as they lie, with the queries split into two e4m3 parts, are exact, but their sums are not:
// the matrix cores keep 12 bits below the largest of 64 products, which put lse off by 1e-3.)
//
// Few rows are bound by the cache's bytes and each step's chain, many by the issue of instructions (a product takes 16 of
// its 32 cycles of it) and by power, which lowers the clock.  Contexts of up to 16K, 32 of them, 28 over 4 heads, with the
// join: 8 nodes 88 us, 16 124, 32 205 (0.70 PFLOP/s; a plain matrix product of bf16 reaches 1.37).  Codes converted once
// for the four waves to bf16 in LDS, twice its bytes: 102, 128 and 213 us; 64 rows a wave, which halves LDS's bytes and
// the conversions, one wave a SIMD: 132, 142 and 243.
#include "cache_walk.h"
#include "tiles.h"
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

// ---------------------------------------------------------------- attention
constexpr float kSlack = 8.f;   // log2 units that a row's maximum may rise by before its sums are rescaled

// A wave's 32 rows; lane (half h, i) owns row i and half h of the contractions.
template <int D>
struct TreeRows {
    u32x4 q[D / 16];     // the query: step 2 c + e takes columns 32 c + 16 h + 8 e ..
    f32x16 o[D / 32];
    float m, l;          // the whole number that the weights are relative to; their sum, of this lane's tokens
    float limit;         // logits beyond it raise m
};
constexpr float kNone = -0x1.fffffep127f;   // m of a row without a token yet: finite, so that a masked logit weighs 0
constexpr int kDepth = 4;   // pages of keys, and of values, in LDS (5 and 6: the same times)

template <int D>
__device__ __forceinline__ void open_tree_rows(const CacheAttnArgs& a, TreeRows<D>& st, const Walk& k, int wr0, int lane) {
    const int G = a.Hq / a.c.Hkv, R = a.T * G, r = min(wr0 + (lane & 31), R - 1);
    const uint16_t* qp = a.q + k.b * a.qs[0] + (k.hk * G + r % G) * a.qs[1] + (r / G) * a.qs[2] + 16 * (lane >> 5);
#pragma unroll
    for (int s = 0; s < D / 16; ++s) st.q[s] = *reinterpret_cast<const u32x4*>(qp + 32 * (s >> 1) + 8 * (s & 1));
#pragma unroll
    for (int x = 0; x < D / 32; ++x) st.o[x] = f32x16{};
    st.m = kNone;
    st.limit = kNone;
    st.l = 0.f;
}

// A workgroup's walk in scalar registers (clamps and ballots left it in vector ones).
__device__ __forceinline__ void make_uniform(Walk& k) {
    for (int32_t* x : {&k.b, &k.c0, &k.c1, &k.tr.r0, &k.tr.len, &k.tr.base, &k.pl.sinks, &k.pl.lo, &k.ch.first, &k.ch.count,
                       &k.ch.index})
        *x = __builtin_amdgcn_readfirstlane(*x);
}

// Which row r of a (sequence, KV head) stands for: its node of the call, -1 where it is behind the sequence's
// nodes (or the last row) and sees nothing.
__device__ __forceinline__ int node_of(const CacheAttnArgs& a, const Walk& k, int r) {
    const int G = a.Hq / a.c.Hkv, t = r / G;
    return r < a.T * G && t < k.tr.len - k.tr.base ? k.b * a.T + t : -1;
}
__device__ __forceinline__ uint64_t below64(int n) { return n >= 64 ? ~0ull : (uint64_t(1) << max(n, 0)) - 1; }
// Which of the 64 tokens from slot j on a row at position pos (of the nodes' places) sees: of the context what its
// position does (without a window all of it), of the nodes those of its bits, word(x) for x >= 0.
template <class Word>
__device__ __forceinline__ uint64_t tokens_seen(const CacheAttnArgs& a, const Walk& k, int pos, int j, Word word) {
    const int base = k.tr.base, len = k.tr.len;
    uint64_t bits = 0;
    if (j < len && j + 63 >= base) {
        const int u = j - base, w = u >> 5;   // (u > -64: the words before the first are empty)
        auto at = [&](int x) { return x >= 0 && x < a.words ? uint64_t(uint32_t(word(x))) : 0; };
        bits = (at(w) | (at(w + 1) << 32)) >> (u & 31);
        if (u & 31) bits |= at(w + 2) << (64 - (u & 31));
        bits &= below64(len - j);
    }
    const uint64_t context = below64(base - j);
    return (bits & ~context) | (context & (~below64(max(pos - a.W + 1, 0) - j) | below64(min(a.S - 1, pos) + 1 - j)));
}
__device__ __forceinline__ int position_of(const CacheAttnArgs& a, const Walk& k, int node) {
    return max(min(a.at ? a.at[node] : k.tr.base, k.tr.len - 1), k.tr.base);
}
__device__ __forceinline__ uint64_t row_sees(const CacheAttnArgs& a, int r, int j, const Walk& k) {
    const int node = node_of(a, k, r);
    if (node < 0) return 0;
    const int32_t* row = a.seen + int64_t(node) * a.words;
    return tokens_seen(a, k, position_of(a, k, node), j, [&](int x) { return row[x]; });
}
// What a tile's rows see, all of them together: the nodes' words, and the first of their positions, which sees the most
// of the context.
struct TileSeen {
    uint32_t words[kMaxNodes / 32];
    int32_t pos;
};
__device__ __forceinline__ void clear_seen(TileSeen& s) {
    if (threadIdx.x < kMaxNodes / 32) s.words[threadIdx.x] = 0;
    if (threadIdx.x == 0) s.pos = INT32_MAX;
}
// A thread's position and the first of its words are asked for at once, and entered with the others when the memory is
// clear.
struct SeenItems {
    const int32_t* words;
    int32_t nodes, items;   // of the tile; their words
    uint32_t word[2];
    int32_t pos;
};
template <int N>
__device__ __forceinline__ void ask_words(const SeenItems& x, int y0, uint32_t (&w)[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e) w[e] = y0 + e * kThreads < x.items ? uint32_t(x.words[y0 + e * kThreads]) : 0;
}
template <int N>
__device__ __forceinline__ void enter_words(const CacheAttnArgs& a, int y0, const uint32_t (&w)[N], TileSeen& s) {
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (w[e]) atomicOr(s.words + (y0 + e * kThreads) % a.words, w[e]);
}
__device__ __forceinline__ SeenItems ask_seen(const CacheAttnArgs& a, const Walk& k, int rows) {
    const int G = a.Hq / a.c.Hkv, t0 = k.tr.r0 / G, t1 = min((k.tr.r0 + rows - 1) / G, k.tr.len - k.tr.base - 1);
    const int node = k.b * a.T + t0;
    SeenItems x{};
    x.nodes = t1 - t0 + 1;
    x.items = x.nodes * a.words;
    x.words = a.seen + int64_t(node) * a.words;
    ask_words(x, threadIdx.x, x.word);
    x.pos = int(threadIdx.x) < x.nodes ? position_of(a, k, node + threadIdx.x) : INT32_MAX;
    return x;
}
__device__ __forceinline__ void enter_seen(const CacheAttnArgs& a, const SeenItems& x, TileSeen& s) {
    enter_words(a, threadIdx.x, x.word, s);
    if (int(threadIdx.x) < x.nodes) atomicMin(&s.pos, x.pos);
    for (int y0 = threadIdx.x + 2 * kThreads; y0 < x.items; y0 += 8 * kThreads) {
        uint32_t w[8];
        ask_words(x, y0, w);
        enter_words(a, y0, w, s);
    }
}
__device__ __forceinline__ uint64_t tile_sees(const CacheAttnArgs& a, const Walk& k, int j, const TileSeen& s) {
    return tokens_seen(a, k, s.pos, j, [&](int x) { return s.words[x]; });
}

// Where the codes of a page lie in LDS: as in memory, rows of a token's D columns (keys) or a column's 64 tokens (values),
// but for the order of a row's 16-byte pieces, which puts those that 16 lanes read in one LDS cycle into distinct banks.
// Which piece of row `row` stands in place c, and where piece c stands: both c ^ this.
template <int D>
__device__ __forceinline__ int key_order(int row) {
    return D == 128 ? ((row >> 1) & 3) | ((row >> 2) & 4) : ((row >> 2) & 1) | ((row >> 3) & 2);
}
__device__ __forceinline__ int value_order(int row) { return (row >> 2) & 3; }
// Which token a row of the S^T tiles stands for: those of half h's accumulators are 16 tokens in a row from 16 h on,
// eight for each step of the second product, whose 16-byte pieces of a column they are.
__device__ __forceinline__ int token_of(int i) { return 4 * (i & 4) + ((i >> 1) & 12) + (i & 3); }

// 16 bytes a lane from `base` + its offset to LDS, lane after lane from `to` on; no wait (but the wait state that M0
// needs between its write and the load).
__device__ __forceinline__ void fetch16(const uint8_t* base, uint32_t offset, uint32_t to) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                 :
                 : "v"(offset), "s"(base), "s"(__builtin_amdgcn_readfirstlane(to))
                 : "memory", "m0");
}
template <int N>
__device__ __forceinline__ void wait_fetched() {   // all but the last N
    asm volatile("s_waitcnt vmcnt(%0)" : : "i"(N) : "memory");
}

// A page's V scale: the power of two enters the values as they are converted, the mantissa (1, where an
// append wrote the page) the weights' exponent, as its logarithm, and leaves their sum again.
struct ValueScale {
    float power, shift, back;
};
__device__ __forceinline__ ValueScale value_scale(float x) {
    const float m = x > 0.f ? 2.f * __builtin_amdgcn_frexp_mantf(x) : x == 0.f ? 1.f : x;
    return ValueScale{__uint_as_float(__float_as_uint(x) & 0x7f800000u), fast_log2(m), 1.f / m};
}

// What a wave carries from one step of 32 tokens to the next: the weights of the 32 before them, whose product with the
// values is still to come.
struct TreeHalf {
    u32x4 p[2];
};
// A lane's logits of 32 tokens, and the largest of them.
struct TreeLogits {
    f32x16 s;
    float top;
};
__device__ __forceinline__ float largest(const f32x16& s) {
    float top = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
    return top;
}

// The 32 tokens in `cur` become weights, while the matrix cores form the logits of the next 32 (codes of keys at kb + kat),
// then the product of the last ones (codes of values at vb, times `power`): each MFMA is followed by vector work that it
// covers.
template <int D>
__device__ __forceinline__ void tree_half(TreeRows<D>& st, TreeLogits& cur, TreeHalf& w, const uint8_t* kb, int kat,
                                          const uint8_t* vb, float fac, ValueScale vs, float power) {
    constexpr int KS = D / 16;
    u32x4 kraw[2], vraw[2], kop[2], vop[2];   // codes of two steps each; operands
    auto read_k = [&](int c) { kraw[c & 1] = *reinterpret_cast<const u32x4*>(kb + (kat ^ (32 * c))); };
    auto read_v = [&](int c) { vraw[c & 1] = *reinterpret_cast<const u32x4*>(vb + 32 * kPage * c); };
    auto convert_k = [&](int x) {
        const u32x4& r = kraw[(x >> 1) & 1];
        kop[x & 1] = x & 1 ? codes_to_bf16(r.z, r.w) : codes_to_bf16(r.x, r.y);
    };
    auto convert_v = [&](int x) {
        const u32x4& r = vraw[(x >> 1) & 1];
        vop[x & 1] = x & 1 ? codes_to_bf16(r.z, r.w, power) : codes_to_bf16(r.x, r.y, power);
    };
    read_k(0);
    read_k(1);
    const float shift = vs.shift - st.m;
    const u32x4 last[2] = {w.p[0], w.p[1]};
    float l[2] = {0.f, 0.f};
    auto weights = [&](int y) {   // of a pair of tokens
        const float a = fast_exp2(__builtin_fmaf(cur.s[2 * y], fac, shift));
        const float b = fast_exp2(__builtin_fmaf(cur.s[2 * y + 1], fac, shift));
        uint32_t ab = pack_bf16x2(a, b);
        l[0] += a;
        l[1] += b;
        asm volatile("" : "+v"(ab), "+v"(l[0]), "+v"(l[1]));   // here, beside the products, and not where they are used
        w.p[y >> 2][y & 3] = ab;
    };
    // Pairs before the logits' products and beside them; the rest beside the first half of the values'.
    constexpr int kPairs = 8, kAhead = 1, kLogits = KS * 5 / 8;
    int y = 0;
    for (; y < kAhead; ++y) weights(y);
    convert_k(0);
    f32x16 next;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int x = 0; x < KS; ++x) {
        next = mfma32(kop[x & 1], st.q[x], x ? next : f32x16{});
        __builtin_amdgcn_sched_barrier(0);
        if (x + 1 < KS) convert_k(x + 1);
        const int goal = kAhead + kLogits * (x + 1) / KS;
#pragma unroll
        for (; y < goal; ++y) weights(y);
        if ((x & 1) == 0 && x / 2 + 2 < KS / 2) read_k(x / 2 + 2);
        if (x >= KS - 2) read_v(x - (KS - 2));
        __builtin_amdgcn_sched_barrier(0);
    }
    convert_v(0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int x = 0; x < KS; ++x) {
        st.o[x >> 1] = mfma32(vop[x & 1], last[x & 1], st.o[x >> 1]);
        __builtin_amdgcn_sched_barrier(0);
        if (x + 1 < KS) convert_v(x + 1);
        const int goal = kAhead + kLogits + (kPairs - kAhead - kLogits) * (x + 1) / (KS / 2);
#pragma unroll
        for (; y < goal && y < kPairs; ++y) weights(y);
        if ((x & 1) == 0 && x / 2 + 2 < KS / 2) read_v(x / 2 + 2);
        if (x == KS - 1) cur = TreeLogits{next, largest(next)};
        __builtin_amdgcn_sched_barrier(0);
    }
    st.l = __builtin_fmaf(l[0] + l[1], vs.back, st.l);
}

// The logits of the first 32 tokens.
template <int D>
__device__ __forceinline__ TreeLogits tree_first(const TreeRows<D>& st, const uint8_t* kb, int kat) {
    f32x16 s{};
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
        const u32x4 raw = *reinterpret_cast<const u32x4*>(kb + (kat ^ (32 * c)));
        s = mfma32(codes_to_bf16(raw.x, raw.y), st.q[2 * c], s);
        s = mfma32(codes_to_bf16(raw.z, raw.w), st.q[2 * c + 1], s);
    }
    return TreeLogits{s, largest(s)};
}

// The product of the weights that are left with their values.
template <int D>
__device__ __forceinline__ void tree_flush(TreeRows<D>& st, const TreeHalf& w, const uint8_t* vb, float power) {
#pragma unroll
    for (int b = 0; b < D / 32; ++b) {
        const u32x4 raw = *reinterpret_cast<const u32x4*>(vb + 32 * kPage * b);
        st.o[b] = mfma32(codes_to_bf16(raw.x, raw.y, power), w.p[0], st.o[b]);
        st.o[b] = mfma32(codes_to_bf16(raw.z, raw.w, power), w.p[1], st.o[b]);
    }
}

// The logits of 32 tokens before they become weights: masks, and the running maximum, which moves only where
// it has to (the weights stay below 2^(kSlack + 1)).  It is a whole number, so that what moves by it moves by a
// power of two: the weights that wait for their product do exactly.
template <int D, class Sees>
__device__ __forceinline__ void tree_top(TreeRows<D>& st, TreeLogits& cur, TreeHalf& w, bool part, Sees mask, float fac) {
    if (part) {
        const uint32_t sees = mask();
        keep_branch();
#pragma unroll
        for (int r = 0; r < 16; ++r)
            if (!((sees >> r) & 1)) cur.s[r] = -INFINITY;
        cur.top = largest(cur.s);
    }
    float top = cur.top * fac;
    if (__any(top > st.limit)) {
        top = half_swap_max(top);
        const float m = top > st.limit ? __builtin_ceilf(top) : st.m;
        const float alpha = fast_exp2(st.m - m);   // (of a row without a token yet: 0 times nothing)
        st.l *= alpha;
#pragma unroll
        for (int b = 0; b < D / 32; ++b) st.o[b] *= alpha;
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int j = 0; j < 4; ++j) w.p[g][j] = pack_bf16x2(bf16_lo(w.p[g][j]) * alpha, bf16_hi(w.p[g][j]) * alpha);
        st.limit = top > st.limit ? m + kSlack : st.limit;
        st.m = m;
    }
}

// A row's results, to out and lse or to this chunk's slot.
template <int D>
__device__ __forceinline__ void close_tree_rows(const CacheAttnArgs& a, TreeRows<D>& st, const Walk& k, int wr0, int rows,
                                                int lane) {
    const int h = lane >> 5, G = a.Hq / a.c.Hkv, R = a.T * G, r = wr0 + (lane & 31);
    st.l = half_swap_sum(st.l);
    if (st.m == kNone) st.m = -INFINITY;
    if (r >= R) return;
    if (node_of(a, k, r) < 0) {   // (pages without a mask have been added to it too)
        st.m = -INFINITY;
        st.l = 0.f;
#pragma unroll
        for (int b = 0; b < D / 32; ++b) st.o[b] = f32x16{};
    }
    if (k.ch.count > 1) {
        const int64_t row = (int64_t(k.ch.first + k.ch.index) * a.c.Hkv + k.hk) * rows + (r - k.tr.r0);
        float* po = a.po + row * D + 4 * h;
#pragma unroll
        for (int b = 0; b < D / 32; ++b)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4*>(po + 32 * b + 8 * g) =
                    f32x4{st.o[b][4 * g], st.o[b][4 * g + 1], st.o[b][4 * g + 2], st.o[b][4 * g + 3]};
        if (h == 0) {
            a.pml[2 * row] = st.m;
            a.pml[2 * row + 1] = st.l;
        }
        return;
    }
    const int t = r / G, hq = k.hk * G + r % G;
    const bool empty = no_key(st.m, st.l);
    const float inv = empty ? 0.f : 1.f / st.l;
    uint16_t* op = a.out + k.b * a.os[0] + hq * a.os[1] + t * a.os[2] + 4 * h;
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            u32x2 pk;
            pk.x = pack_bf16x2(st.o[b][4 * g] * inv, st.o[b][4 * g + 1] * inv);
            pk.y = pack_bf16x2(st.o[b][4 * g + 2] * inv, st.o[b][4 * g + 3] * inv);
            *reinterpret_cast<u32x2*>(op + 32 * b + 8 * g) = pk;
        }
    if (a.lse && h == 0)
        a.lse[(int64_t(k.b) * a.Hq + hq) * a.T + t] = empty ? -INFINITY : (st.m + fast_log2(st.l)) * kLn2;
}

// An even share of a KV head's work: the pages of all row tiles, one tile behind the other, are dealt to the
// workgroups in runs of `each`, so that whatever the raggedness all take as long.  A run may end inside a tile and take
// in several; a tile that lies in one run writes its results, one that is cut leaves a part in slot (workgroup + tile)
// for each, which are neighbours for the join.  Tiles without pages go with the place where they lie.  Pages are counted
// in units of 2^unit, a tile's rounded up, which keeps their sum below 2^31.
// A second tile in a run costs a second start, about four pages' time (9 us).  Where runs can each keep to one tile at
// that price, a tile's units are rounded up to whole runs (2 x 60 nodes of 32 over 8 heads at 2000: 29.0 -> 23.8 us, 16 x
// 16 at 8192, head dim 64: 40.7 -> 37); else every tile counts as so many pages more, before its first, that a run with
// two of them takes fewer (8 x 128 at 8192, 32 over 8 heads 131 -> 123 us, 32 x 16 at 16384, 28 over 4 127 -> 124).
constexpr int kStart = 4;
struct Share {
    int32_t item, total, each, lo, hi;   // the workgroup; units: all, of a run, of this one
    int32_t e, at;                       // the next tile and its first unit
    int32_t last;                        // the last workgroup that has a run
    int32_t whole, start;                // a tile takes a multiple of so many units; so many of them are its start
};
__device__ __forceinline__ int page_units(const CacheAttnArgs& a, const PageList& l) {
    return int((uint32_t(l.count) + (1u << a.unit) - 1) >> a.unit);
}
__device__ __forceinline__ int tile_units(int n, const Share& s) {
    return n == 0 ? 0 : s.whole == 1 ? n + s.start : (n + s.whole - 1) / s.whole * s.whole;
}
__device__ __forceinline__ PageList pages_of_tile(const CacheAttnArgs& a, int e, int rows) {
    const int b = e / a.tiles;
    return tile_pages(a, tile_rows<true>(a, b, length_of(a, b), e % a.tiles, rows));
}
__device__ __forceinline__ bool open_share(const CacheAttnArgs& a, int rows, int lane, Share& s) {
    const int E = a.c.B * a.tiles;
    auto units = [&](int e) { return e < E ? page_units(a, pages_of_tile(a, e, rows)) : 0; };
    int sum = 0, some = 0;
    for (int e = lane; e < E; e += 64) {
        const int n = units(e);
        sum += n;
        some += n > 0;
    }
    s.item = blockIdx.x / a.c.Hkv;
    s.start = a.unit == 0 ? kStart : 0;
    s.whole = 1;
    const int pages = __builtin_amdgcn_readlane(wave_scan(sum), 63);
    s.total = pages + s.start * __builtin_amdgcn_readlane(wave_scan(some), 63);
    s.each = max((s.total + a.items - 1) / a.items, kMinChunk);
    if (E <= 64)
        for (int each = max((pages + a.items - 1) / a.items, kMinChunk); each <= s.each; ++each) {
            const int runs = __builtin_amdgcn_readlane(wave_scan((sum + each - 1) / each), 63);
            if (runs > a.items) continue;
            s.total = runs * each;
            s.each = s.whole = each;
            s.start = 0;
            break;
        }
    s.last = max(s.total - 1, 0) / s.each;
    if (s.item > s.last) return false;
    s.lo = s.item * s.each;
    s.hi = min(s.lo + s.each, s.total);
    s.at = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {   // the first tile that ends behind lo, or lies there without pages
        const int n = tile_units(units(e0 + lane), s), end = s.at + wave_scan(n);
        const uint64_t here = __ballot(e0 + lane < E && (end > s.lo || (n == 0 && end >= s.lo)));
        if (here) {
            const int l = __builtin_ctzll(here);
            s.e = e0 + l;
            s.at = __builtin_amdgcn_readlane(end - n, l);
            return true;
        }
        s.at = __builtin_amdgcn_readlane(end, 63);
    }
    return false;
}
__device__ __forceinline__ bool next_tile(const CacheAttnArgs& a, int rows, Share& s, Walk& k) {
    if (s.e >= a.c.B * a.tiles) return false;
    k.hk = blockIdx.x % a.c.Hkv;
    k.b = s.e / a.tiles;
    k.tr = tile_rows<true>(a, k.b, __builtin_amdgcn_readfirstlane(length_of(a, k.b)), s.e % a.tiles, rows);
    k.pl = tile_pages(a, k.tr);
    const int n = tile_units(page_units(a, k.pl), s), end = s.at + n;
    const int from = n > 0 ? s.at + s.start : s.at;   // its first page
    if (!(from < s.hi || (from == s.total && s.item == s.last))) return false;
    const int first = min(from, max(s.total - 1, 0)) / s.each, last = n > 0 ? (end - 1) / s.each : first;
    k.ch = Chunk{s.e, first + s.e, last - first + 1, s.item - first, 0};
    k.c0 = int(min(int64_t(max(s.lo - from, 0)) << a.unit, int64_t(k.pl.count)));
    k.c1 = int(min(int64_t(min(s.hi, end) - from) << a.unit, int64_t(k.pl.count)));
    if (k.hk == 0 && k.ch.index == 0 && threadIdx.x == 0) {
        a.info[2 * s.e] = k.ch.first;
        a.info[2 * s.e + 1] = k.ch.count;
    }
    ++s.e;
    s.at = end;
    return true;
}

// The two token halves of a tile's rows: the waves of the second leave theirs in `mem`, those of the first add them.
template <int D>
__device__ __forceinline__ void merge_halves(TreeRows<D>& st, bool second, float* mem, int lane) {
    constexpr int N = D / 32;
    float* at = mem + lane;
    if (second) {
#pragma unroll
        for (int b = 0; b < N; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) at[(16 * b + r) * 64] = st.o[b][r];
        at[16 * N * 64] = st.m;
        at[16 * N * 64 + 64] = st.l;
    }
    __syncthreads();
    if (second) return;
    const float m2 = at[16 * N * 64], m = fmaxf(st.m, m2), f1 = fast_exp2(st.m - m), f2 = fast_exp2(m2 - m);
    st.l = st.l * f1 + at[16 * N * 64 + 64] * f2;
#pragma unroll
    for (int b = 0; b < N; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) st.o[b][r] = st.o[b][r] * f1 + at[(16 * b + r) * 64] * f2;
    st.m = m;
}

// A tile's rows over the pages [k.c0, k.c1) of its list, 32 a wave.  SPLIT: of up to 64 rows; two waves share 32, each takes
// half of every page's tokens.
constexpr int tree_rows(bool split) { return split ? 64 : 128; }
template <int D>
struct TreeMemory {
    uint8_t k[kDepth][kPage * D], v[kDepth][kPage * D];
};
template <int D, bool SPLIT>
__device__ __forceinline__ void tree_tile(const CacheAttnArgs& a, const Walk& k, TreeMemory<D>& mem, TileSeen& all) {
    constexpr int NF = D / 64;          // pieces of 16 bytes of a page's keys, and of its values, per thread
    constexpr int kBytes = kPage * D;   // of either
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), th = SPLIT ? w >> 1 : 0;
    // (the two workgroups of a CU start from either half of its SIMDs, so that tiles of few rows use them all)
    const int wr0 = k.tr.r0 + 32 * (SPLIT ? w & 1 : (w + 2 * (blockIdx.x / 256 & 1)) & 3);
    const bool live = wr0 < a.T * (a.Hq / a.c.Hkv);
    TreeRows<D> st;
    open_tree_rows(a, st, k, wr0, lane);
    // this lane's operands: of a token the pieces h, 2 + h, .., of a column the piece of its half of this wave's tokens
    const int i32 = lane & 31, h = lane >> 5, tok = token_of(i32) + 32 * th;
    const int kat = tok * D + 16 * (h ^ key_order<D>(tok)), vat = i32 * kPage + 16 * ((2 * th + h) ^ value_order(i32));
    const int kat1 = kat + 32 * D, vat1 = vat ^ 32;   // of the page's second half
    // what this thread fetches: bytes 16 tid .. of every 4096 of a page
    const int kf = 16 * tid / D, vf = tid / 4, piece = (tid & 3) ^ value_order(vf);
    const uint32_t from_k = kf * D + 16 * ((tid % (D / 16)) ^ key_order<D>(kf)), from_v = kPage * vf + 16 * piece;
    const uint32_t lds_k = lds_addr(mem.k) + 1024 * w, lds_v = lds_addr(mem.v) + 1024 * w;
    // what all rows see in full ends before the first node
    const int base = k.tr.base, len = k.tr.len;
    auto in_part = [&](int t0) { return partly(t0, base - 1, len - 1, a.W, a.S); };
    const int n = k.c1 - k.c0;
    if (n > 0) {
        constexpr int kLooks = 64 - kDepth;   // pages looked up at a time, and those after them
        Pages pages;
        ValueScale scales;
        uint32_t off_lo, off_hi;   // where a page's codes lie
        int x0 = 0;
        // Which tokens of this lane's page some row sees.  (The scale of a page without one may be anything: 1 in its place.)
        uint32_t seen_lo, seen_hi;
        auto mark_pages = [&] {
            const int start = page_start(pages.page, k.pl.page(k.c0 + x0 + lane));
            seen_lo = seen_hi = ~0u;
            if (!__any(in_part(start))) return;
            keep_branch();
            if (!in_part(start)) return;
            const uint64_t sees = tile_sees(a, k, start, all);
            seen_lo = uint32_t(sees);
            seen_hi = uint32_t(sees >> 32);
            if (sees == 0) scales = ValueScale{1.f, 0.f, 1.f};
        };
        auto look = [&](int x) {
            x0 = x;
            pages = look_up(a, k, k.c0 + x, 1, lane);
            scales = value_scale(pages.vs);
            if (x > 0) mark_pages();
            const uint64_t off = (uint64_t(max(pages.page, 0)) * a.c.Hkv + k.hk) * kBytes;
            off_lo = uint32_t(off);
            off_hi = uint32_t(off >> 32);
        };
        clear_seen(all);
        // (without a window the pages that some row does not see in full are the last)
        const bool masked = a.at || in_part(kPage * k.pl.page(k.c1 - 1));
        SeenItems asked{};
        if (masked) asked = ask_seen(a, k, tree_rows(SPLIT));
        look(0);
        // (past the last page as many, of 16 bytes of the pool's first page, so that a step's wait counts the same)
        auto fetch = [&](const uint8_t* codes, uint32_t from, uint32_t to, int i, int slot) {
            const uint64_t off = uint32_t(__builtin_amdgcn_readlane(off_lo, i - x0)) |
                                 uint64_t(uint32_t(__builtin_amdgcn_readlane(off_hi, i - x0))) << 32;
#pragma unroll
            for (int j = 0; j < NF; ++j)
                fetch16(codes + off + 4096 * j, i < n ? from : 0, to + kBytes * slot + 4096 * j);
        };
        __syncthreads();   // the tile before has been read
        if (masked) enter_seen(a, asked, all);
        // Step i: the weights of page i, the logits of the tokens after them and the product of those before with their
        // values.  It reads the keys of pages i (SPLIT: no more) and i + 1 and the values of pages i - 1 and i (SPLIT: not
        // yet), and asks for the keys of page i + kAheadK and the values of page i + kDepth - 2.
        constexpr int kAheadK = SPLIT ? kDepth : kDepth - 1;
        constexpr int kLeft = (SPLIT ? kDepth - 2 : kDepth - 3) * 2 * NF;   // fetches behind those that a step needs
#pragma unroll
        for (int i = 0; i < kAheadK; ++i) {
            fetch(a.c.k, from_k, lds_k, i, i);
            const int v = i + kDepth - 2 - kAheadK;
            if (v >= 0) fetch(a.c.v, from_v, lds_v, v, v);
        }
#pragma unroll
        for (int j = 0; j < NF; ++j)   // (the first weights, which are 0, meet no values yet)
            *reinterpret_cast<u32x4*>(mem.v[kDepth - 1] + 16 * tid + 4096 * j) = u32x4{};
        wait_fetched<SPLIT ? kLeft : kLeft + 2 * NF>();
        __syncthreads();
        TreeLogits cur = tree_first(st, mem.k[0], kat);
        mark_pages();
        TreeHalf left{};   // (no weights yet: 0)
        int kslot = 0, vslot = kDepth - 1;   // of page i's keys, page i - 1's values
        auto after = [](int slot) { return slot == kDepth - 1 ? 0 : slot + 1; };
        auto before = [](int slot) { return slot == 0 ? kDepth - 1 : slot - 1; };
        float power = 1.f;   // of page i - 1
        auto start_of = [&](int i) {
            return __builtin_amdgcn_readfirstlane(page_start(page_at(pages, i - x0), k.pl.page(k.c0 + i)));
        };
        auto seen_of = [&](int i) {
            return uint32_t(__builtin_amdgcn_readlane(seen_lo, i - x0)) |
                   uint64_t(uint32_t(__builtin_amdgcn_readlane(seen_hi, i - x0))) << 32;
        };
        // The values at `slot`, of a page of which some row sees these tokens, are there: codes of the others may stand for
        // anything, NaN among it, which a weight of 0 would not remove; each thread clears those that it has fetched.
        auto enter = [&](int slot, uint64_t sees) {
            wait_fetched<kLeft>();
            if (~sees) {
                keep_branch();
                const u32x4 keep = bytes_of(uint32_t(sees >> (16 * (opaque(tid) & 3 ^ value_order(opaque(tid) / 4)))));
#pragma unroll
                for (int j = 0; j < NF; ++j) *reinterpret_cast<u32x4*>(mem.v[slot] + 16 * tid + 4096 * j) &= keep;
            }
            __syncthreads();
        };
        uint64_t sees0 = ~0ull;   // of page i - 1
        for (int i = 0; i < n; ++i) {
            if (i - x0 >= kLooks) look(i);
            const int start = start_of(i);
            const uint64_t sees = seen_of(i);
            if constexpr (SPLIT) enter(vslot, sees0);
            else enter(after(vslot), sees);
            // Of two waves that could issue the older one does: of a CU's workgroups the second then lags behind the first
            // and works alone in the end.  It leads every other page (128 rows, contexts of 16K: 131 -> 127 us).
            if (blockIdx.x & 256) {
                if (i & 1) __builtin_amdgcn_s_setprio(1);
                else __builtin_amdgcn_s_setprio(0);
            }
            fetch(a.c.k, from_k, lds_k, i + kAheadK, SPLIT ? kslot : before(kslot));
            fetch(a.c.v, from_v, lds_v, i + kDepth - 2, before(vslot));
            const float now = lane_value(scales.power, i - x0);
            if (live) {
                // (the factor stays above 0, as a masked logit times 0 would be NaN)
                const float fac = lane_value(pages.ks, i - x0);
                const ValueScale vs{0.f, lane_value(scales.shift, i - x0), lane_value(scales.back, i - x0)};
                const bool part = in_part(start);
                // what this lane's row sees of its tokens of half x of the page (asked for where some row does not see all)
                auto seen = [&](int x) {
                    return [=, &a, &k] {
                        const int l = opaque(lane);
                        return uint32_t(row_sees(a, wr0 + (l & 31), start + 32 * x, k) >> (16 * (l >> 5)));
                    };
                };
                tree_top(st, cur, left, part, seen(th), fac);
                if constexpr (SPLIT) {   // (the last step's logits are of no page, for nothing)
                    tree_half(st, cur, left, mem.k[after(kslot)], kat, mem.v[vslot] + vat, fac, vs, power);
                } else {
                    tree_half(st, cur, left, mem.k[kslot], kat1, mem.v[vslot] + vat1, fac, vs, power);
                    tree_top(st, cur, left, part, seen(1), fac);
                    tree_half(st, cur, left, mem.k[after(kslot)], kat, mem.v[after(vslot)] + vat, fac, vs, now);
                }
            }
            power = now;
            sees0 = sees;
            kslot = after(kslot);
            vslot = after(vslot);
        }
        if constexpr (SPLIT) enter(vslot, sees0);
        if (live) tree_flush(st, left, mem.v[vslot] + (SPLIT ? vat : vat1), power);
        wait_fetched<0>();
        if constexpr (SPLIT) {
            __syncthreads();
            merge_halves(st, th, reinterpret_cast<float*>(&mem) + (w & 1) * (sizeof(TreeMemory<D>) / 8), lane);
        }
    }
    if (live && th == 0) close_tree_rows(a, st, k, wr0, tree_rows(SPLIT), lane);
}

template <int D, bool SPLIT>
__global__ void __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(D == 128 ? 2 : 3, D == 128 ? 2 : 3)))
tree_rows_kernel(CacheAttnArgs a) {
    __shared__ __attribute__((aligned(16))) TreeMemory<D> mem;
    __shared__ TileSeen all;
    constexpr int kRows = tree_rows(SPLIT);
    const int lane = threadIdx.x & 63;
    Walk k;
    Share share;
    if (a.items > 0) {
        if (!open_share(a, kRows, lane, share) || !next_tile(a, kRows, share, k)) return;
    } else if (!open_walk<false, true>(a, kRows, lane, k)) {
        return;
    }
    do {
        make_uniform(k);
        tree_tile<D, SPLIT>(a, k, mem, all);
    } while (a.items > 0 && next_tile(a, kRows, share, k));
}

}  // namespace

void launch_tree_rows(const CacheAttnArgs& a, int rows, dim3 grid, hipStream_t s) {
    const dim3 t(kThreads);
    if (rows == tree_rows(true)) {
        if (a.c.d == 128) hipLaunchKernelGGL((tree_rows_kernel<128, true>), grid, t, 0, s, a);
        else hipLaunchKernelGGL((tree_rows_kernel<64, true>), grid, t, 0, s, a);
    } else {
        if (a.c.d == 128) hipLaunchKernelGGL((tree_rows_kernel<128, false>), grid, t, 0, s, a);
        else hipLaunchKernelGGL((tree_rows_kernel<64, false>), grid, t, 0, s, a);
    }
}

hipError_t launch_tree_mask(const TreeMaskArgs& a, hipStream_t s) {
    TraceScope _t("tree_mask", s);
    hipLaunchKernelGGL(tree_mask_kernel, dim3(unsigned(a.B)), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace msparse
