// Drafted trees over the paged 8-bit cache: masks and positions, and the attention of
// calls with many rows.
//
// ---- Masks.  Node t of a sequence's tree has a parent among the nodes before it, or none (the child of the
// context's last token).  Its position is lens + the number of its ancestors; it sees itself and
// those ancestors that the window or the sinks leave visible.  A thread walks one node's
// ancestors, which descend, and writes its words from the last to the first as it passes them: no
// word is held or read back.  Bound by latency: the walk's LDS reads, one after the other.
//
// ---- Attention.  The T G rows of a KV head (row r: node r / G, head r % G of the group) are cut
// into tiles of 128, 32 a wave, that walk the pages they see together:
//   S^T = K Q^T      (32x32x16 bf16: A = 32 tokens, B = the queries)
//   online softmax   (a lane owns a row and half of the page's tokens)
//   O^T += V^T P^T   (A = 32 columns, B = P from the S^T registers)
// The codes of a page are converted once for the four waves, to bf16 operands in LDS.  (Products of 8 bits,
// which would take keys as they lie, with the queries split into two e4m3 parts, are exact, but their sums
// are not: the matrix cores keep 12 bits below the largest of 64 products, which put lse off by 1e-3.)
// A page's K scale enters the logits' factor, its V scale the conversion.
#include <type_traits>

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
    u32x4 q[D / 16];     // the query, columns 16 s + 8 h ..
    f32x16 o[D / 32];
    float m, l;          // the whole number that the weights are relative to; their sum, of this lane's tokens
    float limit;         // logits beyond it raise m
};
constexpr float kNone = -0x1.fffffep127f;   // m of a row without a token yet: finite, so that a masked logit weighs 0

template <int D>
__device__ __forceinline__ void open_tree_rows(const CacheAttnArgs& a, TreeRows<D>& st, const Walk& k, int wr0, int lane) {
    const int G = a.Hq / a.c.Hkv, R = a.T * G, r = min(wr0 + (lane & 31), R - 1);
    const uint16_t* qp = a.q + k.b * a.qs[0] + (k.hk * G + r % G) * a.qs[1] + (r / G) * a.qs[2] + 8 * (lane >> 5);
#pragma unroll
    for (int s = 0; s < D / 16; ++s) st.q[s] = *reinterpret_cast<const u32x4*>(qp + 16 * s);
#pragma unroll
    for (int x = 0; x < D / 32; ++x) st.o[x] = f32x16{};
    st.m = kNone;
    st.limit = kNone;
    st.l = 0.f;
}

// A value that the compiler does not know to be the same every time: what a rare branch computes from it is not
// computed ahead of the loop and held in registers.
__device__ __forceinline__ int opaque(int x) {
    asm volatile("" : "+v"(x));
    return x;
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
// Which of the 64 tokens from slot j on row r sees: of the context what its position does (without a window
// that says nothing but that the row is behind it), of the nodes those of its bits.
__device__ __forceinline__ uint64_t row_sees(const CacheAttnArgs& a, int r, int j, const Walk& k) {
    const int node = node_of(a, k, r), base = k.tr.base, len = k.tr.len;
    if (node < 0) return 0;
    uint64_t bits = 0;
    if (j < len && j + 63 >= base) {
        const int u = j - base, w = u >> 5;   // (u > -64: the words before the first are empty)
        const int32_t* row = a.seen + int64_t(node) * a.words;
        auto word = [&](int x) { return x >= 0 && x < a.words ? uint64_t(uint32_t(row[x])) : 0; };
        bits = (word(w) | (word(w + 1) << 32)) >> (u & 31);
        if (u & 31) bits |= word(w + 2) << (64 - (u & 31));
        bits &= below64(len - j);
    }
    const int pos = max(min(a.at ? a.at[node] : base, len - 1), base);
    const uint64_t context = below64(base - j);
    return (bits & ~context) | (context & (~below64(max(pos - a.W + 1, 0) - j) | below64(min(a.S - 1, pos) + 1 - j)));
}

// Where a page lies in LDS, as bf16.  Keys: a token's row of D columns, values: a column's row of 64 tokens, each row
// 16 bytes apart from the next, which puts the 16 rows that an LDS cycle serves into distinct banks.
template <int D>
struct TreePage {
    static constexpr int kKeyRow = 2 * D + 16, kValueRow = 2 * kPage + 16;
    static constexpr int kKeys = kPage * kKeyRow, kValues = D * kValueRow;   // bytes
};

// Which token a row of the S^T tiles stands for: those of a lane's accumulators, eight by eight, are eight
// tokens in a row, the B operand of the second product.
__device__ __forceinline__ int token_of(int i) { return (i & 16) + 2 * (i & 4) + ((i & 8) >> 1) + (i & 3); }

// A page's V scale: the power of two enters the values as they are converted, the mantissa (1, where an
// append wrote the page) the weights' exponent, as its logarithm, and leaves their sum again.
struct ValueScale {
    float power, shift, back;
};
__device__ __forceinline__ ValueScale value_scale(float x) {
    const float m = x > 0.f ? 2.f * __builtin_amdgcn_frexp_mantf(x) : x == 0.f ? 1.f : x;
    return ValueScale{__uint_as_float(__float_as_uint(x) & 0x7f800000u), fast_log2(m), 1.f / m};
}

// What a wave carries from one half of a page to the next: the logits of 32 tokens, and the weights of the
// 32 before them, whose product with the values is still to come.
struct TreeHalf {
    u32x4 p[2];
};

// The 32 tokens in `cur` become weights, while the matrix cores form the logits of the next 32 (keys at kb) and the
// product of the last ones (values at vb): each MFMA is followed by vector work that it covers.
template <int D>
__device__ __forceinline__ void tree_half(TreeRows<D>& st, const f32x16& cur, f32x16& next, TreeHalf& w, const uint8_t* kb,
                                          const uint8_t* vb, int vhalf, float fac, ValueScale vs) {
    constexpr int KS = D / 16, NB = D / 32;
    u32x4 kop[KS / 2], vop[NB];   // the next operands of either product
    auto read_k = [&](int s) { kop[s % (KS / 2)] = *reinterpret_cast<const u32x4*>(kb + 32 * s); };
    auto read_v = [&](int x) {
        vop[x % NB] = *reinterpret_cast<const u32x4*>(vb + 64 * vhalf + 32 * (x / NB) + 32 * TreePage<D>::kValueRow * (x % NB));
    };
#pragma unroll
    for (int s = 0; s < KS / 2; ++s) read_k(s);
#pragma unroll
    for (int x = 0; x < NB; ++x) read_v(x);
    const float shift = vs.shift - st.m;
    const u32x4 last[2] = {w.p[0], w.p[1]};
    float l[2] = {0.f, 0.f};
    auto weights = [&](int r0, int n) {   // pairs r0, r0 + 2, .. below r0 + n
#pragma unroll
        for (int r = r0; r < r0 + n && r < 16; r += 2) {
            const float x = fast_exp2(__builtin_fmaf(cur[r], fac, shift));
            const float y = fast_exp2(__builtin_fmaf(cur[r + 1], fac, shift));
            uint32_t xy = pack_bf16x2(x, y);
            l[0] += x;
            l[1] += y;
            asm volatile("" : "+v"(xy), "+v"(l[0]), "+v"(l[1]));   // here, beside the products, and not where they are used
            w.p[r >> 3][(r & 7) >> 1] = xy;
        }
    };
    // weights before the first product, and beside each pair of products
    constexpr int kAhead = 4, kEach = D == 128 ? 2 : 4;
    static_assert(KS == 2 * NB, "a step for each k-step of the logits and each product with values");
    __builtin_amdgcn_sched_barrier(0);
    weights(0, kAhead);
    int r = kAhead;
#pragma unroll
    for (int x = 0; x < KS; ++x) {
        next = mfma32(kop[x % (KS / 2)], st.q[x], x ? next : f32x16{});
        __builtin_amdgcn_sched_barrier(0);
        st.o[x % NB] = mfma32(vop[x % NB], last[x / NB], st.o[x % NB]);
        __builtin_amdgcn_sched_barrier(0);
        if (x < KS / 2) {
            read_k(x + KS / 2);
            read_v(x + NB);
        }
        weights(r, kEach);
        r += kEach;
        __builtin_amdgcn_sched_barrier(0);
    }
    st.l = __builtin_fmaf(l[0] + l[1], vs.back, st.l);
}

// The logits of the first 32 tokens.
template <int D>
__device__ __forceinline__ void tree_first(const TreeRows<D>& st, f32x16& next, const uint8_t* kb) {
    next = f32x16{};
#pragma unroll
    for (int s = 0; s < D / 16; ++s) next = mfma32(*reinterpret_cast<const u32x4*>(kb + 32 * s), st.q[s], next);
}

// The product of the weights that are left with their values.
template <int D>
__device__ __forceinline__ void tree_flush(TreeRows<D>& st, TreeHalf& w, const uint8_t* vb, int vhalf) {
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int b = 0; b < D / 32; ++b)
            st.o[b] = mfma32(*reinterpret_cast<const u32x4*>(vb + 64 * vhalf + 32 * g + 32 * TreePage<D>::kValueRow * b), w.p[g], st.o[b]);
    w.p[0] = w.p[1] = u32x4{};
}

// The logits of 32 tokens before they become weights: masks, and the running maximum, which moves only where
// it has to (the weights stay below 2^(kSlack + 1)).  It is a whole number, so that what moves by it moves by a
// power of two: the weights that wait for their product do exactly.
template <int D, class Sees>
__device__ __forceinline__ void tree_top(TreeRows<D>& st, f32x16& s, TreeHalf& w, bool part, Sees mask, float fac) {
    if (part) {
        const uint32_t sees = mask();
        keep_branch();
#pragma unroll
        for (int r = 0; r < 16; ++r)
            if (!((sees >> (16 * (r >> 3) + (r & 7))) & 1)) s[r] = -INFINITY;
    }
    float top = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
    top *= fac;
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
        st.m = m;
        st.limit = m + kSlack;
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
struct Share {
    int32_t item, total, each, lo, hi;   // the workgroup; units: all, of a run, of this one
    int32_t e, at;                       // the next tile and its first unit
    int32_t last;                        // the last workgroup that has a run
};
__device__ __forceinline__ int tile_units(const CacheAttnArgs& a, const PageList& l) {
    return int((uint32_t(l.count) + (1u << a.unit) - 1) >> a.unit);
}
__device__ __forceinline__ PageList pages_of_tile(const CacheAttnArgs& a, int e, int rows) {
    const int b = e / a.tiles;
    return tile_pages(a, tile_rows<true>(a, b, length_of(a, b), e % a.tiles, rows));
}
__device__ __forceinline__ bool open_share(const CacheAttnArgs& a, int rows, int lane, Share& s) {
    const int E = a.c.B * a.tiles;
    auto units = [&](int e) { return e < E ? tile_units(a, pages_of_tile(a, e, rows)) : 0; };
    int sum = 0;
    for (int e = lane; e < E; e += 64) sum += units(e);
    s.item = blockIdx.x / a.c.Hkv;
    s.total = __builtin_amdgcn_readlane(wave_scan(sum), 63);
    s.each = max((s.total + a.items - 1) / a.items, kMinChunk);
    s.last = max(s.total - 1, 0) / s.each;
    if (s.item > s.last) return false;
    s.lo = s.item * s.each;
    s.hi = min(s.lo + s.each, s.total);
    s.at = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {   // the first tile that ends behind lo, or lies there without pages
        const int n = units(e0 + lane), end = s.at + wave_scan(n);
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
    if (s.e >= a.c.B * a.tiles || !(s.at < s.hi || (s.at == s.total && s.item == s.last))) return false;
    k.hk = blockIdx.x % a.c.Hkv;
    k.b = s.e / a.tiles;
    k.tr = tile_rows<true>(a, k.b, __builtin_amdgcn_readfirstlane(length_of(a, k.b)), s.e % a.tiles, rows);
    k.pl = tile_pages(a, k.tr);
    const int n = tile_units(a, k.pl), end = s.at + n;
    const int first = min(s.at, max(s.total - 1, 0)) / s.each, last = n > 0 ? (end - 1) / s.each : first;
    k.ch = Chunk{s.e, first + s.e, last - first + 1, s.item - first, 0};
    k.c0 = int(min(int64_t(max(s.lo - s.at, 0)) << a.unit, int64_t(k.pl.count)));
    k.c1 = int(min(int64_t(min(s.hi, end) - s.at) << a.unit, int64_t(k.pl.count)));
    if (k.hk == 0 && k.ch.index == 0 && threadIdx.x == 0) {
        a.info[2 * s.e] = k.ch.first;
        a.info[2 * s.e + 1] = k.ch.count;
    }
    ++s.e;
    s.at = end;
    return true;
}

// A tile's rows over the pages [k.c0, k.c1) of its list.
constexpr int kTreeRows = 128;
template <int D>
__device__ __forceinline__ void tree_tile(const CacheAttnArgs& a, const Walk& k, uint8_t (*kb)[TreePage<D>::kKeys],
                                          uint8_t (*vb)[TreePage<D>::kValues]) {
    constexpr int NV = D / 64;   // 16-byte pieces of a page's keys, and of its values, per thread
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    // (the two workgroups of a CU start from either half of its SIMDs, so that tiles of up to 64 rows, which two waves
    // take, use them all)
    const int wr0 = k.tr.r0 + 32 * ((w + 2 * (blockIdx.x / 256 & 1)) & 3);
    const bool live = wr0 < a.T * (a.Hq / a.c.Hkv);
    TreeRows<D> st;
    open_tree_rows(a, st, k, wr0, lane);
    // this lane's operands: a token's columns from 8 h on, a column's tokens from 8 h on
    const int kat = token_of(lane & 31) * TreePage<D>::kKeyRow + 16 * (lane >> 5);
    const int vat = (lane & 31) * TreePage<D>::kValueRow + 16 * (lane >> 5);
    // what all rows see in full ends before the first node; what none sees lies before `far`
    const int base = k.tr.base, len = k.tr.len, far = base - a.W;
    auto in_part = [&](int t0) { return partly(t0, base - 1, len - 1, a.W, a.S); };
    u32x4 raw_k[2][NV], raw_v[2][NV];   // codes of two pages on their way, the even and the odd one
    auto load = [&](u32x4* raw, const uint8_t* codes, int page) {
        const uint8_t* p = codes + (int64_t(max(page, 0)) * a.c.Hkv + k.hk) * (kPage * D);
#pragma unroll
        for (int n = 0; n < NV; ++n) raw[n] = *reinterpret_cast<const u32x4*>(p + 16 * (tid + kThreads * n));
    };
    auto convert_keys = [&](u32x4* raw, int buf) {
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int x = tid + kThreads * n;
            u32x4* to = reinterpret_cast<u32x4*>(kb[buf] + x / (D / 16) * TreePage<D>::kKeyRow + 32 * (x % (D / 16)));
            to[0] = codes_to_bf16(raw[n].x, raw[n].y);
            to[1] = codes_to_bf16(raw[n].z, raw[n].w);
        }
    };
    // (Codes of tokens that no row sees may stand for anything, NaN among it, which a weight of 0 would not
    // remove: they are cleared.)
    auto convert_values = [&](u32x4* raw, int buf, int t0, float power) {
        if (in_part(t0)) {
            keep_branch();
            const int lim = min(a.S, len);
            const int x0 = t0 + 16 * (opaque(tid) & 3);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t keep = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int x = x0 + 4 * j + e;
                    if (x < len && (x > far || x < lim)) keep |= 0xffu << (8 * e);
                }
#pragma unroll
                for (int n = 0; n < NV; ++n) raw[n][j] &= keep;
            }
        }
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            u32x4* to = reinterpret_cast<u32x4*>(vb[buf] + (tid + kThreads * n) / 4 * TreePage<D>::kValueRow + 32 * (tid & 3));
            to[0] = codes_to_bf16(raw[n].x, raw[n].y, power);
            to[1] = codes_to_bf16(raw[n].z, raw[n].w, power);
        }
    };
    // Halves of pages: 2 i and 2 i + 1 are those of page i.  While half x becomes weights, the logits of half x + 1
    // and the product of half x - 1 with its values are formed.  Interval i, from barrier to barrier, takes the
    // halves 2 i + 1 and 2 i + 2: it reads the keys of page i + 1 and the values of page i, converts the keys of page
    // i + 2 and the values of page i + 1, and asks for the codes that the one after the next converts.
    const int n = k.c1 - k.c0;
    if (n > 0) {
        constexpr int kLooks = 60;   // pages looked up at a time, and the four after them
        Pages pages;
        ValueScale scales;
        int x0 = 0;
        auto look = [&](int x) {
            x0 = x;
            pages = look_up(a, k, k.c0 + x, 1, lane);
            scales = value_scale(pages.vs);
        };
        look(0);
        auto page = [&](int i) { return page_at(pages, i - x0); };
        auto start = [&](int i) { return page_start(page(i), k.pl.page(k.c0 + i)); };
        // (the factor stays above 0, as a masked logit times 0 would be NaN)
        auto factor = [&](int i) { return lane_value(pages.ks, i - x0); };
        auto scale_of = [&](int i) {
            return ValueScale{0.f, lane_value(scales.shift, i - x0), lane_value(scales.back, i - x0)};
        };
        auto load_k = [&](int i) {
            if (i < n) load(raw_k[i & 1], a.c.k, page(i));
        };
        auto load_v = [&](int i) {
            if (i < n) load(raw_v[i & 1], a.c.v, page(i));
        };
        auto values = [&](int i) { convert_values(raw_v[i & 1], i & 1, start(i), lane_value(scales.power, i - x0)); };
        load_k(0);
        load_v(0);
        load_k(1);
        load_v(1);
        __syncthreads();   // the tile before has been read
        convert_keys(raw_k[0], 0);
        load_k(2);
        values(0);
        load_v(2);
        if (n > 1) convert_keys(raw_k[1], 1);
        load_k(3);
        __syncthreads();
        // P: whether i is odd
        auto interval = [&](auto P, int i) {
            __syncthreads();
            // Of two waves that could issue the older one does: of the two workgroups of a CU the first took 316 us and
            // the second, then alone, 409 (8 contexts of up to 64K x 8 heads).  The second leads every other page: 372
            // and 382.
            if (blockIdx.x & 256) __builtin_amdgcn_s_setprio(P);
            if (i - x0 >= kLooks) look(i);
            if (i + 2 < n) convert_keys(raw_k[P], P);
            if (i + 4 < n) load(raw_k[P], a.c.k, page(i + 4));
            if (i + 1 < n) convert_values(raw_v[P ^ 1], P ^ 1, start(i + 1), lane_value(scales.power, i + 1 - x0));
            if (i + 3 < n) load(raw_v[P ^ 1], a.c.v, page(i + 3));
        };
        constexpr std::integral_constant<int, 0> kEven{};
        constexpr std::integral_constant<int, 1> kOdd{};
        if (!live) {
            for (int i = 0; i < n; i += 2) {
                interval(kEven, i);
                if (i + 1 < n) interval(kOdd, i + 1);
            }
            return;
        }
        f32x16 s0, s1;
        TreeHalf left{};   // (no weights yet: 0)
        // what this lane's row sees of half `half` of page i (asked for where some row does not see all)
        auto seen = [&](int i, int half) {
            return [=, &a, &k] {
                const int t0 = start(i) + 32 * half;
                const int l = opaque(lane);
                return uint32_t(row_sees(a, wr0 + (l & 31), t0, k) >> (8 * (l >> 5)));
            };
        };
        bool part = in_part(start(0));
        float fac = factor(0);
        ValueScale vs = scale_of(0);
        tree_first<D>(st, s0, kb[0] + kat);
        tree_top<D>(st, s0, left, part, seen(0, 0), fac);
        tree_half<D>(st, s0, s1, left, kb[0] + kat + 32 * TreePage<D>::kKeyRow, vb[0] + vat, 0, fac, vs);
        auto step = [&](auto P, int i) {
            const uint8_t *kn = kb[P ^ 1] + kat, *vn = vb[P] + vat, *kn2 = kn + 32 * TreePage<D>::kKeyRow;
            interval(P, i);
            tree_top<D>(st, s1, left, part, seen(i, 1), fac);
            tree_half<D>(st, s1, s0, left, kn, vn, 0, fac, vs);
            part = in_part(start(i + 1));
            fac = factor(i + 1);
            vs = scale_of(i + 1);
            tree_top<D>(st, s0, left, part, seen(i + 1, 0), fac);
            tree_half<D>(st, s0, s1, left, kn2, vn, 1, fac, vs);
        };
        int i = 0;
        for (; i + 2 < n; i += 2) {
            step(kEven, i);
            step(kOdd, i + 1);
        }
        if (i + 1 < n) step(kEven, i++);
        const uint8_t* vn = vb[i & 1] + vat;
        if (i & 1) interval(kOdd, i);
        else interval(kEven, i);
        tree_top<D>(st, s1, left, part, seen(i, 1), fac);
        tree_half<D>(st, s1, s0, left, kb[0] + kat, vn, 0, fac, vs);   // (logits of no page, for nothing)
        tree_flush<D>(st, left, vn, 1);
    }
    if (live) close_tree_rows(a, st, k, wr0, kTreeRows, lane);
}

template <int D>
__global__ void __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(D == 128 ? 2 : 3, D == 128 ? 2 : 3)))
tree_rows_kernel(CacheAttnArgs a) {
    __shared__ __attribute__((aligned(16))) uint8_t kb[2][TreePage<D>::kKeys], vb[2][TreePage<D>::kValues];
    const int lane = threadIdx.x & 63;
    Walk k;
    Share share;
    if (a.items > 0) {
        if (!open_share(a, kTreeRows, lane, share) || !next_tile(a, kTreeRows, share, k)) return;
    } else if (!open_walk<false, true>(a, kTreeRows, lane, k)) {
        return;
    }
    do {
        make_uniform(k);
        tree_tile<D>(a, k, kb, vb);
    } while (a.items > 0 && next_tile(a, kTreeRows, share, k));
}

}  // namespace

void launch_tree_rows(const CacheAttnArgs& a, dim3 grid, hipStream_t s) {
    if (a.c.d == 128) hipLaunchKernelGGL(tree_rows_kernel<128>, grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL(tree_rows_kernel<64>, grid, dim3(kThreads), 0, s, a);
}

hipError_t launch_tree_mask(const TreeMaskArgs& a, hipStream_t s) {
    TraceScope _t("tree_mask", s);
    hipLaunchKernelGGL(tree_mask_kernel, dim3(unsigned(a.B)), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace msparse
