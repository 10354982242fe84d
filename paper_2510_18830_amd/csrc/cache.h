// Paged 8-bit cache of keys and values: what the append and the attention over
// it share.
//
// A page holds 64 tokens of every KV head: K codes [64][d] (a token's row is
// contiguous, as its key is read whole) and V codes [d][64] (a column's 64 tokens
// are contiguous: the operand of P V^T runs over tokens, so the attention reads
// either from memory straight into registers, 16 bytes a lane, without LDS).
// Codes are e4m3 (OCP: bias 7, no infinities, 0x7f NaN), with one fp32 scale per
// page and head for K and one for V: value = code * scale.
#pragma once

#include <algorithm>

#include "common.h"
#include "rotary.h"

namespace msparse {

constexpr int kPage = 64;
constexpr int kMaxWidth = 1 << 24;   // pages of a sequence: tokens with a page stay below 2^30
constexpr int kMaxLength = INT32_MAX - (kPage - 1);   // longest sequence; a page that starts here is beyond every row

struct CacheView {
    uint8_t* k;           // [pages, Hkv, 64, d]
    uint8_t* v;           // [pages, Hkv, d, 64]
    float* ks;            // [pages, Hkv]
    float* vs;
    const int32_t* table; // [B, width]: page of each 64 tokens of a sequence
    const int32_t* lens;  // [B]
    int32_t pages, width;
    int32_t B, Hkv, d;
};
// the page of tokens 64 p .. 64 p + 63 of sequence b, -1 if there is none
__device__ __forceinline__ int32_t cache_page(const CacheView& c, int b, int p) {
    if (p >= c.width) return -1;
    const int32_t x = ldc(c.table, int64_t(b) * c.width + p);
    return uint32_t(x) < uint32_t(c.pages) ? x : -1;
}

struct AppendArgs {
    CacheView c;
    const uint16_t *q, *k, *v;                // bf16 [B, heads, T, d]
    int64_t qs[3], ks[3], vs[3], qos[3];      // strides: sequence, head, token
    uint16_t* qout;
    const float* freq;                        // [d / 2] or NULL: no rotation
    Positions pos;                            // pos.at != NULL: in place of lens[b] + t and freq
    const int32_t* counts;                    // [B] or NULL: T
    int32_t Hq, T;
    int32_t P;                                // pages that T tokens can touch
    // workgroups that share a page's KV heads, and its query heads
    int32_t kv_shares, q_shares;
};
// Pairs of columns that a thread takes of a query token, and how many heads' queries a
// workgroup turns side by side where the new tokens of a page are few.
constexpr int kAppendThreads = 256;
constexpr int query_chunks(int d) { return d / 16; }
constexpr int heads_aside(int tokens, int d) {
    return tokens * query_chunks(d) < kAppendThreads ? kAppendThreads / (tokens * query_chunks(d)) : 1;
}
// The shares of a page's heads, a workgroup each, keys and queries apart.  Of the keys'
// heads two each and four shares at the least, more where the pages are few, of 32 heads
// four each; of the queries' steps six each, fewer where the pages are few.  (35 calls of
// 16 to 2049 pages with 1, 2, 4, 8, .. of the one and 0 to 32 of the other: these stay
// within a tenth or so of each call's best.  A workgroup for both, at 576 pages of 28
// over 4 heads 133 us, waits longer than two, 94; one of all heads of 128 sequences of
// one token for eight heads in a row: 21 us, of two 15.)
inline int even_shares(int64_t heads, int64_t shares) {
    const int64_t each = (heads + shares - 1) / shares;
    return int((heads + each - 1) / each);
}
inline void share_heads(AppendArgs& a, int64_t pages) {
    const int64_t hkv = a.c.Hkv, aside = heads_aside(std::min(a.T, kPage), a.c.d), steps = (a.Hq + aside - 1) / aside;
    a.kv_shares = even_shares(hkv, std::min(hkv, std::max({int64_t(4), hkv / 4, 600 / pages})));
    a.q_shares = a.q ? even_shares(steps, std::min(steps, std::max((steps + 5) / 6, 512 / pages - a.kv_shares))) : 0;
    // With positions given, angles cost more than a share of the heads saves where the card is full anyway (us: 2 x
    // 20011 tokens, 28 over 4 heads 157 -> 138; 131072, 32 over 8 652 -> 568; 16 x 500, 28 over 4 41.7 -> 38.2; 64 x 64
    // 27.2 -> 26.7; but 40 x 64, 12 over 4 of 64 columns 11.2 -> 12.8, 64 x 16, 28 over 4 12.6 -> 14.7).
    if (a.pos.at && int64_t(a.c.B) * a.T >= 4096) {
        a.kv_shares = even_shares(hkv, std::min(hkv, std::max(int64_t(2), hkv / 8)));
        a.q_shares = a.q ? even_shares(steps, (steps + 11) / 12) : 0;
    }
}
hipError_t launch_cache_append(const AppendArgs& a, hipStream_t s);

struct CacheAttnArgs {
    CacheView c;
    const uint16_t* q;      // bf16 [B, Hq, T, d]
    int64_t qs[3], os[3];
    uint16_t* out;
    float* lse;             // [B, Hq, T] or NULL
    int32_t Hq, T, W, S;    // W = INT32_MAX: no window
    float scale;
    int32_t tiles;          // row tiles of a (sequence, KV head): its G T rows
    int32_t items;          // chunks aimed at per KV head; 0: chunks of `chunk` pages, up to per_tile of a row tile
    int32_t chunk, per_tile;
    int32_t unit;           // log2 of the pages that the sum over all tiles counts in
    // workspace (slots > 0)
    int32_t* info;          // [B tiles][2]: first chunk, chunks
    float* po;              // [slots, Hkv, rows, d]: sums of the weighted values
    float* pml;             // [slots, Hkv, rows, 2]: running maximum (log2 units), sum of the weights
    int32_t slots;          // 0: one chunk per row tile, nothing to join
    // a tree's nodes (seen != NULL): what row t of a sequence sees among them, its position, their number
    const int32_t* seen;    // [B, T, words]
    const int32_t* at;      // [B, T], NULL without a window
    const int32_t* counts;  // [B] or NULL: T
    int32_t words;
};
// Row tiles and chunks of a call.  rows = G T rows of a (sequence, KV head).
struct CacheAttnPlan {
    int32_t rt, wr;         // 16-row tiles per wave; waves of a workgroup over rows (1: over pages)
    int32_t rows;           // rows of a workgroup
    int32_t tiles, items, chunk, per_tile, unit, slots;
    bool wide;              // a workgroup of many waves per tile
    bool even;              // a tree's many rows: pages dealt to `items` workgroups per KV head, across tiles
};
// workgroups per KV head
inline int64_t cache_attn_groups(const CacheAttnPlan& p, int64_t B) {
    return p.even ? p.items : p.slots > 0 ? p.slots : B * p.tiles;
}
CacheAttnPlan cache_attn_plan(int64_t B, int64_t Hq, int64_t Hkv, int64_t T, int64_t width, int d, int64_t W,
                              int64_t S, bool tree = false);
constexpr int kMaxNodes = 1024;    // of a tree
struct TreeMaskArgs {
    const int32_t* parents; // [B, T]
    const int32_t* lens;    // [B]: tokens before the tree
    const int32_t* counts;  // [B] or NULL: T
    int32_t* at;            // [B, T]
    int32_t* seen;          // [B, T, words]
    int32_t B, T, words, W, S;
};
hipError_t launch_tree_mask(const TreeMaskArgs& a, hipStream_t s);


struct KeepArgs {
    CacheView c;
    const int32_t* counts;  // [B] or NULL: T
    const int32_t* path;    // [B, T]
    const int32_t* kept;    // [B]
    int32_t T;
};
hipError_t launch_cache_keep(const KeepArgs& a, hipStream_t s);

constexpr int kMaxForks = 65536;   // sequences: each looks through all sources
struct ForkArgs {
    CacheView c;
    const int32_t* refs;    // [pages]
    const int32_t* src;     // [N]
    const int32_t* room;    // [N] or NULL
    int32_t* refs_out;      // [pages], may be refs
    int32_t* table_out;     // [N, width]
    int32_t* lens_out;      // [N]
    int32_t* missing;       // [N]
    int32_t N;
    // workspace
    int32_t* need;          // [N]: pages asked for, then those asked for before
    int32_t* list;          // the number of free pages found, and they; or a copy of refs
    int32_t cap;            // pages that the list has room for
};
hipError_t launch_cache_fork(const ForkArgs& a, hipStream_t s);

// a tree's rows in tiles of 128, a workgroup of 256 threads for each place of the grid
void launch_tree_rows(const CacheAttnArgs& a, int rows, dim3 grid, hipStream_t s);
hipError_t launch_cache_attn(const CacheAttnArgs& a, const CacheAttnPlan& p, hipStream_t s);

}  // namespace msparse
