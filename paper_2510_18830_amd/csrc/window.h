// Attention with a sliding window and a few first tokens that stay visible
// (sinks): what its forward and backward kernels share.
//
// Row i of a sequence of n tokens sees the keys j <= i with i - j < window or
// j < sinks.  Every row sees itself, so no row is empty.  Rows and keys are
// walked in tiles of 64 whose borders lie at multiples of 64 from the
// sequence's start; a tile is either seen in full by a wave's rows, not at all,
// or in part, and only then masked, from positions alone (no lists, no mask in
// memory).  Tensors are read where they lie (bf16, any batch, head and token
// stride): the tile loads take an address per lane anyway, and copies in another
// type or order would cost two passes over memory.
#pragma once

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "tiles.h"

namespace msparse {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// A bf16 tensor [batch, heads, tokens, d], rows contiguous; strides in elements.
struct RowView {
    uint16_t* p;
    int64_t batch, head, token;
};

// Most workgroups of a launch: 512 threads each stay below 2^32
constexpr int64_t kMaxGroups = int64_t(1) << 22;

// Blocks of `rows` rows that one head's sequences have, at most (packed: fewer than a grid
// with room for `seq` rows in every sequence).
inline int64_t row_blocks(int64_t B, int64_t seq, int64_t tokens, int64_t rows) {
    const int64_t all = B * ((seq + rows - 1) / rows);
    return tokens > 0 ? std::min(all, tokens / rows + B) : all;
}
// Grids of packed sequences: with room for `seq` rows in every sequence, so that walks can
// start in an order over all of them (cell_of), or, where few of these workgroups would
// find rows, by the tensors' rows: tokens / rows + B blocks, those of sequence b from the
// block starts[b] / rows + b on, which is at least as many as it needs before the next
// one's first.  A workgroup then looks its sequence up among the starts.
// Forward and backward in us, room for `seq` -> by rows, by the ratio of their blocks (12
// over 4 heads of dimension 64; 28 over 4 of 128):
//                                    no window                  window 1024, 4 sinks
//   1.7  16 of 100 to 4000 tokens    941 -> 1036, 3819 -> 4035  606 -> 616, 2420 -> 2381
//   2.2  12 of 400 to 1200, one 2200 233 -> 247,  863 -> 739    206 -> 202, 736 -> 729
//   3.1  16 of 300 to 1200, one 3000 315 -> 329,  1162 -> 1004  267 -> 240, 899 -> 806
//   3.6  12 of 600 to 2500, one 8000 1097 -> 1007, 4019 -> 3312 486 -> 442, 1843 -> 1766
//   32   64 of 30 to 400, one 16384  3446 -> 2179, 13316 -> 8513 915 -> 392, 3005 -> 1549
inline bool grid_by_rows(int64_t B, int64_t Hq, int64_t seq, int64_t tokens) {
    constexpr int64_t kRoom = 2;
    const int64_t all = B * ((seq + 63) / 64);
    return tokens > 0 && (all > kRoom * (tokens / 64 + B) || all > kMaxGroups / Hq);
}
inline int64_t grid_blocks(bool by_rows, int64_t B, int64_t seq, int64_t tokens, int64_t rows) {
    return by_rows ? tokens / rows + B : B * ((seq + rows - 1) / rows);
}

// The key-major backward's workgroups for a group of keys: near_slots for the query
// tiles of its window (every head of the KV group: near_chunk of them each), and for
// one with sinks far_slots for the tiles beyond (far_chunk each, no more than a
// window's: 8 heads x 2048, window 256, sinks 4, head dim 128: dK / dV 34 us with 16
// tiles each, 24 with 6).  A group with more than one leaves partial sums: those with
// sinks, or, where windows are cut too, all of them.
//
// Grids by rows: windows are not cut.  The chunks of all sequences share far_slots for a
// KV head and sink group, those of sequence b from the slot far_slot(b) on, and only groups
// with rows beyond their window leave partial sums, by far_index(b): the sequence itself,
// or, where fewer can be long enough for such rows (far_unit tokens at least), its start
// in units of that length.
struct KeyPlan {
    int32_t near_slots, near_chunk, sink_groups, far_slots, far_chunk, part_groups;
    int32_t far_docs, far_unit;
};
// Windows are cut, into 8 tiles at least:
//   d 64    while all workgroups are resident at once, three a CU, which pays for the sums
//           (dK / dV and sums 36 -> 30 us for 8 x 1024 causal, 64 groups; 58 -> 48 for 8 x
//           2048); beyond that it costs (16 x 2048, 256 groups at head dim 128: 61 -> 85)
//   d 128   one workgroup a CU walks alone, so where that shortens the longest walk by
//           more than the further starts and the partial sums cost, by a model of the time
//           of sequences of the mean length: the longest walk, or all walks over the CUs
//           and a last round, kStart steps (a tile each) for each workgroup's start, kStep
//           us a step; the sums a launch and their bytes twice at 4 TB/s (backward in us,
//           cut while all are resident -> by the model: 16 over 2 heads x 8192 causal 1135 ->
//           1015, 28 over 4 x 4096 529 -> 491, 5 documents of 8000 tokens together of 8 over 2
//           heads 342 -> 261; 10 of 3563 of 12 over 4 84 -> 88)
inline KeyPlan key_plan(int64_t B, int64_t Hkv, int64_t G, int64_t seq, int64_t tokens, int64_t W, int64_t S, int d,
                        int64_t keys, int64_t resident, bool by_rows) {
    KeyPlan p{1, 1, 0, 0, 1, 0, 0, 0};
    if (seq <= 0) return p;
    const int64_t tiles = (seq + 63) / 64, groups = (seq + keys - 1) / keys, bk = B * Hkv;
    const int64_t wide = std::min(tiles, (keys + W - 2) / 64 + 1);   // query tiles of a group's window and head
    const int64_t walk = G * wide, first = W / 64;   // (the rows of tiles before are inside the window of key 0)
    if (by_rows) {
        p.near_chunk = int32_t(walk);
        if (S == 0 || W >= seq || first >= tiles) return p;
        p.sink_groups = p.part_groups = int32_t((std::min(S, seq) + keys - 1) / keys);
        const int64_t least = 64 * ((keys - 2 + W) / 64 + 1) + 1;   // rows of a sequence with some beyond a window
        p.far_docs = int32_t(std::min(B, tokens / least + 1));
        p.far_unit = p.far_docs < B ? int32_t(least) : 0;
        const int64_t items = std::max<int64_t>(1, std::min<int64_t>(256, 1024 / (Hkv * p.sink_groups)));
        p.far_chunk = int32_t(std::max(std::min<int64_t>(16, walk), (G * (tokens / 64) + items - 1) / items));
        p.far_slots = int32_t(G * (tokens / 64 + B) / p.far_chunk + p.far_docs);
        return p;
    }
    if (S > 0 && W < seq && first < tiles) {
        p.sink_groups = p.part_groups = int32_t((std::min(S, seq) + keys - 1) / keys);
        const int64_t beyond = G * (tiles - first);      // query tiles beyond a group's window, at most
        const int64_t items = std::max<int64_t>(1, std::min<int64_t>(256, 1024 / (bk * p.sink_groups)));
        p.far_chunk = int32_t(std::max(std::min<int64_t>(16, walk), (beyond + items - 1) / items));
        p.far_slots = int32_t((beyond + p.far_chunk - 1) / p.far_chunk);
    }
    p.near_chunk = int32_t(walk);
    // (the grid and the partial sums have room for `seq` keys in every sequence)
    const int64_t most = std::min(walk / 8, 16 * resident / (bk * groups));
    if (d == 64) {
        const int64_t room = resident - bk * p.sink_groups * p.far_slots;
        const int64_t cuts = std::min(room / (Hkv * row_blocks(B, seq, tokens, keys)), most);
        if (cuts > 1) p.near_chunk = int32_t((walk + cuts - 1) / cuts);
    } else {
        const int64_t length = tokens > 0 ? std::min(seq, (tokens + B - 1) / B) : seq;   // of the mean sequence
        const int64_t n = (length + keys - 1) / keys, last = (length + 63) / 64;
        const double kStep = 1.8, kStart = 8, part_us = double(2 * 2 * keys * d * 4) / 4e6;
        const int64_t far = bk * p.sink_groups * G * std::max<int64_t>(last - first, 0);
        double best = 0;
        for (int64_t cuts = 1; cuts <= std::min<int64_t>(most, 8) && bk * n <= 4 * resident; ++cuts) {
            const int64_t chunk = (walk + cuts - 1) / cuts;
            int64_t chunks = 0, total = far;
            for (int64_t g = 0; g < n; ++g) {
                const int64_t steps = G * std::min(wide, last - g * keys / 64);
                chunks += bk * ((steps + chunk - 1) / chunk);
                total += bk * steps;
            }
            double steps = (double(total) + kStart * double(chunks)) / double(resident);
            // a last round, of the last groups' walks (from 85 % on, as XCDs get uneven numbers)
            const int64_t late = G * std::min(wide, last - n * 3 / 4 * keys / 64);
            if (20 * chunks > 17 * resident) steps += double(std::min(chunk, late));
            const double us = std::max(steps, double(chunk) + kStart) * kStep +
                              (cuts > 1 ? 7 + part_us * double(chunks) : 0.0);
            if (cuts == 1 || us < best) {
                best = cuts == 1 ? 0.95 * us : us;
                p.near_chunk = int32_t(chunk);
            }
        }
    }
    p.near_slots = int32_t((walk + p.near_chunk - 1) / p.near_chunk);
    if (p.near_slots > 1) p.part_groups = int32_t(groups);
    return p;
}

struct WindowArgs {
    RowView q, k, v, out, dout, dq, dk, dv;
    float* lse;            // [batch, Hq, seq], packed: [Hq, tokens]
    const int32_t* starts; // packed: [batch + 1] first rows of the sequences (NULL: batch x seq)
    int64_t tokens;        // packed: rows of every tensor
    int32_t B, Hq, Hkv, seq, d;
    int32_t W, S;          // W = INT32_MAX: no window
    float scale;
    bool by_rows;          // grids by the rows of the packed tensors
    // backward workspace
    float* rows;           // [Hq][2][rows_pad]: lse log2(e) and Delta of every row, sequences from a multiple of 64 on
    int64_t rows_pad;
    float* part;           // partial dK, dV: [lines part_groups][near_slots], then [B Hkv sink_groups][far_slots],
    KeyPlan plan;          //   each [2][keys of a group][d]; lines = B Hkv, by rows Hkv far_docs (and Hkv for B Hkv)
};

// Where sequence b lies: `row` its first row (packed), n its length.  Starts out
// of order or beyond the tensors are cut to [0, tokens], lengths to `seq`.
struct Sequence {
    int64_t row;
    int32_t b, n;
};
__device__ __forceinline__ int64_t cut_start(const WindowArgs& a, int32_t start) {
    return min(max(int64_t(start), int64_t(0)), a.tokens);
}
__device__ __forceinline__ Sequence sequence(const WindowArgs& a, int b) {
    Sequence s{0, b, a.seq};
    if (a.starts) {
        const int64_t r0 = cut_start(a, ldc(a.starts, b));
        const int64_t r1 = max(cut_start(a, ldc(a.starts, b + 1)), r0);
        s.row = r0;
        s.n = int32_t(min(r1 - r0, int64_t(a.seq)));
    }
    return s;
}
__device__ __forceinline__ uint16_t* head_rows(const WindowArgs& a, const RowView& v, const Sequence& s, int h) {
    return v.p + (a.starts ? s.row * v.token : s.b * v.batch) + h * v.head;
}
__device__ __forceinline__ int64_t lse_row(const WindowArgs& a, const Sequence& s, int h) {
    return a.starts ? h * a.tokens + s.row : (int64_t(s.b) * a.Hq + h) * a.seq;
}
// First row of a sequence in the backward's row values.  Packed sequences take
// whole blocks of 64: the next multiple of 64 plus one block for each sequence
// before, so that two never share one.
__host__ __device__ inline int64_t padded_rows(int64_t n) { return (n + 63) / 64 * 64; }
__device__ __forceinline__ int64_t value_row(const WindowArgs& a, const Sequence& s) {
    return a.starts ? padded_rows(s.row) + 64 * int64_t(s.b) : s.b * padded_rows(a.seq);
}

// Grids by rows.  What sequence b has its own of, counted over all: first(start, b), which
// ascends.  The last sequence with first <= x, 64 looked at in a step, one a lane.
template <class First>
__device__ __forceinline__ int last_sequence(const WindowArgs& a, int64_t x, First first) {
    const int lane = threadIdx.x & 63;
    int b = 0, n = a.B;   // it is one of b .. b + n - 1
    while (n > 1) {
        const int step = (n + 63) / 64;
        const bool in = lane * step < n;
        const int mine = in ? b + lane * step : b;
        const uint64_t upto = __ballot(in && first(cut_start(a, a.starts[mine]), mine) <= x);
        const int l = upto ? 63 - __builtin_clzll(upto) : 0;
        b += l * step;
        n = min(step, n - l * step);
    }
    return __builtin_amdgcn_readfirstlane(b);
}
__device__ __forceinline__ int64_t first_block(int64_t start, int b, int rows) { return start / rows + b; }
// (sequence, its block) of block x of `rows` rows; a block of none: -1
__device__ __forceinline__ void block_of(const WindowArgs& a, int64_t x, int rows, int& b, int& block) {
    b = last_sequence(a, x, [&](int64_t start, int i) { return first_block(start, i, rows); });
    block = int(max(x - first_block(cut_start(a, ldc(a.starts, b)), b, rows), int64_t(-1)));
}
// First slot of a sequence's chunks of sink rows, and its place among the partial sums.
__device__ __forceinline__ int64_t far_index(const WindowArgs& a, int64_t start, int b) {
    return a.plan.far_unit > 0 ? start / a.plan.far_unit : b;
}
__device__ __forceinline__ int64_t far_slot(const WindowArgs& a, int64_t start, int b) {
    return a.Hq / a.Hkv * first_block(start, b, 64) / a.plan.far_chunk + far_index(a, start, b);
}

// The key tiles that the rows i0 .. i1 see: those of the window from the
// diagonal down (the running maximum is set early), then the sinks'.
struct KeyWalk {
    int32_t hi, window_tiles, tiles, sink_tiles;
    __device__ __forceinline__ int32_t tile(int t) const {
        return t < window_tiles ? hi - t : tiles - 1 - t;
    }
};
__device__ __forceinline__ KeyWalk key_walk(int i0, int i1, int W, int S) {
    KeyWalk k;
    k.hi = i1 >> 6;
    const int lo = max(i0 - W + 1, 0) >> 6;   // W <= INT32_MAX: no overflow for i0 >= 0
    k.window_tiles = k.hi - lo + 1;
    k.sink_tiles = min((S + 63) >> 6, lo);
    k.tiles = k.window_tiles + k.sink_tiles;
    return k;
}

// How rows i0 .. i1 see keys j0 .. j1.
enum Sight { kNone, kPart, kFull };
__device__ __forceinline__ Sight sight(int i0, int i1, int j0, int j1, int W, int S) {
    if (j0 > i1 || (j1 <= i0 - W && j0 >= S)) return kNone;
    if (j1 <= i0 && (j0 > i1 - W || j1 < S)) return kFull;
    return kPart;
}
// i sees j; lim = min(S - 1, i)
__device__ __forceinline__ bool sees(int i, int j, int W, int lim) {
    return uint32_t(i - j) < uint32_t(W) || j <= lim;
}

// 64 rows from row0 on (rows past the end: the last one) into a DMA tile.
template <int D, int P, int NW>
__device__ __forceinline__ void dma_sequence(uint16_t* tile, const uint16_t* src, int64_t stride, int row0, int last,
                                             int wave, int lane) {
    using T = DmaTile<D, P>;
    constexpr int NC = D / 8;
    static_assert(T::kGroups % NW == 0, "whole instructions per wave");
#pragma unroll
    for (int j = 0; j < T::kGroups / NW; ++j) {
        const int g = wave + NW * j;
        const int r = min(row0 + g + T::kGroups * (lane / NC), last);
        dma16(src + r * stride + (lane % NC) * 8, lds_addr(tile + T::goff(g) / 2));
    }
}

// 8 consecutive accumulator values to bf16 x 8
template <int BASE>
__device__ __forceinline__ u32x4 pack8_bf16(const f32x16& acc) {
    u32x4 r;
    r.x = pack_bf16x2(acc[BASE + 0], acc[BASE + 1]);
    r.y = pack_bf16x2(acc[BASE + 2], acc[BASE + 3]);
    r.z = pack_bf16x2(acc[BASE + 4], acc[BASE + 5]);
    r.w = pack_bf16x2(acc[BASE + 6], acc[BASE + 7]);
    return r;
}

// Where item u of `lines` x `cells` items lies: the first kRun cells of every line, then
// the next ones.  A line is a (sequence, KV head); its cells are row tiles, the last
// first, or groups of keys, the first first: where there is no window the longest walks
// start first in all lines, and a run's neighbours share tiles in an XCD's L2.  (Line
// after line, 28 over 4 heads x 16K without a window took 1913 us forward, 2480 dQ and
// 4700 dK / dV, so 1870, 2420 and 3320; 7 documents of 20K tokens together, window 1024,
// 780 us dK / dV, so 690; one sequence in a window takes the same.)
constexpr int kRun = 8;
__device__ __forceinline__ void cell_of(int64_t u, int64_t lines, int cells, int& line, int& cell) {
    const int first = int(u / (kRun * lines)) * kRun, run = min(cells - first, kRun);
    const int64_t r = u - first * lines;
    line = int(r / run);
    cell = first + int(r % run);
}
// (sequence, head, tile of `rows` rows) of workgroup t; the heads of a group are
// neighbours.  False where there is none.
template <bool BY_ROWS>
__device__ __forceinline__ bool window_tile_of(const WindowArgs& a, int64_t t, int rows, int& b, int& h, int& tile) {
    const int G = a.Hq / a.Hkv, cells = BY_ROWS ? int(a.tokens / rows) + a.B : (a.seq + rows - 1) / rows;
    const int64_t lines = BY_ROWS ? a.Hkv : int64_t(a.B) * a.Hkv, u = xcd_chunk(t, lines * cells * G);
    int line, cell;
    cell_of(u / G, lines, cells, line, cell);
    tile = cells - 1 - cell;
    h = line % a.Hkv * G + int(u % G);
    b = line / a.Hkv;
    if (!BY_ROWS) return true;
    block_of(a, tile, rows, b, tile);
    return tile >= 0;
}

// f(head dim, whether the grid is by rows), as types: the kernels' template arguments.  (A
// test in the kernels instead costs dK / dV 1.5 % where the grid is not by rows.)
template <class F>
void window_variant(const WindowArgs& a, F f) {
    const auto by_dim = [&](auto by_rows) {
        if (a.d == 128) f(std::integral_constant<int, 128>(), by_rows);
        else f(std::integral_constant<int, 64>(), by_rows);
    };
    if (a.by_rows) by_dim(std::true_type());
    else by_dim(std::false_type());
}

hipError_t launch_window_fwd(const WindowArgs& a, hipStream_t s);
hipError_t launch_window_bwd(const WindowArgs& a, hipStream_t s);
// Keys that a workgroup of the key-major backward takes, and how many of them run at once.
int window_key_group(int d);
int window_key_resident(int d);

}  // namespace msparse
