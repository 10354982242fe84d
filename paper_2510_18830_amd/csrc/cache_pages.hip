// Rearranging what the paged cache holds: the tokens of an accepted path move to the
// places behind the context, and sequences continue others, their full pages shared.
#include "cache.h"
#include "codes.h"
#include "trace.h"

namespace msparse {

namespace {

constexpr int kThreads = 256;

// ---------------------------------------------------------------- tokens
// Slot L0 + i takes what slot L0 + path[i] holds (L0: the context's length).  A path ascends, so a
// target's source lies at or behind it, and runs of kKeepPages pages done in ascending order read what
// no earlier one has written.  A workgroup owns the keys or the values of one head of a sequence: it
// looks up where the tokens of a run lie (a thread a slot), reads their codes into LDS, finds each
// page's scale (its own, or what tokens from other pages need) and writes them, older tokens too
// where the scale has grown.
// Bound by latency, lengths, path, table, scales, codes, one after the other for each run, and with many
// tokens by V's bytes, one by one of their columns.  Pages one by one, by two, by four (us): 64 sequences,
// 8 heads of 128, 5 tokens kept of 16 8.4, 7.5, 7.8; 256 of them 19.8, 17.3, 23.2 (fewer fit a CU); 32 with
// 128 of 256 43.5, 40.3, 37.8; 7, 2 heads of 64, 100 of 200 20.2, 17.8, 16.4.
constexpr int kKeepPages = 2, kRun = kKeepPages * kPage;   // pages of a run, their slots
constexpr int kFlight = 4;   // a thread's loads in flight
template <int D>
__global__ void __launch_bounds__(kThreads) cache_keep_kernel(KeepArgs a) {
    constexpr int kRow = D + 16;
    __shared__ __attribute__((aligned(16))) uint8_t tok[kRun * kRow];   // the moved tokens' codes, [slot][column]
    __shared__ int from[kRun];      // the page where a slot's token lies, -1: it stays
    __shared__ int slot_of[kRun];   // its slot there
    __shared__ float was_of[kRun];  // and its scale there
    __shared__ int page_of[kKeepPages], others[kKeepPages];
    __shared__ float scale_of[kKeepPages];
    __shared__ uint32_t top_of[kKeepPages];             // the largest value from other pages
    const int tid = threadIdx.x;
    const bool value = blockIdx.x & 1;
    const int hk = (blockIdx.x >> 1) % a.c.Hkv, b = (blockIdx.x >> 1) / a.c.Hkv;
    const int len = min(max(ldc(a.c.lens, b), 0), kMaxLength);
    const int nodes = min(a.counts ? min(max(ldc(a.counts, b), 0), a.T) : a.T, len);
    const int first = len - nodes, kept = min(max(ldc(a.kept, b), 0), nodes);
    if (kept == 0) return;
    uint8_t* codes = value ? a.c.v : a.c.k;
    float* scales = value ? a.c.vs : a.c.ks;
    auto base = [&](int page) { return codes + (int64_t(page) * a.c.Hkv + hk) * (kPage * D); };
    auto largest = [&](uint32_t w, float sc) {
        const float x[4] = {__builtin_amdgcn_cvt_f32_fp8(w, 0), __builtin_amdgcn_cvt_f32_fp8(w, 1),
                            __builtin_amdgcn_cvt_f32_fp8(w, 2), __builtin_amdgcn_cvt_f32_fp8(w, 3)};
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) top = fmaxf(top, finite_abs(x[j] * sc));
        return top;
    };
    for (int lp0 = first / kPage; lp0 <= (first + kept - 1) / kPage; lp0 += kKeepPages) {
        // the run's slots that take a token
        const int c0 = max(first - lp0 * kPage, 0), c1 = min(first + kept - lp0 * kPage, kRun);
        if (tid < kRun) {
            const int i = min(max(lp0 * kPage + tid - first, 0), kept - 1), u = a.path[int64_t(b) * a.T + i];
            const int page = tid / kPage < (c1 + kPage - 1) / kPage ? cache_page(a.c, b, lp0 + tid / kPage) : -1;
            const bool takes = page >= 0 && tid >= c0 && tid < c1 && u > i && u < nodes;
            const int slot = takes ? first + u : 0, p = cache_page(a.c, b, slot / kPage), f = takes ? p : -1;
            const float was = scales[int64_t(max(page, 0)) * a.c.Hkv + hk];
            const float there = scales[int64_t(max(f, 0)) * a.c.Hkv + hk];
            const bool moves = f >= 0 && f != page;
            from[tid] = f;
            slot_of[tid] = slot % kPage;
            was_of[tid] = moves ? there : was;
            const bool some = __any(moves);   // (a wave is a page)
            if (tid % kPage == 0) {
                page_of[tid / kPage] = page;
                others[tid / kPage] = some;
                scale_of[tid / kPage] = was;
                top_of[tid / kPage] = 0;
            }
        }
        __syncthreads();
        // the moved tokens' codes; the largest value among those of other pages, for each page
        float top[kKeepPages] = {};
        auto note = [&](float x, int c) {
#pragma unroll
            for (int g = 0; g < kKeepPages; ++g) top[g] = fmaxf(top[g], c / kPage == g ? x : 0.f);
        };
        if (!value) {
            constexpr int C = D / 16;   // pieces of a token
            for (int x = c0 * C + tid; x < c1 * C; x += kThreads) {
                const int c = x / C, y = x % C, f = from[c];
                const u32x4 w = *reinterpret_cast<const u32x4*>(base(max(f, 0)) + slot_of[c] * D + 16 * y);
                if (f < 0) continue;
                *reinterpret_cast<u32x4*>(tok + c * kRow + 16 * y) = w;
                if (f != page_of[c / kPage])
#pragma unroll
                    for (int j = 0; j < 4; ++j) note(largest(w[j], was_of[c]), c);
            }
        } else {
            for (int x0 = c0 * D + tid; x0 < c1 * D; x0 += kFlight * kThreads) {
                uint8_t w[kFlight];
#pragma unroll
                for (int e = 0; e < kFlight; ++e) {   // (of a token that stays, any byte)
                    const int x = min(x0 + e * kThreads, c1 * D - 1), c = x / D;
                    w[e] = base(max(from[c], 0))[x % D * kPage + slot_of[c]];
                }
#pragma unroll
                for (int e = 0; e < kFlight; ++e) {
                    const int x = x0 + e * kThreads, c = x / D;
                    if (x >= c1 * D || from[c] < 0) continue;
                    tok[c * kRow + x % D] = w[e];
                    if (from[c] != page_of[c / kPage])
                        note(finite_abs(__builtin_amdgcn_cvt_f32_fp8(w[e], 0) * was_of[c]), c);
                }
            }
        }
#pragma unroll
        for (int g = 0; g < kKeepPages; ++g)
            if (others[g]) {
                const float most = wave_max(top[g]);
                if (tid % 64 == 0) atomicMax(top_of + g, __float_as_uint(most));
            }
        __syncthreads();   // also: every read of these pages is done
        for (int g = 0; g < kKeepPages; ++g) {
            const int page = page_of[g];
            const int s0 = max(c0 - g * kPage, 0), s1 = min(c1 - g * kPage, kPage);   // slots that take a token
            if (page < 0 || s0 >= s1) continue;
            const int at0 = g * kPage;   // of the page's slots in the run
            const float was = scale_of[g];
            const float now = others[g] ? fmaxf(was, code_scale(__uint_as_float(top_of[g]))) : was;
            const bool grown = now > was;
            if (!value) {   // every word of a moved token, or, where the scale has grown, an older one
                const int r0 = grown ? 0 : s0;
                for (int x = tid; x < (s1 - r0) * (D / 4); x += kThreads) {
                    const int s = r0 + x / (D / 4), c = x % (D / 4);
                    const int f = s < s0 ? -1 : from[at0 + s];
                    if (f < 0 && !grown) continue;
                    uint32_t* at = reinterpret_cast<uint32_t*>(base(page) + s * D) + c;
                    const uint32_t w = f < 0 ? *at : *reinterpret_cast<const uint32_t*>(tok + (at0 + s) * kRow + 4 * c);
                    const float sc = f < 0 ? was : was_of[at0 + s];
                    *at = sc == now ? w : rescale4(w, sc / now);
                }
            } else {   // a thread a row: every word that holds a slot of one
                const int w0 = grown ? 0 : s0 / 4, w1 = (s1 + 3) / 4;
                for (int w = w0 + tid / D; w < w1; w += kThreads / D) {
                    const int row = tid % D;
                    uint32_t* at = reinterpret_cast<uint32_t*>(base(page) + row * kPage) + w;
                    const uint32_t held = *at;
                    uint32_t r = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int s = 4 * w + e, f = s < s0 || s >= s1 ? -1 : from[at0 + s];
                        uint32_t code = f < 0 ? (held >> (8 * e)) & 0xffu : tok[(at0 + s) * kRow + row];
                        const float sc = f < 0 ? was : was_of[at0 + s];
                        if (s < s1 && sc != now) code = rescale4(code, sc / now) & 0xffu;   // (the same for a wave)
                        r |= code << (8 * e);
                    }
                    *at = r;
                }
            }
            if (grown && tid == 0) scales[int64_t(page) * a.c.Hkv + hk] = now;
        }
        __syncthreads();   // LDS is read
    }
}

// ---------------------------------------------------------------- sequences
// Sequence n of the result continues sequence src[n]: it shares that one's full pages; the page
// that is not full goes to the first that continues it and is copied for the others, so that no
// page that a sequence appends to is shared.  refs counts the table entries that hold a page: a
// page is free at 0.  Integers throughout; every choice is by order of sequences, entries and page
// numbers, so that equal calls give equal tables.
constexpr int32_t kAsked = -2;   // an entry that waits for a page

struct Want {
    int32_t s, len, full, held, room;   // pages: full ones, those that hold tokens, those wanted
};
__device__ __forceinline__ Want want_of(const ForkArgs& a, int n) {
    Want w{};
    w.s = ldc(a.src, n);
    if (uint32_t(w.s) >= uint32_t(a.c.B)) {
        w.s = -1;
    } else {
        w.len = int32_t(min(int64_t(max(ldc(a.c.lens, w.s), 0)), int64_t(a.c.width) * kPage));
    }
    const int32_t tokens = max(a.room ? ldc(a.room, n) : 0, w.len);
    w.full = w.len / kPage;
    w.held = (w.len + kPage - 1) / kPage;
    w.room = int32_t(min((int64_t(tokens) + kPage - 1) / kPage, int64_t(a.c.width)));
    return w;
}
__device__ __forceinline__ int block_sum(int x, int* red) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    int r = 0;
    for (int w = 0; w < int(blockDim.x) / 64; ++w) r += red[w];
    return r;
}
// sum over the threads before this one; `all`: over all
template <class N>
__device__ __forceinline__ N block_before(N x, N* red, N& all) {
    N inc = x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const N y = __shfl_up(inc, o);
        if (lane >= o) inc += y;
    }
    __syncthreads();
    if (lane == 63) red[wave] = inc;
    __syncthreads();
    N before = 0;
    all = 0;
    for (int w = 0; w < int(blockDim.x) / 64; ++w) {
        if (w < wave) before += red[w];
        all += red[w];
    }
    return before + inc - x;
}

__global__ void __launch_bounds__(kThreads) fork_refs_kernel(ForkArgs a) {
    const int p = blockIdx.x * kThreads + threadIdx.x;
    if (p < a.c.pages) a.refs_out[p] = a.refs[p];
}

// Workgroups 0 .. B - 1: an old sequence's pages, counted down or up.  The others: a new row, its
// shared pages and how many it asks for.
__global__ void __launch_bounds__(kThreads) fork_rows_kernel(ForkArgs a) {
    __shared__ int red[kThreads / 64];
    const int tid = threadIdx.x;
    if (int(blockIdx.x) < a.c.B) {
        const int s = blockIdx.x;
        int first = INT32_MAX, takers = 0;
        for (int n = tid; n < a.N; n += kThreads)
            if (a.src[n] == s) {
                first = min(first, n);
                ++takers;
            }
        takers = block_sum(takers, red);
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) first = min(first, __shfl_xor(first, o));
        __syncthreads();
        if ((tid & 63) == 0) red[tid >> 6] = first;
        __syncthreads();
        first = min(min(red[0], red[1]), min(red[2], red[3]));
        const Want w = takers ? want_of(a, first) : Want{};
        for (int i = tid; i < a.c.width; i += kThreads) {
            const int p = cache_page(a.c, s, i);
            if (p < 0) continue;
            const int change = !takers ? -1 : i < w.full ? takers - 1 : i < w.room ? 0 : -1;
            if (change) atomicAdd(a.refs_out + p, change);
        }
        return;
    }
    const int n = blockIdx.x - a.c.B;
    const Want w = want_of(a, n);
    int before = 0;
    if (w.s >= 0)
        for (int i = tid; i < n; i += kThreads) before += a.src[i] == w.s;
    const bool leads = w.s >= 0 && block_sum(before, red) == 0;
    int asked = 0;
    for (int i = tid; i < a.c.width; i += kThreads) {
        int32_t e = -1;
        if (i < w.room) {
            const int p = w.s >= 0 ? cache_page(a.c, w.s, i) : -1;
            if (p >= 0 && (leads || i < w.full)) e = p;
            else if (p >= 0 || i >= w.held) e = kAsked;   // (tokens without a page stay without one)
        }
        asked += e == kAsked;
        a.table_out[int64_t(n) * a.c.width + i] = e;
    }
    asked = block_sum(asked, red);
    if (tid == 0) a.need[n] = asked;
}

// One workgroup: what the rows before each ask for, and as many free pages as all do.
constexpr int kListThreads = 1024;
__global__ void __launch_bounds__(kListThreads) fork_list_kernel(ForkArgs a) {
    __shared__ int red[kListThreads / 64];
    __shared__ int64_t red64[kListThreads / 64];
    const int tid = threadIdx.x;
    int64_t total = 0;   // (a row may ask for kMaxWidth pages, so 128 of them for 2^31)
    for (int n0 = 0; n0 < a.N; n0 += kListThreads) {
        const int n = n0 + tid;
        int64_t all;
        const int64_t before = block_before(int64_t(n < a.N ? a.need[n] : 0), red64, all);
        if (n < a.N) a.need[n] = int32_t(min(total + before, int64_t(1) << 30));   // (no pool has as many pages)
        total += all;
    }
    const int most = int(min(total, int64_t(a.cap)));
    int found = 0;
    constexpr int E = 8;
    for (int p0 = 0; p0 < a.c.pages && found < most; p0 += E * kListThreads) {
        int free[E], mine = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int p = p0 + E * tid + e;
            free[e] = p < a.c.pages && a.refs_out[p] == 0;
            mine += free[e];
        }
        int all, at = found + block_before(mine, red, all);
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (free[e]) {
                if (at < most) a.list[1 + at] = p0 + E * tid + e;
                ++at;
            }
        found = min(found + all, most);
    }
    if (tid == 0) a.list[0] = found;
}

// One page to another: thread t of `threads`.
__device__ __forceinline__ void copy_page(const CacheView& c, int of, int to, int t, int threads) {
    const int64_t bytes = int64_t(c.Hkv) * kPage * c.d, part = bytes / 16;
    const u32x4* k0 = reinterpret_cast<const u32x4*>(c.k + of * bytes);
    const u32x4* v0 = reinterpret_cast<const u32x4*>(c.v + of * bytes);
    u32x4* k1 = reinterpret_cast<u32x4*>(c.k + to * bytes);
    u32x4* v1 = reinterpret_cast<u32x4*>(c.v + to * bytes);
    int64_t x = t;
    for (; x + 3 * int64_t(threads) < part; x += 4 * int64_t(threads)) {
        u32x4 k[4], v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            k[j] = k0[x + j * threads];
            v[j] = v0[x + j * threads];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            k1[x + j * threads] = k[j];
            v1[x + j * threads] = v[j];
        }
    }
    for (; x < part; x += threads) {
        k1[x] = k0[x];
        v1[x] = v0[x];
    }
    for (int h = t; h < c.Hkv; h += threads) {
        c.ks[int64_t(to) * c.Hkv + h] = c.ks[int64_t(of) * c.Hkv + h];
        c.vs[int64_t(to) * c.Hkv + h] = c.vs[int64_t(of) * c.Hkv + h];
    }
}

// A row's pages, and a share of the copy of its last one (1, 2, 4 and 8 of them: 44.9, 41.8, 38.0 and
// 39.4 us a call for 1024 rows).
constexpr int kCopyShares = 4;
__global__ void __launch_bounds__(kThreads) fork_fill_kernel(ForkArgs a) {
    __shared__ int red[kThreads / 64];
    const int n = blockIdx.x / kCopyShares, share = blockIdx.x % kCopyShares, tid = threadIdx.x;
    const Want w = want_of(a, n);
    const int found = a.list[0], first = a.need[n];
    int32_t* row = a.table_out + int64_t(n) * a.c.width;
    // The page that is not full is asked for first, by all but the one that keeps it.  Every share
    // goes by the sources' table, as share 0 rewrites the row.
    int copy = -1, of = -1;
    if (w.s >= 0 && w.held > w.full) {
        of = cache_page(a.c, w.s, w.full);
        int before = 0;
        for (int i = tid; i < n; i += kThreads) before += a.src[i] == w.s;
        const bool leads = block_sum(before, red) == 0;
        if (of >= 0 && !leads) copy = first < found ? a.list[1 + first] : -2;
    }
    if (copy >= 0) copy_page(a.c, of, copy, share * kThreads + tid, kCopyShares * kThreads);
    if (share != 0) return;
    int rank = first, asked = 0;
    for (int i0 = 0; i0 < a.c.width; i0 += kThreads) {
        const int i = i0 + tid;
        const bool ask = i < a.c.width && row[i] == kAsked;
        int all;
        const int at = rank + block_before(int(ask), red, all);
        if (ask) {
            const int p = at < found ? a.list[1 + at] : -1;
            row[i] = p;
            if (p >= 0) a.refs_out[p] = 1;
        }
        rank += all;
        asked += all;
    }
    if (tid == 0) {
        a.missing[n] = asked - min(max(found - first, 0), asked);
        a.lens_out[n] = copy == -2 ? w.full * kPage : w.len;
    }
}

// All of it in one launch: every workgroup makes up the same counts in LDS from refs, sources and
// table, finds its own row's pages there by their order, and writes its row, its share of the new
// counts and its copy.  What rows ask for follows from their lengths alone but for a first taker's
// pages behind its tokens, which are counted on the way.  A call is bound by its chains of reads and
// by launches: 9.9 us against 14 for 8 sequences with 16 entries each, 15.9 against 20.1 for 256
// from 64 with 24 and 4000 pages, 17.9 against 22.1 for 64 from 8 with 1024 and 10000 pages, 22.0
// against 22.2 for 256 from 64 with 133 and 9800.  Beyond that the work that every workgroup
// repeats costs more: 24 us against 18 for 128 with 128 and 19000 pages, 62 against 39 for 1024
// from 64.  Many words are read by 1024 threads (the third of these 19.8 us with 512), few by 512
// (the first 11.3 with 1024).
struct SmallFork {   // where each lies, in words; bytes: of all, -1: more than LDS is given
    int32_t first, takers, full, held, room, gaps, given, bytes;
};
constexpr int kSmallBytes = 80 * 1024;   // two workgroups a CU
constexpr int64_t kSmallRows = 256, kSmallReads = 20000;   // rows; words that each workgroup reads
constexpr int64_t kSmallFew = 6000;   // of them, that 512 threads read
__host__ __device__ inline SmallFork small_fork(int64_t pages, int64_t B, int64_t width) {
    SmallFork f{};
    int64_t at = pages;
    for (int32_t* x : {&f.first, &f.takers, &f.full, &f.held, &f.room, &f.gaps}) {
        *x = int32_t(at < kSmallBytes ? at : 0);
        at += B;
    }
    f.given = int32_t(at < kSmallBytes ? at : 0);
    at += width;
    f.bytes = at * 4 <= kSmallBytes - 256 ? int32_t(at * 4) : -1;
    return f;
}

template <int kSmallThreads>
__global__ void __launch_bounds__(kSmallThreads) fork_small_kernel(ForkArgs a, SmallFork f) {
    extern __shared__ int32_t lds[];
    __shared__ int red[kSmallThreads / 64];
    int32_t *count = lds, *first = lds + f.first, *takers = lds + f.takers, *full = lds + f.full, *held = lds + f.held,
            *room = lds + f.room, *gaps = lds + f.gaps, *given = lds + f.given;
    const int tid = threadIdx.x, n = blockIdx.x;
    constexpr int E = 8;   // loads in flight
    for (int p0 = tid; p0 < a.c.pages; p0 += E * kSmallThreads) {
        int c[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int p = p0 + e * kSmallThreads;
            c[e] = p < a.c.pages ? a.refs[p] : 0;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int p = p0 + e * kSmallThreads;
            if (p < a.c.pages) count[p] = c[e];
        }
    }
    for (int s = tid; s < a.c.B; s += kSmallThreads) {
        first[s] = INT32_MAX;
        takers[s] = gaps[s] = 0;
    }
    __syncthreads();
    for (int m = tid; m < a.N; m += kSmallThreads) {
        const int s = a.src[m];
        if (uint32_t(s) < uint32_t(a.c.B)) {
            atomicMin(first + s, m);
            atomicAdd(takers + s, 1);
        }
    }
    __syncthreads();
    for (int s = tid; s < a.c.B; s += kSmallThreads) {   // what the first taker keeps
        const Want w = takers[s] ? want_of(a, first[s]) : Want{};
        full[s] = w.full;
        held[s] = w.held;
        room[s] = w.room;
    }
    __syncthreads();
    const int entries = a.c.B * a.c.width;
    for (int x0 = tid; x0 < entries; x0 += E * kSmallThreads) {
        int p[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int x = x0 + e * kSmallThreads;
            p[e] = x < entries ? a.c.table[x] : -1;
            p[e] = uint32_t(p[e]) < uint32_t(a.c.pages) ? p[e] : -1;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int x = x0 + e * kSmallThreads;
            if (x >= entries) break;
            const int s = x / a.c.width, i = x - s * a.c.width, t = takers[s];
            const int change = !t ? -1 : i < full[s] ? t - 1 : i < room[s] ? 0 : -1;
            if (p[e] >= 0 && change) atomicAdd(count + p[e], change);
            if (p[e] < 0 && i >= held[s] && i < room[s]) atomicAdd(gaps + s, 1);
        }
    }
    __syncthreads();
    // what the rows ask for: this one, those before it, all
    auto asks = [&](int m) {
        const Want w = want_of(a, m);
        if (w.s >= 0 && first[w.s] == m) return gaps[w.s];
        const bool copy = w.s >= 0 && w.held > w.full && cache_page(a.c, w.s, w.full) >= 0;
        return w.room - w.held + copy;
    };
    int before = 0, all = 0;
    for (int m = tid; m < a.N; m += kSmallThreads) {
        const int x = asks(m);
        all += x;
        if (m < n) before += x;
    }
    before = block_sum(before, red);
    all = block_sum(all, red);
    const int asked = asks(n);
    // the free pages in order: this row's, and a share of the new counts
    const int64_t c0 = int64_t(a.c.pages) * n / a.N, c1 = int64_t(a.c.pages) * (n + 1) / a.N;
    int found = 0;
    for (int p0 = 0; p0 < a.c.pages; p0 += E * kSmallThreads) {
        int c[E], mine = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int p = p0 + E * tid + e;
            c[e] = p < a.c.pages ? count[p] : 1;
            mine += c[e] == 0;
        }
        int here, at = found + block_before(mine, red, here);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int p = p0 + E * tid + e;
            if (p >= c0 && p < c1) a.refs_out[p] = c[e] == 0 && at < all ? 1 : c[e];
            if (c[e] == 0) {
                if (at >= before && at < before + asked) given[at - before] = p;
                ++at;
            }
        }
        found += here;
    }
    __syncthreads();
    const int got = min(max(found - before, 0), asked);
    const Want w = want_of(a, n);
    const bool leads = w.s >= 0 && first[w.s] == n;
    int rank = 0;
    for (int i0 = 0; i0 < a.c.width; i0 += kSmallThreads) {
        const int i = i0 + tid;
        const int p = i < w.room && w.s >= 0 ? cache_page(a.c, w.s, i) : -1;
        const bool keeps = p >= 0 && (leads || i < w.full);
        const bool ask = i < w.room && !keeps && (p >= 0 || i >= w.held);
        int here;
        const int at = rank + block_before(int(ask), red, here);
        if (i < a.c.width) a.table_out[int64_t(n) * a.c.width + i] = keeps ? p : ask && at < got ? given[at] : -1;
        rank += here;
    }
    const int of = w.s >= 0 && !leads && w.held > w.full ? cache_page(a.c, w.s, w.full) : -1;
    if (of >= 0 && got > 0) copy_page(a.c, of, given[0], tid, kSmallThreads);   // (what such a row asks for first)
    if (tid == 0) {
        a.missing[n] = asked - got;
        a.lens_out[n] = of >= 0 && got == 0 ? w.full * kPage : w.len;
    }
}

}  // namespace

hipError_t launch_cache_keep(const KeepArgs& a, hipStream_t s) {
    TraceScope _t("cache_keep", s);
    const dim3 g(unsigned(int64_t(a.c.B) * a.c.Hkv * 2)), t(kThreads);
    if (a.c.d == 128) hipLaunchKernelGGL(cache_keep_kernel<128>, g, t, 0, s, a);
    else hipLaunchKernelGGL(cache_keep_kernel<64>, g, t, 0, s, a);
    return hipGetLastError();
}

hipError_t launch_cache_fork(const ForkArgs& a, hipStream_t s) {
    TraceScope _t("cache_fork", s);
    const dim3 t(kThreads), by_pages(unsigned((int64_t(a.c.pages) + kThreads - 1) / kThreads));
    const SmallFork f = small_fork(a.c.pages, a.c.B, a.c.width);
    const int64_t reads = int64_t(a.c.B) * a.c.width + a.c.pages;
    if (f.bytes > 0 && a.N <= kSmallRows && reads <= kSmallReads) {
        ForkArgs b = a;
        if (a.refs == a.refs_out) {   // (the counts are read by all while they are written)
            b.refs_out = a.list;
            hipLaunchKernelGGL(fork_refs_kernel, by_pages, t, 0, s, b);
            b.refs = a.list;
            b.refs_out = a.refs_out;
        }
        if (reads > kSmallFew) hipLaunchKernelGGL(fork_small_kernel<1024>, dim3(unsigned(a.N)), dim3(1024), f.bytes, s, b, f);
        else hipLaunchKernelGGL(fork_small_kernel<512>, dim3(unsigned(a.N)), dim3(512), f.bytes, s, b, f);
        return hipGetLastError();
    }
    if (a.refs != a.refs_out) hipLaunchKernelGGL(fork_refs_kernel, by_pages, t, 0, s, a);
    hipLaunchKernelGGL(fork_rows_kernel, dim3(unsigned(int64_t(a.c.B) + a.N)), t, 0, s, a);
    hipLaunchKernelGGL(fork_list_kernel, dim3(1), dim3(kListThreads), 0, s, a);
    hipLaunchKernelGGL(fork_fill_kernel, dim3(unsigned(int64_t(a.N) * kCopyShares)), t, 0, s, a);
    return hipGetLastError();
}

}  // namespace msparse
