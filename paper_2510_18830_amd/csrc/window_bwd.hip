// Backward of the attention with a sliding window and sinks.  With z = scale q k^T
// and P = exp(z - lse) on the visible entries, Delta_i = dO_i . O_i:
//   dV = P^T dO,  dZ = P o (dO V^T - Delta),  dQ = scale dZ K,  dK = scale dZ^T Q,
// dK and dV summed over the query heads of each KV head.
//
// Launches on the caller's stream, all deterministic (no atomics):
//   rows    lse log2(e) and Delta of every row, in blocks of 64 from each
//           sequence's start (rows past its end: P = 0)
//   dq      query-major, as the forward: S^T = K Q^T, dP^T = V dO^T, dQ^T += K^T dZ^T
//   dkdv    key-major over pairs of 64-key blocks: S = Q K^T, dP = dO V^T,
//           dV^T += dO^T P, dK^T += Q^T dZ over the heads of the KV group and the
//           query tiles of the pair's window.  Sink keys are seen by every later
//           row too: a walk over the whole sequence for a single pair, so those
//           rows are cut into chunks, a workgroup each, and the chunks' sums go
//           to the workspace (fp32)
//   sinks   adds them up, chunks in order.
// All products take bf16 operands with fp32 accumulation: P and dZ are rounded to
// the inputs' type (8 significant bits), each term of the sums independently.
#include "window.h"
#include "trace.h"

namespace msparse {

namespace {

// ------------------------------------------------------------------ row values
constexpr int kRowThreads = 256;

// 16 lanes per row; a workgroup takes 64 rows.
template <int D>
__global__ void __launch_bounds__(kRowThreads) window_rows_kernel(WindowArgs a) {
    constexpr int PER = D / 16;
    const int blocks = (a.seq + 63) >> 6, bh = blockIdx.x / blocks, i0 = 64 * (blockIdx.x % blocks);
    const int h = bh % a.Hq;
    const Sequence sq = sequence(a, bh / a.Hq);
    if (i0 >= sq.n) return;
    const int64_t v0 = value_row(a, sq);
    float* lse2 = a.rows + int64_t(2 * h) * a.rows_pad + v0;
    float* delta = lse2 + a.rows_pad;
    const uint16_t* gp = head_rows(a, a.dout, sq, h);
    const uint16_t* op = head_rows(a, a.out, sq, h);
    const float* lse = a.lse + lse_row(a, sq, h);
    const int sub = threadIdx.x & 15;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int i = i0 + 16 * u + (threadIdx.x >> 4), r = min(i, sq.n - 1);
        const uint32_t* g = reinterpret_cast<const uint32_t*>(gp + r * a.dout.token + sub * PER);
        const uint32_t* o = reinterpret_cast<const uint32_t*>(op + r * a.out.token + sub * PER);
        float acc = 0.f;
#pragma unroll
        for (int j = 0; j < PER / 2; ++j) acc += bf16_lo(g[j]) * bf16_lo(o[j]) + bf16_hi(g[j]) * bf16_hi(o[j]);
#pragma unroll
        for (int off = 8; off >= 1; off >>= 1) acc += __shfl_xor(acc, off);
        if (sub == 0) {
            lse2[i] = i < sq.n ? lse[i] * kLog2e : INFINITY;
            delta[i] = i < sq.n ? acc : 0.f;
        }
    }
}

// ------------------------------------------------------------------ dQ
constexpr int kDqThreads = 256, kDqRows = 128;

template <int D>
struct WinDq {
    static constexpr int KD = D / 16, ND = D / 32;
    u32x4 q[KD], g[KD];
    f32x16 acc[ND];
    float lse2, dlt;
};

// One tile; the key halves run one after the other, so one half's S^T / dP^T
// accumulators are live and two waves share a SIMD.
template <int D>
__device__ __forceinline__ void dq_tile(const uint16_t* kt, const uint16_t* vt, bool masked, int i, int j0, int W,
                                        int S, WinDq<D>& st, int lane, float c2) {
    constexpr int KD = WinDq<D>::KD, ND = WinDq<D>::ND;
    const int h = lane >> 5, l32 = lane & 31;
    u32x4 fk[2], fv[2], ak[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        f32x16 sa = f32x16{}, pa = f32x16{};
        auto read_sd = [&](int set, int s) {
            fk[set] = dma_read16<D, kDualPad>(kt, 32 * c + l32, h + 2 * s);
            fv[set] = dma_read16<D, kDualPad>(vt, 32 * c + l32, h + 2 * s);
        };
        auto read_tr = [&](int b) {
#pragma unroll
            for (int j = 0; j < 2; ++j) ak[j] = dma_read_tr<D, kDualPad>(kt, 16 * (2 * c + j), 32 * b, lane);
        };
        read_sd(0, 0);
#pragma unroll
        for (int k = 0; k < KD; ++k) {
            const int set = k & 1;
            if (k + 1 < KD) read_sd(set ^ 1, k + 1);
            else read_tr(0);
            __builtin_amdgcn_sched_barrier(0);
            sa = mfma32(fk[set], st.q[k], sa);
            pa = mfma32(fv[set], st.g[k], pa);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float p = fast_exp2(__builtin_fmaf(sa[r], c2, -st.lse2));
            sa[r] = p * (pa[r] - st.dlt);
        }
        if (masked) {
            keep_branch();
            const int lim = min(S - 1, i);
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (!sees(i, j0 + 32 * c + 8 * (r >> 2) + 4 * h + (r & 3), W, lim)) sa[r] = 0.f;
        }
        u32x4 zb[2];
        zb[0] = pack8_bf16<0>(sa);
        zb[1] = pack8_bf16<8>(sa);
#pragma unroll
        for (int b = 0; b < ND; ++b) {
            if (b > 0) read_tr(b);
#pragma unroll
            for (int j = 0; j < 2; ++j) st.acc[b] = mfma32(ak[j], zb[j], st.acc[b]);
        }
    }
}

template <int D>
__global__ void __launch_bounds__(kDqThreads)
    __attribute__((amdgpu_waves_per_eu(D == 64 ? 3 : 2, D == 64 ? 3 : 2))) window_dq_kernel(WindowArgs a) {
    constexpr int KD = WinDq<D>::KD, ND = WinDq<D>::ND;
    constexpr int TE = DmaTile<D, kDualPad>::kElems;
    __shared__ uint16_t k0s[TE], v0s[TE], k1s[TE], v1s[TE];
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, l32 = lane & 31;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    int b, hq, tile;
    window_tile_of(a, blockIdx.x, (a.seq + kDqRows - 1) / kDqRows, b, hq, tile);
    const Sequence sq = sequence(a, b);
    const int i0 = tile * kDqRows;
    if (i0 >= sq.n) return;
    const int last = sq.n - 1;
    const int hk = hq / (a.Hq / a.Hkv);
    const uint16_t* kp = head_rows(a, a.k, sq, hk);
    const uint16_t* vp = head_rows(a, a.v, sq, hk);
    const int w0 = i0 + 32 * w, i = w0 + l32, ic = min(i, last);
    WinDq<D> st;
    {
        const uint16_t* qp = head_rows(a, a.q, sq, hq) + ic * a.q.token;
        const uint16_t* gp = head_rows(a, a.dout, sq, hq) + ic * a.dout.token;
#pragma unroll
        for (int s = 0; s < KD; ++s) {
            st.q[s] = *reinterpret_cast<const u32x4*>(qp + 16 * s + 8 * h);
            st.g[s] = *reinterpret_cast<const u32x4*>(gp + 16 * s + 8 * h);
        }
        const float* rv = a.rows + int64_t(2 * hq) * a.rows_pad + value_row(a, sq) + ic;
        st.lse2 = rv[0];
        st.dlt = rv[a.rows_pad];
    }
#pragma unroll
    for (int x = 0; x < ND; ++x) st.acc[x] = f32x16{};
    const float c2 = a.scale * kLog2e;
    const KeyWalk walk = key_walk(i0, min(i0 + kDqRows - 1, last), a.W, a.S);
    auto load = [&](uint16_t* kt, uint16_t* vt, int t) {
        const int row0 = 64 * walk.tile(t);
        dma_sequence<D, kDualPad, 4>(kt, kp, a.k.token, row0, last, w, lane);
        dma_sequence<D, kDualPad, 4>(vt, vp, a.v.token, row0, last, w, lane);
    };
    load(k0s, v0s, 0);
    wait_vmem();
    __syncthreads();
    auto step = [&](int t, const uint16_t* ck, const uint16_t* cv, uint16_t* nk, uint16_t* nv) {
        if (t + 1 < walk.tiles) load(nk, nv, t + 1);
        const int j0 = 64 * walk.tile(t);
        const Sight seen = sight(w0, w0 + 31, j0, j0 + 63, a.W, a.S);
        if (seen != kNone && w0 <= last) dq_tile<D>(ck, cv, seen == kPart, i, j0, a.W, a.S, st, lane, c2);
        __builtin_amdgcn_sched_barrier(0);
        wait_vmem();
        __syncthreads();
    };
    for (int t = 0; t < walk.tiles; t += 2) {
        step(t, k0s, v0s, k1s, v1s);
        if (t + 1 < walk.tiles) step(t + 1, k1s, v1s, k0s, v0s);
    }
    if (i > last) return;
    uint16_t* dq = head_rows(a, a.dq, sq, hq) + i * a.dq.token;
#pragma unroll
    for (int x = 0; x < ND; ++x)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            u32x2 pk;
            pk.x = pack_bf16x2(st.acc[x][4 * g + 0] * a.scale, st.acc[x][4 * g + 1] * a.scale);
            pk.y = pack_bf16x2(st.acc[x][4 * g + 2] * a.scale, st.acc[x][4 * g + 3] * a.scale);
            *reinterpret_cast<u32x2*>(dq + 32 * x + 8 * g + 4 * h) = pk;
        }
}

// ------------------------------------------------------------------ dK / dV
// Eight waves per pair of key blocks: wave (block, key half, row half) holds 32
// keys' K in registers and takes 32 of each query tile's 64 rows; V of the pair
// lies in LDS.  The row halves' sums are added at the end, in a fixed order.
constexpr int kKvThreads = 512;

template <int D>
struct WinTile {   // a staged query tile: Q rows, dO rows, 64 lse2, 64 Delta
    static constexpr int kPart = DmaTile<D, kDualPad>::kElems;
    static constexpr int kQ = 0, kG = kPart, kRw = 2 * kPart, kElems = 2 * kPart + 256;
};

// Rows 32 rh .. 32 rh + 31 of the query tile t (first row i0) against this lane's
// key j (row `key` of vt).
template <int D>
__device__ __forceinline__ void kv_tile(const uint16_t* t, const u32x4* kreg, const uint16_t* vt, bool masked, int i0,
                                        int j, int W, int S, int key, int rh, float c2, int lane, f32x16* dv,
                                        f32x16* dk) {
    using T = WinTile<D>;
    constexpr int KD = D / 16, ND = D / 32;
    const int h = lane >> 5, l32 = lane & 31;
    f32x16 sacc = f32x16{}, pacc = f32x16{};
    {
        u32x4 fq[2], fg[2], fv[2];
        auto rd = [&](int set, int s) {
            fq[set] = dma_read16<D, kDualPad>(t + T::kQ, 32 * rh + l32, h + 2 * s);
            fg[set] = dma_read16<D, kDualPad>(t + T::kG, 32 * rh + l32, h + 2 * s);
            fv[set] = dma_read16<D, kRowPad>(vt, key, h + 2 * s);
        };
        rd(0, 0);
#pragma unroll
        for (int s = 0; s < KD; ++s) {
            const int set = s & 1;
            if (s + 1 < KD) rd(set ^ 1, s + 1);
            __builtin_amdgcn_sched_barrier(0);
            sacc = mfma32(fq[set], kreg[s], sacc);
            pacc = mfma32(fg[set], fv[set], pacc);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // P and dZ as bf16 B operands
    u32x4 pb[2], zb[2];
    const float* lse2 = reinterpret_cast<const float*>(t + T::kRw);
    const float* dlt = lse2 + 64;
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
        const int row0 = 32 * rh + 8 * q4 + 4 * h;
        const f32x4 l4 = *reinterpret_cast<const f32x4*>(lse2 + row0);
        const f32x4 d4 = *reinterpret_cast<const f32x4*>(dlt + row0);
        float pv[4], zv[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = 4 * q4 + e;
            pv[e] = fast_exp2(__builtin_fmaf(sacc[r], c2, -l4[e]));
            zv[e] = pv[e] * (pacc[r] - d4[e]);
        }
        const int x = q4 >> 1, w0 = 2 * (q4 & 1);
        pb[x][w0] = pack_bf16x2(pv[0], pv[1]);
        pb[x][w0 + 1] = pack_bf16x2(pv[2], pv[3]);
        zb[x][w0] = pack_bf16x2(zv[0], zv[1]);
        zb[x][w0 + 1] = pack_bf16x2(zv[2], zv[3]);
    }
    if (masked) {   // clear the halves of unseen entries
        keep_branch();
        const int first = i0 + 32 * rh + 4 * h;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int i = first + 8 * (r >> 2) + (r & 3);
            if (!sees(i, j, W, min(S - 1, i))) {
                const uint32_t keep = (r & 1) ? 0x0000FFFFu : 0xFFFF0000u;
                pb[r >> 3][(r & 7) >> 1] &= keep;
                zb[r >> 3][(r & 7) >> 1] &= keep;
            }
        }
    }
    u32x4 av[2][2], ak[2][2];   // [set][k-step]: dO^T, Q^T of one 32-wide d block
    auto rt = [&](int set, int b) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            av[set][x] = dma_read_tr<D, kDualPad>(t + T::kG, 32 * rh + 16 * x, 32 * b, lane);
            ak[set][x] = dma_read_tr<D, kDualPad>(t + T::kQ, 32 * rh + 16 * x, 32 * b, lane);
        }
    };
    rt(0, 0);
#pragma unroll
    for (int b = 0; b < ND; ++b) {
        const int set = b & 1;
        if (b + 1 < ND) rt(set ^ 1, b + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            dv[b] = mfma32(av[set][x], pb[x], dv[b]);
            dk[b] = mfma32(ak[set][x], zb[x], dk[b]);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

// The query tiles of a key pair: its window's, tiles lo .. hi of every head of
// the group, and those beyond it up to the sequence's end (sink pairs).
struct QueryRange {
    int lo, hi, end;
};
__device__ __forceinline__ QueryRange query_range(const Sequence& sq, int pair, int W) {
    QueryRange r;
    r.end = (sq.n + 63) >> 6;
    r.lo = 2 * pair;
    const int64_t far = (int64_t(128) * pair + 126 + W) >> 6;   // the last tile with a row that sees the last key
    r.hi = int(min(far, int64_t(r.end - 1)));
    return r;
}

// Workgroups 0 .. B Hkv sink_pairs (slots - 1) - 1: the chunks of the sink keys'
// rows beyond the window (the longest walks first); the rest: pairs of key blocks.
template <int D>
__global__ void __launch_bounds__(kKvThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
window_dkdv_kernel(WindowArgs a) {
    constexpr int KD = D / 16, ND = D / 32;
    constexpr int TE = WinTile<D>::kElems, VE = DmaTile<D, kRowPad>::kElems;
    __shared__ __attribute__((aligned(16))) uint16_t tb[2 * TE];
    __shared__ __attribute__((aligned(16))) uint16_t vsm[2 * VE];
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, l32 = lane & 31;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = w >> 2, kh = (w >> 1) & 1, rh = w & 1;
    const int BK = a.B * a.Hkv, G = a.Hq / a.Hkv;
    const int pairs = (a.seq + 127) >> 7;
    const int64_t extra = int64_t(BK) * a.sink_pairs * (a.slots - 1);
    int bk, pair, slot;      // slot: 0 the window, 1 .. a chunk beyond
    if (int64_t(blockIdx.x) < extra) {
        bk = int(blockIdx.x / (a.sink_pairs * (a.slots - 1)));
        const int r = int(blockIdx.x % (a.sink_pairs * (a.slots - 1)));
        pair = r / (a.slots - 1);
        slot = 1 + r % (a.slots - 1);
    } else {
        const int64_t u = xcd_chunk(blockIdx.x - extra, int64_t(BK) * pairs);
        bk = int(u / pairs);
        pair = int(u % pairs);
        slot = 0;
    }
    const int b = bk / a.Hkv, hk = bk % a.Hkv;
    const Sequence sq = sequence(a, b);
    if (128 * pair >= sq.n) return;
    const int last = sq.n - 1;
    const QueryRange range = query_range(sq, pair, a.W);
    // entries [e0, e1) of the walk: head g = e / width, tile base + e % width
    int base = range.lo, width = range.hi - range.lo + 1, e0 = 0, e1 = G * width;
    if (slot > 0) {
        base = range.hi + 1;
        width = range.end - base;
        e0 = (slot - 1) * a.chunk;
        e1 = min(e0 + a.chunk, G * width);
        if (e0 >= e1) return;
    }
    const int key = 32 * kh + l32;
    const int j0 = 128 * pair + 64 * half, j = j0 + key;
    const bool live = j0 <= last && (slot == 0 || j0 < a.S);
    const uint16_t* kp = head_rows(a, a.k, sq, hk);
    u32x4 kreg[KD];
#pragma unroll
    for (int s = 0; s < KD; ++s)
        kreg[s] = *reinterpret_cast<const u32x4*>(kp + min(j, last) * a.k.token + 16 * s + 8 * h);
    const uint16_t* vp = head_rows(a, a.v, sq, hk);
    dma_sequence<D, kRowPad, 8>(vsm, vp, a.v.token, 128 * pair, last, w, lane);
    dma_sequence<D, kRowPad, 8>(vsm + VE, vp, a.v.token, 128 * pair + 64, last, w, lane);
    const uint16_t* vt = vsm + half * VE;
    f32x16 dv[ND], dk[ND];
#pragma unroll
    for (int x = 0; x < ND; ++x) {
        dv[x] = f32x16{};
        dk[x] = f32x16{};
    }
    const float c2 = a.scale * kLog2e;
    const int64_t v0 = value_row(a, sq);
    auto load = [&](uint16_t* t, int e) {
        const int hq = hk * G + e / width, row0 = 64 * (base + e % width);
        dma_sequence<D, kDualPad, 8>(t + WinTile<D>::kQ, head_rows(a, a.q, sq, hq), a.q.token, row0, last, w, lane);
        dma_sequence<D, kDualPad, 8>(t + WinTile<D>::kG, head_rows(a, a.dout, sq, hq), a.dout.token, row0, last, w,
                                     lane);
        if (w == 0 && lane < 32) {   // lse2 -> floats 0..63, Delta -> floats 64..127
            const float* rv = a.rows + int64_t(2 * hq) * a.rows_pad + v0 + row0;
            dma16(lane < 16 ? rv + 4 * lane : rv + a.rows_pad + 4 * (lane - 16), lds_addr(t + WinTile<D>::kRw));
        }
    };
    load(tb, e0);
    wait_vmem();
    __syncthreads();
    auto step = [&](int e, const uint16_t* ct, uint16_t* nt) {
        if (e + 1 < e1) load(nt, e + 1);
        const int i0 = 64 * (base + e % width), r0 = i0 + 32 * rh, k0 = j0 + 32 * kh;
        const Sight seen = sight(r0, r0 + 31, k0, k0 + 31, a.W, a.S);
        if (live && seen != kNone) kv_tile<D>(ct, kreg, vt, seen == kPart, i0, j, a.W, a.S, key, rh, c2, lane, dv, dk);
        __builtin_amdgcn_sched_barrier(0);
        wait_vmem();
        __syncthreads();
    };
    for (int e = e0; e < e1; e += 2) {
        step(e, tb, tb + TE);
        if (e + 1 < e1) step(e + 1, tb + TE, tb);
    }
    // add the row halves (through LDS, every tile has been read)
    float* red = reinterpret_cast<float*>(tb);
    constexpr int kSlot = ND * 16 * 64;
    static_assert(sizeof(tb) >= 4 * kSlot * 4, "reduction space");
    float* mine = red + (2 * half + kh) * kSlot;
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
        f32x16* acc = pass == 0 ? dv : dk;
        if (rh == 1)
#pragma unroll
            for (int x = 0; x < ND; ++x)
#pragma unroll
                for (int r = 0; r < 16; ++r) mine[(x * 16 + r) * 64 + lane] = acc[x][r];
        __syncthreads();
        if (rh == 0)
#pragma unroll
            for (int x = 0; x < ND; ++x)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[x][r] += mine[(x * 16 + r) * 64 + lane];
        __syncthreads();
    }
    if (rh != 0 || j > last || !live) return;
    if (pair < a.sink_pairs) {
        float* p = a.part + ((int64_t(bk) * a.sink_pairs + pair) * a.slots + slot) * (2 * 128 * D) +
                   (64 * half + key) * D + 4 * h;
#pragma unroll
        for (int x = 0; x < ND; ++x)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4 y, z;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    y[e] = dk[x][4 * g + e];
                    z[e] = dv[x][4 * g + e];
                }
                *reinterpret_cast<f32x4*>(p + 32 * x + 8 * g) = y;
                *reinterpret_cast<f32x4*>(p + 128 * D + 32 * x + 8 * g) = z;
            }
        return;
    }
    uint16_t* dkp = head_rows(a, a.dk, sq, hk) + j * a.dk.token + 4 * h;
    uint16_t* dvp = head_rows(a, a.dv, sq, hk) + j * a.dv.token + 4 * h;
#pragma unroll
    for (int x = 0; x < ND; ++x)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            u32x2 y, z;
            y.x = pack_bf16x2(dk[x][4 * g + 0] * a.scale, dk[x][4 * g + 1] * a.scale);
            y.y = pack_bf16x2(dk[x][4 * g + 2] * a.scale, dk[x][4 * g + 3] * a.scale);
            z.x = pack_bf16x2(dv[x][4 * g + 0], dv[x][4 * g + 1]);
            z.y = pack_bf16x2(dv[x][4 * g + 2], dv[x][4 * g + 3]);
            *reinterpret_cast<u32x2*>(dkp + 32 * x + 8 * g) = y;
            *reinterpret_cast<u32x2*>(dvp + 32 * x + 8 * g) = z;
        }
}

// dK and dV of the sink pairs' keys: the window's sum, then the chunks in order.
// Keys of such a pair that are no sinks have no chunks.  One thread per 4 columns.
constexpr int kSumThreads = 256;
template <int D>
__global__ void __launch_bounds__(kSumThreads) window_sinks_kernel(WindowArgs a) {
    constexpr int C = D / 4;
    const int per = 2 * 128 * C / kSumThreads;   // workgroups per pair
    const int item = blockIdx.x / per;
    const int bk = item / a.sink_pairs, pair = item % a.sink_pairs;
    const int t = (blockIdx.x % per) * kSumThreads + threadIdx.x;
    const int which = t / (128 * C), key = t / C % 128, c = 4 * (t % C);
    const int b = bk / a.Hkv, hk = bk % a.Hkv;
    const Sequence sq = sequence(a, b);
    const int j = 128 * pair + key;
    if (j >= sq.n) return;
    const QueryRange range = query_range(sq, pair, a.W);
    const int beyond = (a.Hq / a.Hkv) * (range.end - 1 - range.hi);
    // a block of 64 keys without a sink has no chunks
    const int used = (j & ~63) < a.S ? 1 + (beyond + a.chunk - 1) / a.chunk : 1;
    const float* p = a.part + int64_t(item) * a.slots * (2 * 128 * D) + which * (128 * D) + key * D + c;
    f32x4 sum = *reinterpret_cast<const f32x4*>(p);
    int s = 1;
    for (; s + 8 <= used; s += 8) {
        f32x4 x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = *reinterpret_cast<const f32x4*>(p + int64_t(s + u) * (2 * 128 * D));
#pragma unroll
        for (int u = 0; u < 8; ++u) sum += x[u];
    }
    for (; s < used; ++s) sum += *reinterpret_cast<const f32x4*>(p + int64_t(s) * (2 * 128 * D));
    const RowView& v = which == 0 ? a.dk : a.dv;
    const float f = which == 0 ? a.scale : 1.f;
    u32x2 pk;
    pk.x = pack_bf16x2(sum.x * f, sum.y * f);
    pk.y = pack_bf16x2(sum.z * f, sum.w * f);
    *reinterpret_cast<u32x2*>(head_rows(a, v, sq, hk) + j * v.token + c) = pk;
}

}  // namespace

hipError_t launch_window_bwd(const WindowArgs& a, hipStream_t s) {
    const bool wide = a.d == 128;
    {
        TraceScope _t("window_rows", s);
        const dim3 g(unsigned(int64_t(a.B) * a.Hq * ((a.seq + 63) / 64))), t(kRowThreads);
        if (wide) hipLaunchKernelGGL(window_rows_kernel<128>, g, t, 0, s, a);
        else hipLaunchKernelGGL(window_rows_kernel<64>, g, t, 0, s, a);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    {
        TraceScope _t("window_dq", s);
        const dim3 g(unsigned(int64_t(a.B) * a.Hq * ((a.seq + kDqRows - 1) / kDqRows))), t(kDqThreads);
        if (wide) hipLaunchKernelGGL(window_dq_kernel<128>, g, t, 0, s, a);
        else hipLaunchKernelGGL(window_dq_kernel<64>, g, t, 0, s, a);
    }
    if ((e = hipGetLastError()) != hipSuccess) return e;
    {
        TraceScope _t("window_dkdv", s);
        const int64_t bk = int64_t(a.B) * a.Hkv;
        const int64_t extra = bk * a.sink_pairs * std::max(0, a.slots - 1);
        const dim3 g(unsigned(extra + bk * ((a.seq + 127) / 128))), t(kKvThreads);
        if (wide) hipLaunchKernelGGL(window_dkdv_kernel<128>, g, t, 0, s, a);
        else hipLaunchKernelGGL(window_dkdv_kernel<64>, g, t, 0, s, a);
    }
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (a.sink_pairs > 0) {
        TraceScope _t("window_sinks", s);
        const dim3 g(unsigned(int64_t(a.B) * a.Hkv * a.sink_pairs * (2 * 128 * a.d / 4 / kSumThreads))), t(kSumThreads);
        if (wide) hipLaunchKernelGGL(window_sinks_kernel<128>, g, t, 0, s, a);
        else hipLaunchKernelGGL(window_sinks_kernel<64>, g, t, 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace msparse
