// Backward of the attention with a sliding window and sinks.  With z = scale q k^T
// and P = exp(z - lse) on the visible entries, Delta_i = dO_i . O_i:
//   dV = P^T dO,  dZ = P o (dO V^T - Delta),  dQ = scale dZ K,  dK = scale dZ^T Q,
// dK and dV summed over the query heads of each KV head.
//
// Launches on the caller's stream, all deterministic (no atomics):
//   dq      query-major, as the forward: S^T = K Q^T, dP^T = V dO^T, dQ^T += K^T dZ^T;
//           it leaves lse log2(e) and Delta of its rows for the next pass, in blocks of
//           64 from each sequence's start (rows past its end: P = 0)
//   dkdv    key-major over groups of 64-key blocks: S = Q K^T, dP = dO V^T,
//           dV^T += dO^T P, dK^T += Q^T dZ over the heads of the KV group and the
//           query tiles of the keys' window.  Sink keys are seen by every later
//           row too: a walk over the whole sequence for a single group, so those
//           rows are cut into chunks, a workgroup each, and the chunks' sums go
//           to the workspace (fp32); on small grids the windows' walks are too
//   sums    adds them up, chunks in order.
// Bound like the forward: 32 over 8 heads x 128K, window 4096, 64 sinks, head dim 128:
// dq 12.1 ms, dkdv 16.2 (1090 TFLOP/s of the 7 products that the two issue for 5, S and
// dP twice), sums 0.02.
// All products take bf16 operands with fp32 accumulation: P and dZ are rounded to
// the inputs' type (8 significant bits), each term of the sums independently.
#include "window.h"
#include "trace.h"

namespace msparse {

namespace {

// ------------------------------------------------------------------ dQ
constexpr int kDqThreads = 256, kDqRows = 128;
// Workgroups of 128 rows up to which the split kernel runs (both in us, 128
// rows -> split; heads x tokens, window):
//   d 128   28 (4 x 777, 256): 29 -> 17.5; 128: 41 -> 36 (4 x 4096, 1024), 57 -> 45 (8 x
//           2048, all); 192: 31 -> 42 (12 x 2048, 512); 256: 33 -> 42
//   d 64    28: 18 -> 13; 128: 30 -> 23.5, 40 -> 27; 256: 24 -> 21 (16 x 2048, 512), 41 -> 36
//           (16 x 2048, all); 384: 29.8 -> 29.4; 512: 33 -> 35, 70.5 -> 75 (8 x 8192, 2048)
template <int D>
constexpr int64_t kSplitGrid = D == 128 ? 128 : 256;

template <int D>
struct WinDq {
    static constexpr int KD = D / 16, ND = D / 32;
    u32x4 q[KD], g[KD];
    f32x16 acc[ND];
    float lse2, dlt;
};

// One tile of keys from j0 on against the rows w0 .. w0 + 31, of which i is this lane's.
// The key halves run one after the other, so one half's S^T / dP^T accumulators are
// live and two waves share a SIMD.  A half that no row sees is left out (the sinks'
// second, often one at either end of the window: 65K tokens, window 1024, 4 sinks:
// 1610 -> 1555 us, 850 -> 812 at head dim 64).
template <int D>
__device__ __forceinline__ void dq_tile(const uint16_t* kt, const uint16_t* vt, int w0, int i, int j0, int W, int S,
                                        WinDq<D>& st, int lane, float c2) {
    constexpr int KD = WinDq<D>::KD, ND = WinDq<D>::ND;
    const int h = lane >> 5, l32 = lane & 31;
    u32x4 fk[2], fv[2], ak[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const Sight seen = sight(w0, w0 + 31, j0 + 32 * c, j0 + 32 * c + 31, W, S);
        if (seen == kNone) continue;
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
        if (seen == kPart) {
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

// This lane's share of Delta = sum P dP over one tile.
template <int D>
__device__ __forceinline__ float delta_tile(const uint16_t* kt, const uint16_t* vt, int w0, int i, int j0, int W, int S,
                                            const WinDq<D>& st, int lane, float c2) {
    const int h = lane >> 5, l32 = lane & 31, lim = min(S - 1, i);
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const Sight seen = sight(w0, w0 + 31, j0 + 32 * c, j0 + 32 * c + 31, W, S);
        if (seen == kNone) continue;
        f32x16 sa = f32x16{}, pa = f32x16{};
#pragma unroll
        for (int k = 0; k < WinDq<D>::KD; ++k) {
            sa = mfma32(dma_read16<D, kDualPad>(kt, 32 * c + l32, h + 2 * k), st.q[k], sa);
            pa = mfma32(dma_read16<D, kDualPad>(vt, 32 * c + l32, h + 2 * k), st.g[k], pa);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float p = fast_exp2(__builtin_fmaf(sa[r], c2, -st.lse2)) * pa[r];
            sum += seen == kFull || sees(i, j0 + 32 * c + 8 * (r >> 2) + 4 * h + (r & 3), W, lim) ? p : 0.f;
        }
    }
    return sum;
}

// Rows that see few keys take Delta from the weights and products themselves, in a walk
// of its own, instead of dO . O: O's rounding to bf16 is as large as the other roundings
// of dQ and dK there, and falls with the number of keys that O averages over.  Error of
// dQ and dK by their norm, and time of the backward pass of 64 heads x 1024 rows of 128:
// window 4: 3.0e-3, 62 us with dO . O, 2.35e-3, 70 us with the walk; window 16 and 4
// sinks: 2.5e-3, 90 and 2.35e-3, 99; window 64: 2.45e-3, 63 and 2.35e-3, 70; window 100
// and 4 sinks: 2.4e-3, 90 and 2.35e-3, 102.
constexpr int kFewKeys = 64;
__device__ __forceinline__ bool few_keys(const WindowArgs& a, int i1) {
    return min(int64_t(a.W) + a.S, int64_t(i1) + 1) <= kFewKeys;
}

// Row i's operands, lse log2(e) and dO . O
template <int D>
__device__ __forceinline__ void open_rows(const WindowArgs& a, const Sequence& sq, int hq, int i, int h,
                                          WinDq<D>& st) {
    constexpr int KD = WinDq<D>::KD;
    const int ic = min(i, sq.n - 1);
    const uint16_t* qp = head_rows(a, a.q, sq, hq) + ic * a.q.token;
    const uint16_t* gp = head_rows(a, a.dout, sq, hq) + ic * a.dout.token;
    const uint16_t* op = head_rows(a, a.out, sq, hq) + ic * a.out.token;
    u32x4 o[KD];
#pragma unroll
    for (int s = 0; s < KD; ++s) {
        st.q[s] = *reinterpret_cast<const u32x4*>(qp + 16 * s + 8 * h);
        st.g[s] = *reinterpret_cast<const u32x4*>(gp + 16 * s + 8 * h);
        o[s] = *reinterpret_cast<const u32x4*>(op + 16 * s + 8 * h);
    }
    st.lse2 = a.lse[lse_row(a, sq, hq) + ic] * kLog2e;
    float acc = 0.f;
#pragma unroll
    for (int s = 0; s < KD; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            acc += bf16_lo(st.g[s][e]) * bf16_lo(o[s][e]) + bf16_hi(st.g[s][e]) * bf16_hi(o[s][e]);
    st.dlt = half_swap_sum(acc);
#pragma unroll
    for (int x = 0; x < WinDq<D>::ND; ++x) st.acc[x] = f32x16{};
}
// lse log2(e) and Delta of row i for the key-major pass
template <int D>
__device__ __forceinline__ void leave_rows(const WindowArgs& a, const Sequence& sq, int hq, int i, const WinDq<D>& st) {
    if (i >= padded_rows(sq.n)) return;
    float* rv = a.rows + int64_t(2 * hq) * a.rows_pad + value_row(a, sq) + i;
    rv[0] = i < sq.n ? st.lse2 : INFINITY;   // a row past the end: P = 0
    rv[a.rows_pad] = i < sq.n ? st.dlt : 0.f;
}
template <int D>
__device__ __forceinline__ void store_dq(const WindowArgs& a, const Sequence& sq, int hq, int i, int h,
                                         const WinDq<D>& st) {
    uint16_t* dq = head_rows(a, a.dq, sq, hq) + i * a.dq.token;
#pragma unroll
    for (int x = 0; x < WinDq<D>::ND; ++x)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            u32x2 pk;
            pk.x = pack_bf16x2(st.acc[x][4 * g + 0] * a.scale, st.acc[x][4 * g + 1] * a.scale);
            pk.y = pack_bf16x2(st.acc[x][4 * g + 2] * a.scale, st.acc[x][4 * g + 3] * a.scale);
            *reinterpret_cast<u32x2*>(dq + 32 * x + 8 * g + 4 * h) = pk;
        }
}

template <int D, bool BY_ROWS>
__global__ void __launch_bounds__(kDqThreads)
    __attribute__((amdgpu_waves_per_eu(D == 64 ? 3 : 2, D == 64 ? 3 : 2))) window_dq_kernel(WindowArgs a) {
    constexpr int TE = DmaTile<D, kDualPad>::kElems;
    __shared__ uint16_t k0s[TE], v0s[TE], k1s[TE], v1s[TE];
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, l32 = lane & 31;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    int b, hq, tile;
    if (!window_tile_of<BY_ROWS>(a, blockIdx.x, kDqRows, b, hq, tile)) return;
    const Sequence sq = sequence(a, b);
    const int i0 = tile * kDqRows;
    if (i0 >= sq.n) return;
    const int last = sq.n - 1;
    const int hk = hq / (a.Hq / a.Hkv);
    const uint16_t* kp = head_rows(a, a.k, sq, hk);
    const uint16_t* vp = head_rows(a, a.v, sq, hk);
    const int w0 = i0 + 32 * w, i = w0 + l32;
    WinDq<D> st;
    open_rows(a, sq, hq, i, h, st);
    const float c2 = a.scale * kLog2e;
    const int i1 = min(i0 + kDqRows - 1, last);
    const KeyWalk walk = key_walk(i0, i1, a.W, a.S);
    auto load = [&](uint16_t* kt, uint16_t* vt, int t) {
        const int row0 = 64 * walk.tile(t);
        dma_sequence<D, kDualPad, 4>(kt, kp, a.k.token, row0, last, w, lane);
        dma_sequence<D, kDualPad, 4>(vt, vp, a.v.token, row0, last, w, lane);
    };
    // tile(kt, vt, j0) for every tile of the walk
    auto walk_tiles = [&](auto tile) {
        load(k0s, v0s, 0);
        wait_vmem();
        __syncthreads();
        auto step = [&](int t, const uint16_t* ck, const uint16_t* cv, uint16_t* nk, uint16_t* nv) {
            if (t + 1 < walk.tiles) load(nk, nv, t + 1);
            const int j0 = 64 * walk.tile(t);
            if (w0 <= last) tile(ck, cv, j0);
            __builtin_amdgcn_sched_barrier(0);
            wait_vmem();
            __syncthreads();
        };
        for (int t = 0; t < walk.tiles; t += 2) {
            step(t, k0s, v0s, k1s, v1s);
            if (t + 1 < walk.tiles) step(t + 1, k1s, v1s, k0s, v0s);
        }
    };
    if (few_keys(a, i1)) {
        float sum = 0.f;
        walk_tiles([&](const uint16_t* kt, const uint16_t* vt, int j0) {
            sum += delta_tile<D>(kt, vt, w0, i, j0, a.W, a.S, st, lane, c2);
        });
        st.dlt = half_swap_sum(sum);
    }
    if (h == 0) leave_rows(a, sq, hq, i, st);
    walk_tiles([&](const uint16_t* kt, const uint16_t* vt, int j0) {
        dq_tile<D>(kt, vt, w0, i, j0, a.W, a.S, st, lane, c2);
    });
    if (i <= last) store_dq(a, sq, hq, i, h, st);
}

// Small grids: 64 rows per workgroup, two halves on alternate tiles (as the
// forward's); the second half's sum is added to the first's.
template <int D, bool BY_ROWS>
__global__ void __launch_bounds__(kDqThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
window_dq_split_kernel(WindowArgs a) {
    constexpr int ND = WinDq<D>::ND;
    constexpr int TE = DmaTile<D, kDualPad>::kElems;
    __shared__ __attribute__((aligned(16))) uint16_t kb[2][2][TE], vb[2][2][TE];   // [half][parity]
    __shared__ float share[2][2][64];
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, l32 = lane & 31;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), half = w >> 1, rh = w & 1;
    int b, hq, tile;
    if (!window_tile_of<BY_ROWS>(a, blockIdx.x, 64, b, hq, tile)) return;
    const Sequence sq = sequence(a, b);
    const int i0 = 64 * tile;
    if (i0 >= sq.n) return;
    const int last = sq.n - 1;
    const int hk = hq / (a.Hq / a.Hkv);
    const uint16_t* kp = head_rows(a, a.k, sq, hk);
    const uint16_t* vp = head_rows(a, a.v, sq, hk);
    const int w0 = i0 + 32 * rh, i = w0 + l32;
    const float c2 = a.scale * kLog2e;
    const int i1 = min(i0 + 63, last);
    const KeyWalk walk = key_walk(i0, i1, a.W, a.S);
    const int steps = (walk.tiles + 1) >> 1;
    auto load = [&](int t) {   // tile 2 t + half
        const int row0 = 64 * walk.tile(2 * t + half);
        dma_sequence<D, kDualPad, 2>(kb[half][t & 1], kp, a.k.token, row0, last, rh, lane);
        dma_sequence<D, kDualPad, 2>(vb[half][t & 1], vp, a.v.token, row0, last, rh, lane);
    };
    if (half < walk.tiles) load(0);
    WinDq<D> st;
    open_rows(a, sq, hq, i, h, st);
    auto walk_tiles = [&](auto tile) {   // tile 0 is on its way
        for (int t = 0; t < steps; ++t) {
            wait_vmem();
            __syncthreads();   // tile t has landed, and the buffers of tile t - 1 are read
            if (2 * (t + 1) + half < walk.tiles) load(t + 1);
            if (2 * t + half < walk.tiles) {
                const int j0 = 64 * walk.tile(2 * t + half);
                if (w0 <= last) tile(kb[half][t & 1], vb[half][t & 1], j0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if (few_keys(a, i1)) {
        float sum = 0.f;
        walk_tiles([&](const uint16_t* kt, const uint16_t* vt, int j0) {
            sum += delta_tile<D>(kt, vt, w0, i, j0, a.W, a.S, st, lane, c2);
        });
        share[half][rh][lane] = half_swap_sum(sum);
        __syncthreads();       // every tile has been read
        st.dlt = share[0][rh][lane] + share[1][rh][lane];
        if (half < walk.tiles) load(0);
    }
    if (half == 0 && h == 0) leave_rows(a, sq, hq, i, st);
    walk_tiles([&](const uint16_t* kt, const uint16_t* vt, int j0) {
        dq_tile<D>(kt, vt, w0, i, j0, a.W, a.S, st, lane, c2);
    });
    __syncthreads();   // every tile has been read
    float* x1 = reinterpret_cast<float*>(&kb[0][0][0]) + rh * (ND * 16 * 64);
    static_assert(sizeof(kb) >= 2 * ND * 16 * 64 * 4, "exchange space");
    if (half == 1)
#pragma unroll
        for (int x = 0; x < ND; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) x1[(x * 16 + r) * 64 + lane] = st.acc[x][r];
    __syncthreads();
    if (half == 1 || i > last) return;
#pragma unroll
    for (int x = 0; x < ND; ++x)
#pragma unroll
        for (int r = 0; r < 16; ++r) st.acc[x][r] += x1[(x * 16 + r) * 64 + lane];
    store_dq(a, sq, hq, i, h, st);
}

// ------------------------------------------------------------------ dK / dV
// Four waves per block of 64 keys: wave (key half, row half) holds 32 keys' K in
// registers and takes 32 of each query tile's 64 rows; V of the block lies in LDS.
// The row halves' sums are added at the end, in a fixed order.  At head dim 128 a
// workgroup has two blocks, which share the staged query tiles (two waves per SIMD,
// one workgroup a CU); at 64 one, three workgroups a CU (16K tokens, 12 over 4 heads,
// window 1024: 154 us, with two blocks 172).
template <int D>
constexpr int kKeyBlocks = D == 128 ? 2 : 1;

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

// The query tiles of the keys j0 .. j1: their window's, tiles lo .. hi of every head
// of the group, and those beyond it up to the sequence's end (sink keys).
struct QueryRange {
    int lo, hi, end;
};
__device__ __forceinline__ QueryRange query_range(const Sequence& sq, int j0, int j1, int W) {
    QueryRange r;
    r.end = (sq.n + 63) >> 6;
    r.lo = j0 >> 6;
    const int64_t far = (int64_t(j1) - 1 + W) >> 6;   // the last tile with a row that sees the last key
    r.hi = int(min(far, int64_t(r.end - 1)));
    return r;
}

// Workgroups 0 .. B Hkv sink_groups far_slots - 1 (by rows: Hkv for B Hkv): the chunks of
// the sink keys' rows beyond the window; the rest: groups of kKeyBlocks key blocks,
// near_slots for each.
template <int D, bool BY_ROWS>
__global__ void __launch_bounds__(256 * kKeyBlocks<D>)
    __attribute__((amdgpu_waves_per_eu(D == 128 ? 2 : 3, D == 128 ? 2 : 3))) window_dkdv_kernel(WindowArgs a) {
    constexpr int KD = D / 16, ND = D / 32, KB = kKeyBlocks<D>, KEYS = 64 * KB, NW = 4 * KB;
    constexpr int TE = WinTile<D>::kElems, VE = DmaTile<D, kRowPad>::kElems;
    __shared__ __attribute__((aligned(16))) uint16_t tb[2 * TE];
    __shared__ __attribute__((aligned(16))) uint16_t vsm[KB * VE];
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, l32 = lane & 31;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = w >> 2, kh = (w >> 1) & 1, rh = w & 1;
    const int BK = BY_ROWS ? a.Hkv : a.B * a.Hkv, G = a.Hq / a.Hkv;
    const int groups = BY_ROWS ? int(a.tokens / KEYS) + a.B : (a.seq + KEYS - 1) / KEYS;
    const KeyPlan& p = a.plan;
    const int64_t extra = int64_t(BK) * p.sink_groups * p.far_slots;
    const bool far = int64_t(blockIdx.x) < extra;
    const int64_t u = far ? blockIdx.x : xcd_chunk(blockIdx.x - extra, int64_t(BK) * groups * p.near_slots);
    int slot = int(u % (far ? p.far_slots : p.near_slots));
    const int item = int(u / (far ? p.far_slots : p.near_slots));
    int group, bk;
    if (far) {
        group = item % p.sink_groups;
        bk = item / p.sink_groups;
    } else {
        cell_of(item, BK, groups, bk, group);
    }
    const int hk = bk % a.Hkv;
    int b = bk / a.Hkv;
    if (BY_ROWS && far) {
        b = last_sequence(a, slot, [&](int64_t start, int i) { return far_slot(a, start, i); });
        slot -= int(far_slot(a, cut_start(a, ldc(a.starts, b)), b));
        if (slot < 0) return;
    } else if (BY_ROWS) {
        block_of(a, group, KEYS, b, group);
        if (group < 0) return;
    }
    const Sequence sq = sequence(a, b);
    if (KEYS * group >= sq.n) return;
    const int last = sq.n - 1;
    const QueryRange range = query_range(sq, KEYS * group, KEYS * group + KEYS - 1, a.W);
    // entries [e0, e1) of the walk: head g = e / width, tile base + e % width
    const int base = far ? range.hi + 1 : range.lo;
    const int width = far ? range.end - base : range.hi - range.lo + 1;
    const int chunk = far ? p.far_chunk : p.near_chunk;
    if (BY_ROWS && int64_t(slot) * chunk >= G * width) return;   // (a slot that no sequence has may be far out)
    const int e0 = slot * chunk, e1 = min(e0 + chunk, G * width);
    if (e0 >= e1) return;
    const int key = 32 * kh + l32;
    const int j0 = KEYS * group + 64 * half, j = j0 + key;
    const bool live = j0 <= last && (!far || j0 < a.S);
    const uint16_t* kp = head_rows(a, a.k, sq, hk);
    u32x4 kreg[KD];
#pragma unroll
    for (int s = 0; s < KD; ++s)
        kreg[s] = *reinterpret_cast<const u32x4*>(kp + min(j, last) * a.k.token + 16 * s + 8 * h);
    const uint16_t* vp = head_rows(a, a.v, sq, hk);
#pragma unroll
    for (int x = 0; x < KB; ++x)
        dma_sequence<D, kRowPad, NW>(vsm + x * VE, vp, a.v.token, KEYS * group + 64 * x, last, w, lane);
    const uint16_t* vt = vsm + half * VE;
    f32x16 dv[ND], dk[ND];
#pragma unroll
    for (int x = 0; x < ND; ++x) {
        dv[x] = f32x16{};
        dk[x] = f32x16{};
    }
    const float c2 = a.scale * kLog2e;
    const int64_t v0 = value_row(a, sq);
    // the walk's next entry to load
    int lg = e0 / width, lt = e0 % width;
    auto load = [&](uint16_t* t) {
        const int hq = hk * G + lg, row0 = 64 * (base + lt);
        dma_sequence<D, kDualPad, NW>(t + WinTile<D>::kQ, head_rows(a, a.q, sq, hq), a.q.token, row0, last, w, lane);
        dma_sequence<D, kDualPad, NW>(t + WinTile<D>::kG, head_rows(a, a.dout, sq, hq), a.dout.token, row0, last, w,
                                      lane);
        if (w == 0 && lane < 32) {   // lse2 -> floats 0..63, Delta -> floats 64..127
            const float* rv = a.rows + int64_t(2 * hq) * a.rows_pad + v0 + row0;
            dma16(lane < 16 ? rv + 4 * lane : rv + a.rows_pad + 4 * (lane - 16), lds_addr(t + WinTile<D>::kRw));
        }
        if (++lt == width) {
            lt = 0;
            ++lg;
        }
    };
    int ct = lt;   // the tile of the entry computed
    load(tb);
    wait_vmem();
    __syncthreads();
    auto step = [&](int e, const uint16_t* cur, uint16_t* nxt) {
        const int next = lt;
        if (e + 1 < e1) load(nxt);
        const int i0 = 64 * (base + ct), r0 = i0 + 32 * rh, k0 = j0 + 32 * kh;
        const Sight seen = sight(r0, r0 + 31, k0, k0 + 31, a.W, a.S);
        if (live && seen != kNone) kv_tile<D>(cur, kreg, vt, seen == kPart, i0, j, a.W, a.S, key, rh, c2, lane, dv, dk);
        __builtin_amdgcn_sched_barrier(0);
        ct = next;
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
    static_assert(sizeof(tb) >= 2 * KB * kSlot * 4, "reduction space");
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
    if (rh != 0 || j > last || !live || (far && j >= a.S)) return;
    if (far || (group < p.part_groups && (!BY_ROWS || range.end - 1 > range.hi))) {
        const int64_t lines = BY_ROWS ? int64_t(a.Hkv) * p.far_docs : BK;
        const int64_t line = BY_ROWS ? int64_t(hk) * p.far_docs + far_index(a, sq.row, b) : bk;
        const int64_t at = far ? lines * p.part_groups * p.near_slots + u
                               : (line * p.part_groups + group) * p.near_slots + slot;
        float* o = a.part + at * (2 * KEYS * D) + (64 * half + key) * D + 4 * h;
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
                *reinterpret_cast<f32x4*>(o + 32 * x + 8 * g) = y;
                *reinterpret_cast<f32x4*>(o + KEYS * D + 32 * x + 8 * g) = z;
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

// dK and dV of the keys of part_groups: the sums of their window's chunks, then, for
// sinks, those of the rows beyond, in order.  A thread per 4 columns, which waits for
// its loads kBatch at a time.
constexpr int kSumThreads = 256;
template <int D>
__device__ __forceinline__ void add_slots(f32x4& sum, const float* p, int n) {
    constexpr int64_t kStep = 2 * 64 * kKeyBlocks<D> * D;
    constexpr int kBatch = 16;
    for (int s = 0; s < n; s += kBatch) {
        f32x4 x[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            x[u] = s + u < n ? *reinterpret_cast<const f32x4*>(p + (s + u) * kStep) : f32x4{};
#pragma unroll
        for (int u = 0; u < kBatch; ++u) sum += x[u];
    }
}
template <int D>
__global__ void __launch_bounds__(kSumThreads) window_sums_kernel(WindowArgs a) {
    constexpr int C = D / 4, KEYS = 64 * kKeyBlocks<D>;
    const KeyPlan& p = a.plan;
    const int item = blockIdx.x;   // (line, group); a line: (sequence, KV head), by rows (KV head, far_index)
    const int line = item / p.part_groups, group = item % p.part_groups;
    const int t = blockIdx.y * kSumThreads + threadIdx.x;
    const int which = t / (KEYS * C), key = t / C % KEYS, c = 4 * (t % C);
    const int hk = a.by_rows ? line / p.far_docs : line % a.Hkv, G = a.Hq / a.Hkv;
    int b = line / a.Hkv;
    if (a.by_rows) {   // of the sequences with this index the last, as one with rows beyond its window is
        const int index = line % p.far_docs;
        b = last_sequence(a, index, [&](int64_t start, int i) { return far_index(a, start, i); });
        if (far_index(a, cut_start(a, ldc(a.starts, b)), b) != index) return;
    }
    const Sequence sq = sequence(a, b);
    const int j = KEYS * group + key;
    if (j >= sq.n) return;
    const QueryRange range = query_range(sq, KEYS * group, KEYS * group + KEYS - 1, a.W);
    if (a.by_rows && range.end - 1 <= range.hi) return;
    const int64_t lines = a.by_rows ? int64_t(a.Hkv) * p.far_docs : int64_t(a.B) * a.Hkv;
    const int64_t far0 = a.by_rows ? (int64_t(hk) * p.sink_groups + group) * p.far_slots + far_slot(a, sq.row, b)
                                   : (int64_t(line) * p.sink_groups + group) * p.far_slots;
    const float* part = a.part + which * (KEYS * D) + key * D + c;
    f32x4 sum = f32x4{};
    add_slots<D>(sum, part + int64_t(item) * p.near_slots * (2 * KEYS * D),
                 (G * (range.hi - range.lo + 1) + p.near_chunk - 1) / p.near_chunk);
    if (j < a.S && group < p.sink_groups)
        add_slots<D>(sum, part + (lines * p.part_groups * p.near_slots + far0) * (2 * KEYS * D),
                     (G * (range.end - 1 - range.hi) + p.far_chunk - 1) / p.far_chunk);
    const RowView& v = which == 0 ? a.dk : a.dv;
    const float f = which == 0 ? a.scale : 1.f;
    u32x2 pk;
    pk.x = pack_bf16x2(sum.x * f, sum.y * f);
    pk.y = pack_bf16x2(sum.z * f, sum.w * f);
    *reinterpret_cast<u32x2*>(head_rows(a, v, sq, hk) + j * v.token + c) = pk;
}

}  // namespace

int window_key_resident(int d) { return d == 128 ? 256 : 768; }   // one or three a CU
int window_key_group(int d) { return 64 * (d == 128 ? kKeyBlocks<128> : kKeyBlocks<64>); }

hipError_t launch_window_bwd(const WindowArgs& a, hipStream_t s) {
    const bool wide = a.d == 128;
    {
        TraceScope _t("window_dq", s);
        const int64_t most = wide ? kSplitGrid<128> : kSplitGrid<64>;
        const bool split = a.Hq * row_blocks(a.B, a.seq, a.tokens, kDqRows) <= most;
        const dim3 g(unsigned(a.Hq * grid_blocks(a.by_rows, a.B, a.seq, a.tokens, split ? 64 : kDqRows))), t(kDqThreads);
        window_variant(a, [&](auto dim, auto by_rows) {
            constexpr int D = decltype(dim)::value;
            constexpr bool R = decltype(by_rows)::value;
            if (split) hipLaunchKernelGGL((window_dq_split_kernel<D, R>), g, t, 0, s, a);
            else hipLaunchKernelGGL((window_dq_kernel<D, R>), g, t, 0, s, a);
        });
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t bk = (a.by_rows ? 1 : int64_t(a.B)) * a.Hkv;
    {
        TraceScope _t("window_dkdv", s);
        const int keys = window_key_group(a.d);
        const int64_t groups = a.Hkv * grid_blocks(a.by_rows, a.B, a.seq, a.tokens, keys);
        const dim3 g(unsigned(bk * a.plan.sink_groups * a.plan.far_slots + groups * a.plan.near_slots));
        window_variant(a, [&](auto dim, auto by_rows) {
            constexpr int D = decltype(dim)::value;
            hipLaunchKernelGGL((window_dkdv_kernel<D, decltype(by_rows)::value>), g, dim3(256 * kKeyBlocks<D>), 0, s, a);
        });
    }
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (a.plan.part_groups > 0) {
        TraceScope _t("window_sums", s);
        // 8 or 32 workgroups per group, along y: along x too, a launch of 2^19 groups would have 2^32 threads
        const int64_t lines = a.by_rows ? int64_t(a.Hkv) * a.plan.far_docs : bk;
        const dim3 g(unsigned(lines * a.plan.part_groups), unsigned(2 * window_key_group(a.d) * a.d / 4 / kSumThreads));
        const dim3 t(kSumThreads);
        if (wide) hipLaunchKernelGGL(window_sums_kernel<128>, g, t, 0, s, a);
        else hipLaunchKernelGGL(window_sums_kernel<64>, g, t, 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace msparse
