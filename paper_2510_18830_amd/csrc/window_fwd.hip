// Forward of the attention with a sliding window and sinks.  Bound by the matrix
// cores and the softmax terms beside them, at long lengths by the power they take:
// 16 over 2 heads x 32K, window 4096, 64 sinks, head dim 128: 1.09 ms, 960 TFLOP/s on
// the visible pairs.
//
// One workgroup of four wavefronts per (sequence, query head, 128 rows), 32 rows
// a wave.  Key tiles of 64 are staged by direct global->LDS loads, the next one
// in flight while the current one is computed.  Per tile and wave:
//   S^T = K Q^T    (A = K rows from LDS, B = the wave's Q rows in registers)
//   online softmax (a lane owns a query row, lane l ^ 32 the other half of its keys)
//   O^T += V^T P^T (A = V^T read transposed from LDS, B = P from the S^T registers)
// Both products take bf16 operands: P is rounded to V's type (8 significant bits,
// the rounding that the output itself gets), and the sum that normalises O is
// that of the rounded weights, so a row with nearly all its weight on one key
// keeps that key's value exactly; lse is made from the unrounded sum.
#include "window.h"
#include "trace.h"

namespace msparse {

namespace {

constexpr float kSlack = 8.f;        // log2 units
constexpr int kFwdRows = 128;        // query rows per workgroup
constexpr int kFwdThreads = 256;
// Workgroups of 128 rows up to which the split kernel runs instead (both in us,
// 128 rows -> split; heads x tokens, window):
//   d 128   28 (4 x 777, 256): 16.7 -> 11.8; 128: 33.2 -> 25.9 (4 x 4096, 1024), 46.6 ->
//           35.9 (8 x 2048, all); 192: 23.9 -> 31.8 (12 x 2048, 512); 256: 25.2 -> 32.8
//   d 64    28: 12.7 -> 8.0; 128: 24.3 -> 15.5, 34.8 -> 22.2; 256: 18.2 -> 14.3 (16 x
//           2048, 512); 384: 24.0 -> 22.8; 512: 24.1 -> 25.9, 57.8 -> 62.6 (8 x 8192, 2048)
template <int D>
constexpr int64_t kSplitGrid = D == 128 ? 128 : 384;

template <int D>
struct WinRows {
    static constexpr int KD = D / 16;   // k-steps over head_dim
    static constexpr int ND = D / 32;   // 32-wide output column blocks
    u32x4 q[KD];
    f32x16 o[ND];
    float m = -INFINITY;        // running maximum (log2 units)
    float l = 0.f, lr = 0.f;    // sums of the weights and of the rounded weights
};

// Sum of the bf16 weights in four packed operands, both halves of the row.
__device__ __forceinline__ float row_sum_bf16(const u32x4* pb) {
    const bf16x2 one = {(__bf16)1.f, (__bf16)1.f};
    float a = 0.f, b = 0.f;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const uint32_t w0 = pb[g].x, w1 = pb[g].y, w2 = pb[g].z, w3 = pb[g].w;
        a = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w0), one, a, false);
        b = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w1), one, b, false);
        a = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w2), one, a, false);
        b = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w3), one, b, false);
    }
    return half_swap_sum(a + b);
}

// One tile of the keys j0 .. j0 + 63; i = this lane's row.  c2 = scale log2(e).
template <int D>
__device__ __forceinline__ void win_tile(const uint16_t* kt, const uint16_t* vt, bool masked, int i, int j0, int W,
                                         int S, WinRows<D>& st, int lane, float c2) {
    constexpr int KD = WinRows<D>::KD, ND = WinRows<D>::ND;
    const int h = lane >> 5, l32 = lane & 31;
    // operands in groups of two k-steps, read one group ahead of their MFMAs
    f32x16 sacc[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) sacc[c] = f32x16{};
    u32x4 fk[2][2][2];   // [set][k-step of group][c]
    auto read_group = [&](int set, int s0) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int c = 0; c < 2; ++c) fk[set][j][c] = dma_read16<D, kRowPad>(kt, 32 * c + l32, h + 2 * (s0 + j));
    };
    read_group(0, 0);
#pragma unroll
    for (int s0 = 0; s0 < KD; s0 += 2) {
        const int set = (s0 >> 1) & 1;
        if (s0 + 2 < KD) read_group(set ^ 1, s0 + 2);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int c = 0; c < 2; ++c) sacc[c] = mfma32(fk[set][j][c], st.q[s0 + j], sacc[c]);
        __builtin_amdgcn_sched_barrier(0);
    }
    u32x4 av[2][4];   // V^T operands of one d block, read one block ahead
    auto read_tr = [&](int set, int b) {
#pragma unroll
        for (int g = 0; g < 4; ++g) av[set][g] = dma_read_tr<D, kTrPad>(vt, 16 * g, 32 * b, lane);
    };
    read_tr(0, 0);
    __builtin_amdgcn_sched_barrier(0);
    if (masked) {
        keep_branch();
        const int lim = min(S - 1, i);
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (!sees(i, j0 + 32 * c + 8 * (r >> 2) + 4 * h + (r & 3), W, lim)) sacc[c][r] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sacc[c][r]);
    mx = half_swap_max(mx) * c2;
    // lazy rescaling: the weights stay below 2^kSlack, so the accumulators move
    // only where a tile raises a row's maximum by more than that
    const bool raise = mx > st.m + kSlack;
    if (__any(raise)) {
        const float m = raise ? mx : st.m;
        const float alpha = st.m == -INFINITY ? 0.f : fast_exp2(st.m - m);
        st.l *= alpha;
        st.lr *= alpha;
#pragma unroll
        for (int b = 0; b < ND; ++b) st.o[b] *= alpha;
        st.m = m;
    }
    const float m_use = st.m == -INFINITY ? 0.f : st.m;
    float l0 = 0.f, l1 = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        sacc[0][r] = fast_exp2(__builtin_fmaf(sacc[0][r], c2, -m_use));
        sacc[1][r] = fast_exp2(__builtin_fmaf(sacc[1][r], c2, -m_use));
        l0 += sacc[0][r];
        l1 += sacc[1][r];
    }
    st.l += half_swap_sum(l0 + l1);
    u32x4 pb[4];
    pb[0] = pack8_bf16<0>(sacc[0]);
    pb[1] = pack8_bf16<8>(sacc[0]);
    pb[2] = pack8_bf16<0>(sacc[1]);
    pb[3] = pack8_bf16<8>(sacc[1]);
    st.lr += row_sum_bf16(pb);
#pragma unroll
    for (int b = 0; b < ND; ++b) {
        const int set = b & 1;
        if (b + 1 < ND) read_tr(set ^ 1, b + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int g = 0; g < 4; ++g) st.o[b] = mfma32(av[set][g], pb[g], st.o[b]);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// out and lse of this lane's row i
template <int D>
__device__ __forceinline__ void store_rows(const WindowArgs& a, const WinRows<D>& st, const Sequence& sq, int hq, int i,
                                           int h) {
    constexpr int ND = WinRows<D>::ND;
    const float inv = 1.f / st.lr;
    uint16_t* op = head_rows(a, a.out, sq, hq) + i * a.out.token;
#pragma unroll
    for (int x = 0; x < ND; ++x)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            u32x2 pk;
            pk.x = pack_bf16x2(st.o[x][4 * g + 0] * inv, st.o[x][4 * g + 1] * inv);
            pk.y = pack_bf16x2(st.o[x][4 * g + 2] * inv, st.o[x][4 * g + 3] * inv);
            *reinterpret_cast<u32x2*>(op + 32 * x + 8 * g + 4 * h) = pk;
        }
    if (h == 0) a.lse[lse_row(a, sq, hq) + i] = (st.m + fast_log2(st.l)) * kLn2;
}

// Two waves per SIMD at head dim 128 (256 registers), three at 64.
template <int D, bool BY_ROWS>
__global__ void __launch_bounds__(kFwdThreads) __attribute__((amdgpu_waves_per_eu(2, D == 64 ? 3 : 2)))
window_fwd_kernel(WindowArgs a) {
    constexpr int KD = WinRows<D>::KD, ND = WinRows<D>::ND;
    constexpr int KE = DmaTile<D, kRowPad>::kElems, VE = DmaTile<D, kTrPad>::kElems;
    __shared__ uint16_t k0s[KE], v0s[VE], k1s[KE], v1s[VE];
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, l32 = lane & 31;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    int b, hq, tile;
    if (!window_tile_of<BY_ROWS>(a, blockIdx.x, kFwdRows, b, hq, tile)) return;
    const Sequence sq = sequence(a, b);
    const int i0 = tile * kFwdRows;
    if (i0 >= sq.n) return;
    const int last = sq.n - 1;
    const int hk = hq / (a.Hq / a.Hkv);
    const uint16_t* kp = head_rows(a, a.k, sq, hk);
    const uint16_t* vp = head_rows(a, a.v, sq, hk);
    const int w0 = i0 + 32 * w, i = w0 + l32;    // the wave's first row, this lane's row
    WinRows<D> st;
    {
        const uint16_t* qp = head_rows(a, a.q, sq, hq) + min(i, last) * a.q.token;
#pragma unroll
        for (int s = 0; s < KD; ++s) st.q[s] = *reinterpret_cast<const u32x4*>(qp + 16 * s + 8 * h);
    }
#pragma unroll
    for (int x = 0; x < ND; ++x) st.o[x] = f32x16{};
    const float c2 = a.scale * kLog2e;
    const KeyWalk walk = key_walk(i0, min(i0 + kFwdRows - 1, last), a.W, a.S);
    auto load = [&](uint16_t* kt, uint16_t* vt, int t) {
        const int row0 = 64 * walk.tile(t);
        dma_sequence<D, kRowPad, 4>(kt, kp, a.k.token, row0, last, w, lane);
        dma_sequence<D, kTrPad, 4>(vt, vp, a.v.token, row0, last, w, lane);
    };
    load(k0s, v0s, 0);
    wait_vmem();
    __syncthreads();
    auto step = [&](int t, const uint16_t* ck, const uint16_t* cv, uint16_t* nk, uint16_t* nv) {
        if (t + 1 < walk.tiles) load(nk, nv, t + 1);
        const int j0 = 64 * walk.tile(t);
        const Sight seen = sight(w0, w0 + 31, j0, j0 + 63, a.W, a.S);
        if (seen != kNone && w0 <= last) win_tile<D>(ck, cv, seen == kPart, i, j0, a.W, a.S, st, lane, c2);
        __builtin_amdgcn_sched_barrier(0);
        wait_vmem();
        __syncthreads();
    };
    for (int t = 0; t < walk.tiles; t += 2) {
        step(t, k0s, v0s, k1s, v1s);
        if (t + 1 < walk.tiles) step(t + 1, k1s, v1s, k0s, v0s);
    }
    if (i <= last) store_rows(a, st, sq, hq, i, h);
}

// Small grids: 64 rows per workgroup, waves (row half, key half); the key halves walk
// alternate tiles with tile buffers of their own and are joined at the end, the
// second's (m, sums, O) into the first's.  A row tile's walk is bound by latency:
// half of it by half the rows each is faster while twice the workgroups, of which one
// fits a CU where two do otherwise (two where three do, at head dim 64), are resident
// at once.
template <int D, bool BY_ROWS>
__global__ void __launch_bounds__(kFwdThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
window_fwd_split_kernel(WindowArgs a) {
    constexpr int KD = WinRows<D>::KD, ND = WinRows<D>::ND;
    constexpr int KE = DmaTile<D, kRowPad>::kElems, VE = DmaTile<D, kTrPad>::kElems;
    __shared__ __attribute__((aligned(16))) uint16_t kb[2][2][KE], vb[2][2][VE];   // [half][parity]
    __shared__ float part[2][3][64];
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
    const KeyWalk walk = key_walk(i0, min(i0 + 63, last), a.W, a.S);
    const int steps = (walk.tiles + 1) >> 1;
    auto load = [&](int t) {   // tile 2 t + half
        const int row0 = 64 * walk.tile(2 * t + half);
        dma_sequence<D, kRowPad, 2>(kb[half][t & 1], kp, a.k.token, row0, last, rh, lane);
        dma_sequence<D, kTrPad, 2>(vb[half][t & 1], vp, a.v.token, row0, last, rh, lane);
    };
    if (half < walk.tiles) load(0);
    WinRows<D> st;
    const uint16_t* qp = head_rows(a, a.q, sq, hq) + min(i, last) * a.q.token;
#pragma unroll
    for (int s = 0; s < KD; ++s) st.q[s] = *reinterpret_cast<const u32x4*>(qp + 16 * s + 8 * h);
#pragma unroll
    for (int x = 0; x < ND; ++x) st.o[x] = f32x16{};
    for (int t = 0; t < steps; ++t) {
        wait_vmem();
        __syncthreads();   // tile t has landed, and the buffers of tile t - 1 are read
        if (2 * (t + 1) + half < walk.tiles) load(t + 1);
        if (2 * t + half < walk.tiles) {
            const int j0 = 64 * walk.tile(2 * t + half);
            const Sight seen = sight(w0, w0 + 31, j0, j0 + 63, a.W, a.S);
            if (seen != kNone && w0 <= last)
                win_tile<D>(kb[half][t & 1], vb[half][t & 1], seen == kPart, i, j0, a.W, a.S, st, lane, c2);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();   // every tile has been read
    float* ox = reinterpret_cast<float*>(&kb[0][0][0]) + rh * (ND * 16 * 64);
    static_assert(sizeof(kb) >= 2 * ND * 16 * 64 * 4, "exchange space");
    if (half == 1) {
#pragma unroll
        for (int x = 0; x < ND; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) ox[(x * 16 + r) * 64 + lane] = st.o[x][r];
        part[rh][0][lane] = st.m;
        part[rh][1][lane] = st.l;
        part[rh][2][lane] = st.lr;
    }
    __syncthreads();
    if (half == 1 || i > last) return;
    const float m1 = part[rh][0][lane], m = fmaxf(st.m, m1);
    const float a0 = st.m == -INFINITY ? 0.f : fast_exp2(st.m - m), a1 = m1 == -INFINITY ? 0.f : fast_exp2(m1 - m);
    st.m = m;
    st.l = st.l * a0 + part[rh][1][lane] * a1;
    st.lr = st.lr * a0 + part[rh][2][lane] * a1;
#pragma unroll
    for (int x = 0; x < ND; ++x)
#pragma unroll
        for (int r = 0; r < 16; ++r) st.o[x][r] = st.o[x][r] * a0 + ox[(x * 16 + r) * 64 + lane] * a1;
    store_rows(a, st, sq, hq, i, h);
}

}  // namespace

hipError_t launch_window_fwd(const WindowArgs& a, hipStream_t s) {
    const int64_t most = a.d == 128 ? kSplitGrid<128> : kSplitGrid<64>;
    const bool split = a.Hq * row_blocks(a.B, a.seq, a.tokens, kFwdRows) <= most;
    TraceScope _t("window_fwd", s);
    const dim3 g(unsigned(a.Hq * grid_blocks(a.by_rows, a.B, a.seq, a.tokens, split ? 64 : kFwdRows))), t(kFwdThreads);
    window_variant(a, [&](auto dim, auto by_rows) {
        constexpr int D = decltype(dim)::value;
        constexpr bool R = decltype(by_rows)::value;
        if (split) hipLaunchKernelGGL((window_fwd_split_kernel<D, R>), g, t, 0, s, a);
        else hipLaunchKernelGGL((window_fwd_kernel<D, R>), g, t, 0, s, a);
    });
    return hipGetLastError();
}

}  // namespace msparse
