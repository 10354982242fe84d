// C ABI of libmsparse: argument validation, workspace carve-up and launches.
// Every check runs on the host before the first launch, so an error return
// leaves the stream untouched.
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <initializer_list>
#include <mutex>
#include <string>

#include "cache.h"
#include "common.h"
#include "kernels.h"
#include "operands.h"
#include "rotate.h"
#include "window.h"

using namespace msparse;

namespace {

thread_local std::string g_last_error;

msparse_status fail(msparse_status st, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    g_last_error = buf;
    return st;
}

// Every tensor named in the header's conventions is read or written with
// 16-byte vector accesses; NULL (an optional tensor) passes.
bool misaligned(std::initializer_list<const void*> ps) {
    for (const void* p : ps)
        if (reinterpret_cast<uintptr_t>(p) & 15u) return true;
    return false;
}

// arrays of 32-bit words that are read one by one
bool odd_words(std::initializer_list<const void*> ps) {
    for (const void* p : ps)
        if (reinterpret_cast<uintptr_t>(p) & 3u) return true;
    return false;
}

bool sync_check_enabled() {
    static int v = [] {
        const char* e = getenv("MSPARSE_SYNC_CHECK");
        return (e && e[0] && e[0] != '0') ? 1 : 0;
    }();
    return v != 0;
}

msparse_status check_hip(hipError_t e, hipStream_t s, const char* what) {
    if (e != hipSuccess) return fail(MSPARSE_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
    if (sync_check_enabled()) {
        // a stream under graph capture cannot be synchronised: its work runs
        // at replay, so the check is skipped there
        hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
        e = hipStreamIsCapturing(s, &cap);
        if (e == hipSuccess && cap == hipStreamCaptureStatusNone) e = hipStreamSynchronize(s);
        if (e == hipSuccess) e = hipGetLastError();
        if (e != hipSuccess) return fail(MSPARSE_ERR_HIP, "%s (sync check): %s", what, hipGetErrorString(e));
    }
    return MSPARSE_OK;
}

constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

// Bump allocator over the caller's workspace.
struct Carve {
    char* base;
    size_t off = 0;
    template <class T>
    T* take(size_t count) {
        T* p = base ? reinterpret_cast<T*>(base + off) : nullptr;
        off = align_up(off + count * sizeof(T));
        return p;
    }
};

float resolve_scale(const msparse_dims* d) { return d->scale > 0.f ? d->scale : 1.0f / std::sqrt(float(d->head_dim)); }

msparse_status check_dims(const msparse_dims* d, bool same_len) {
    if (!d) return fail(MSPARSE_ERR_INVALID, "dims is NULL");
    if (d->batch < 1 || d->heads_q < 1 || d->heads_kv < 1 || d->seq_q < 0 || d->seq_k < 0)
        return fail(MSPARSE_ERR_INVALID, "batch, heads must be >= 1 and lengths >= 0");
    if (d->heads_q % d->heads_kv != 0)
        return fail(MSPARSE_ERR_INVALID, "heads_q (%d) is not a multiple of heads_kv (%d)", d->heads_q, d->heads_kv);
    if (d->head_dim != 64 && d->head_dim != 128)
        return fail(MSPARSE_ERR_UNSUPPORTED, "head_dim %d (supported: 64, 128)", d->head_dim);
    if (d->block != kBlock) return fail(MSPARSE_ERR_UNSUPPORTED, "block %d (supported: 64)", d->block);
    if (d->causal != 1) return fail(MSPARSE_ERR_UNSUPPORTED, "only causal attention is supported");
    if (d->seq_q % kBlock || d->seq_k % kBlock)
        return fail(MSPARSE_ERR_UNSUPPORTED, "sequence lengths (%d, %d) must be multiples of 64", d->seq_q, d->seq_k);
    if (same_len && d->seq_q != d->seq_k) return fail(MSPARSE_ERR_INVALID, "seq_q != seq_k");
    if (!std::isfinite(d->scale)) return fail(MSPARSE_ERR_INVALID, "scale is not finite");
    const int64_t big = int64_t(d->batch) * d->heads_q * int64_t(std::max(d->seq_q, d->seq_k));
    if (big > (int64_t(1) << 31) - 1) return fail(MSPARSE_ERR_UNSUPPORTED, "batch * heads * seq exceeds 2^31 rows");
    return MSPARSE_OK;
}

struct RingInfo {
    int32_t world = 1, rank = 0, step = 0, layout = MSPARSE_LAYOUT_STRIPED, shard = 0;
};

// Shard held by `rank` at `step`: flat ring, or the hierarchical order of
// Algorithm 2 (outer ring over nodes of `inner` cards, inner ring per node).
int32_t ring_shard(int32_t world, int32_t inner, int32_t rank, int32_t step) {
    if (world < 1 || rank < 0 || rank >= world || step < 0 || step >= world) return -1;
    if (inner < 0 || (inner > 0 && world % inner != 0)) return -1;
    if (inner <= 1 || inner == world) return ((rank - step) % world + world) % world;
    const int32_t nodes = world / inner;
    const int32_t node = rank / inner, card = rank % inner;
    const int32_t i = step / inner, j = step % inner;
    return ((node - i) % nodes + nodes) % nodes * inner + ((card - j) % inner + inner) % inner;
}

msparse_status check_ring(const msparse_dims* d, const msparse_ring* r, RingInfo* out) {
    RingInfo ri;
    if (r) {
        if (r->world < 1 || r->rank < 0 || r->rank >= r->world || r->step < 0 || r->step >= r->world)
            return fail(MSPARSE_ERR_INVALID, "ring world %d rank %d step %d", r->world, r->rank, r->step);
        if (r->layout != MSPARSE_LAYOUT_STRIPED && r->layout != MSPARSE_LAYOUT_ZIGZAG)
            return fail(MSPARSE_ERR_INVALID, "ring layout %d", r->layout);
        if (r->inner < 0 || (r->inner > 0 && r->world % r->inner != 0))
            return fail(MSPARSE_ERR_INVALID, "ring inner %d does not divide world %d", r->inner, r->world);
        ri.world = r->world;
        ri.rank = r->rank;
        ri.step = r->step;
        ri.layout = r->layout;
        ri.shard = ring_shard(r->world, r->inner, r->rank, r->step);
        if (r->layout == MSPARSE_LAYOUT_ZIGZAG && (d->seq_q / kBlock) % 2 != 0)
            return fail(MSPARSE_ERR_UNSUPPORTED, "zigzag shards need an even number of 64-token blocks");
    }
    if (d->seq_q != d->seq_k) return fail(MSPARSE_ERR_INVALID, "query and KV shards must have equal length");
    const int64_t ng = int64_t(d->seq_q) * ri.world;
    if (ng > (int64_t(1) << 30)) return fail(MSPARSE_ERR_UNSUPPORTED, "global sequence too long");
    *out = ri;
    return MSPARSE_OK;
}

// ------------------------------------------------------------------ index
struct IndexPlan {
    IndexArgs a{};
    size_t bytes = 0;
};

IndexPlan plan_index(const msparse_dims* d, int32_t k_v, int32_t k_s, const RingInfo& ri, void* ws,
                     bool own_ptrs) {
    IndexPlan p;
    IndexArgs& a = p.a;
    a.BH = d->batch * d->heads_q;
    a.k_v = k_v;
    a.k_s = k_s;
    a.nqb = d->seq_q / kBlock;
    a.nkb = d->seq_k / kBlock;
    a.nb = a.nqb * ri.world;
    a.world = ri.world;
    a.rank = ri.rank;
    a.shard = ri.shard;
    a.layout = ri.layout;
    const int64_t ng = int64_t(a.nb) * kBlock;
    a.vwords = int32_t((ng + 31) / 32);
    a.dwords = (a.nb + 31) / 32;
    Carve c{static_cast<char*>(ws)};
    a.chunk = index_chunk(a.BH, std::max(a.nqb, a.nkb));
    a.nchq = (a.nqb + a.chunk - 1) / a.chunk;
    a.nchk = (a.nkb + a.chunk - 1) / a.chunk;
    a.vbits = c.take<uint32_t>(size_t(a.BH) * a.vwords);
    a.vlist = c.take<int32_t>(size_t(a.BH) * k_v);
    a.vcnt = c.take<int32_t>(a.BH);
    a.dlist = c.take<int32_t>(size_t(a.BH) * a.nb);
    a.dcnt = c.take<int32_t>(a.BH);
    a.dbits = c.take<uint32_t>(size_t(a.BH) * a.dwords);
    a.dpre = c.take<int32_t>(size_t(a.BH) * (a.dwords + 1));
    a.cumv = c.take<int32_t>(size_t(a.BH) * (a.nb + 1));
    a.drun = c.take<int32_t>(a.BH);
    a.cnt_blk = c.take<int64_t>(size_t(a.BH) * a.nqb);
    a.cnt_col = c.take<int64_t>(size_t(a.BH) * a.nqb);
    a.cnt_kblk = c.take<int64_t>(size_t(a.BH) * a.nkb);
    a.cnt_vcol = c.take<int64_t>(a.BH);
    // Offsets of the calls that keep none, and in the same place the chunk totals
    // of the count pass: no more chunks than blocks, so they end before the last
    // offset, the one that such a call reads (shards are of equal length, so the
    // three arrays lie at equal distances).  Reserved either way, so that the
    // size query does not depend on the mode.
    const size_t nq = size_t(a.BH) * a.nqb, nk = size_t(a.BH) * a.nkb;
    const size_t first = c.off;
    int64_t* blk_ptr = c.take<int64_t>(nq + 1);
    a.scan_sums = blk_ptr;
    a.scan_stride = int64_t((c.off - first) / sizeof(int64_t));
    int64_t* col_ptr = c.take<int64_t>(nq + 1);
    int64_t* kblk_ptr = c.take<int64_t>(nk + 1);
    int64_t* vcol_ptr = c.take<int64_t>(size_t(a.BH) + 1);
    if (own_ptrs) {
        a.blk_ptr = blk_ptr;
        a.col_ptr = col_ptr;
        a.kblk_ptr = kblk_ptr;
        a.vcol_ptr = vcol_ptr;
    }
    p.bytes = c.off;
    return p;
}

msparse_status check_index_inputs(const msparse_dims* d, const int32_t* v_idx, int32_t k_v, const int32_t* s_idx,
                                  int32_t k_s, const msparse_ring* ring, RingInfo* ri) {
    msparse_status st = check_dims(d, false);
    if (st) return st;
    if ((st = check_ring(d, ring, ri))) return st;
    if (!v_idx || !s_idx) return fail(MSPARSE_ERR_INVALID, "v_idx / s_idx is NULL");
    const int64_t ng = int64_t(d->seq_q) * ri->world;
    if (k_v < 1 || k_v > ng || k_s < 1 || k_s > ng)
        return fail(MSPARSE_ERR_INVALID, "budgets k_v=%d k_s=%d outside [1, %lld]", k_v, k_s, (long long)ng);
    if (d->seq_q == 0) return fail(MSPARSE_ERR_INVALID, "empty sequence");
    const int64_t items = int64_t(d->batch) * d->heads_q * std::max(d->seq_q, d->seq_k) / kBlock;
    if (items > kMaxIndexItems)
        return fail(MSPARSE_ERR_UNSUPPORTED, "%lld (head, block) items exceed the index build's %lld",
                    (long long)items, (long long)kMaxIndexItems);
    return MSPARSE_OK;
}

msparse_status check_index_struct(const msparse_dims* d, const msparse_index* x, bool need_transpose) {
    if (!x) return fail(MSPARSE_ERR_INVALID, "index is NULL");
    if (!x->blk_ptr || !x->col_ptr || !x->q_blk_global || !x->k_blk_global || !x->diag_bits)
        return fail(MSPARSE_ERR_INVALID, "index arrays are NULL");
    if ((x->blk_cap > 0 && !x->blk_idx) || (x->col_cap > 0 && !x->col_idx))
        return fail(MSPARSE_ERR_INVALID, "index entry arrays are NULL");
    if (need_transpose && (!x->kblk_ptr || !x->vcol_ptr || (x->blk_cap > 0 && !x->kblk_idx) ||
                           (x->vcol_cap > 0 && !x->vcol_idx)))
        return fail(MSPARSE_ERR_INVALID, "transposed index arrays are NULL");
    if (x->blk_cap < 0 || x->col_cap < 0 || x->vcol_cap < 0) return fail(MSPARSE_ERR_INVALID, "negative capacity");
    if (x->world < 1) return fail(MSPARSE_ERR_INVALID, "index world %d < 1", x->world);
    (void)d;
    return MSPARSE_OK;
}

// ------------------------------------------------------------------ allocation-free index build
// Scratch of msparse_build_index_noalloc: file-scope device memory, one copy
// per GPU, made when the code object loads on that GPU and held until the
// process ends.  In host code `scratch` names a host-side stand-in, not a
// device address: the address each GPU uses comes from hipGetSymbolAddress
// (scratch_on_current_device) and is the only one passed to kernels.
constexpr size_t kNoallocScratchBytes = size_t(64) << 20;
constexpr int kMaxDevices = 256;

}  // namespace

static __device__ __align__(256) unsigned char scratch[kNoallocScratchBytes];

namespace {

std::mutex g_scratch_mu;
void* g_scratch_ptr[kMaxDevices] = {};

// The current device's copy of `scratch`, looked up once per device (with
// that device current) and kept.
msparse_status scratch_on_current_device(void** out) {
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return fail(MSPARSE_ERR_HIP, "hipGetDevice: %s", hipGetErrorString(e));
    if (dev < 0 || dev >= kMaxDevices) return fail(MSPARSE_ERR_UNSUPPORTED, "device %d beyond %d", dev, kMaxDevices);
    std::lock_guard<std::mutex> lock(g_scratch_mu);
    if (!g_scratch_ptr[dev]) {
        void* p = nullptr;
        e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
        if (e != hipSuccess || !p)
            return fail(MSPARSE_ERR_HIP, "hipGetSymbolAddress(scratch) on device %d: %s", dev, hipGetErrorString(e));
        g_scratch_ptr[dev] = p;
    }
    *out = g_scratch_ptr[dev];
    return MSPARSE_OK;
}

}  // namespace

extern "C" {

const char* msparse_strerror(msparse_status s) {
    switch (s) {
        case MSPARSE_OK: return "ok";
        case MSPARSE_ERR_INVALID: return "invalid argument";
        case MSPARSE_ERR_UNSUPPORTED: return "unsupported configuration";
        case MSPARSE_ERR_CAPACITY: return "index capacity too small";
        case MSPARSE_ERR_WORKSPACE: return "workspace too small";
        case MSPARSE_ERR_HIP: return "HIP runtime error";
    }
    return "unknown status";
}

const char* msparse_last_error(void) { return g_last_error.c_str(); }

int32_t msparse_ring_shard(int32_t world, int32_t inner, int32_t rank, int32_t step) {
    return ring_shard(world, inner, rank, step);
}

// ------------------------------------------------------------------ index
size_t msparse_index_workspace(const msparse_dims* dims, int32_t k_v, int32_t k_s, const msparse_ring* ring) {
    RingInfo ri;
    if (check_dims(dims, false) || check_ring(dims, ring, &ri) || k_v < 1 || k_s < 1) return 0;
    return plan_index(dims, k_v, k_s, ri, nullptr, true).bytes;
}

msparse_status msparse_index_count(const msparse_dims* dims, const int32_t* v_idx, int32_t k_v, const int32_t* s_idx,
                                   int32_t k_s, const msparse_ring* ring, int64_t* blk_nnz, int64_t* col_nnz,
                                   int64_t* vcol_nnz, void* ws, size_t ws_bytes, void* stream) {
    RingInfo ri;
    msparse_status st = check_index_inputs(dims, v_idx, k_v, s_idx, k_s, ring, &ri);
    if (st) return st;
    if (!blk_nnz || !col_nnz || !vcol_nnz) return fail(MSPARSE_ERR_INVALID, "count outputs are NULL");
    IndexPlan p = plan_index(dims, k_v, k_s, ri, ws, true);
    if (!ws || ws_bytes < p.bytes)
        return fail(MSPARSE_ERR_WORKSPACE, "index workspace %zu < %zu bytes", ws_bytes, p.bytes);
    p.a.v_idx = v_idx;
    p.a.s_idx = s_idx;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if ((st = check_hip(launch_index_prep(p.a, s), s, "index prep"))) return st;
    if ((st = check_hip(launch_index_count(p.a, s), s, "index count"))) return st;
    if ((st = check_hip(launch_index_scan(p.a, s), s, "index scan"))) return st;
    int64_t tot[3];
    const int64_t nq = int64_t(p.a.BH) * p.a.nqb;
    hipError_t e = hipMemcpyAsync(&tot[0], p.a.blk_ptr + nq, 8, hipMemcpyDeviceToHost, s);
    if (e == hipSuccess) e = hipMemcpyAsync(&tot[1], p.a.col_ptr + nq, 8, hipMemcpyDeviceToHost, s);
    if (e == hipSuccess) e = hipMemcpyAsync(&tot[2], p.a.vcol_ptr + p.a.BH, 8, hipMemcpyDeviceToHost, s);
    if (e == hipSuccess) e = hipStreamSynchronize(s);
    if (e != hipSuccess) return fail(MSPARSE_ERR_HIP, "index count readback: %s", hipGetErrorString(e));
    *blk_nnz = tot[0];
    *col_nnz = tot[1];
    *vcol_nnz = tot[2];
    return MSPARSE_OK;
}

msparse_status msparse_build_index(const msparse_dims* dims, const int32_t* v_idx, int32_t k_v, const int32_t* s_idx,
                                   int32_t k_s, const msparse_ring* ring, const msparse_index* index, void* ws,
                                   size_t ws_bytes, void* stream) {
    RingInfo ri;
    msparse_status st = check_index_inputs(dims, v_idx, k_v, s_idx, k_s, ring, &ri);
    if (st) return st;
    if ((st = check_index_struct(dims, index, true))) return st;
    if (index->world != ri.world)
        return fail(MSPARSE_ERR_INVALID, "index world %d differs from the ring world %d", index->world, ri.world);
    IndexPlan p = plan_index(dims, k_v, k_s, ri, ws, false);
    if (!ws || ws_bytes < p.bytes)
        return fail(MSPARSE_ERR_WORKSPACE, "index workspace %zu < %zu bytes", ws_bytes, p.bytes);
    // Without an overflow flag the capacities must cover the worst case.
    const int64_t BH = p.a.BH, nqb = p.a.nqb, nkb = p.a.nkb;
    const int64_t dmax = std::min<int64_t>(p.a.nb, 2 * int64_t(k_s));
    const int64_t blk_bound = BH * nqb * std::min<int64_t>(nkb, dmax);
    const int64_t col_bound = BH * nqb * std::min<int64_t>(k_v, nkb * kBlock);
    const int64_t vcol_bound = BH * std::min<int64_t>(k_v, nkb * kBlock);
    if (!index->overflow && (index->blk_cap < blk_bound || index->col_cap < col_bound || index->vcol_cap < vcol_bound))
        return fail(MSPARSE_ERR_CAPACITY,
                    "capacities (%lld, %lld, %lld) below the worst case (%lld, %lld, %lld) and no overflow flag",
                    (long long)index->blk_cap, (long long)index->col_cap, (long long)index->vcol_cap,
                    (long long)blk_bound, (long long)col_bound, (long long)vcol_bound);
    IndexArgs& a = p.a;
    a.v_idx = v_idx;
    a.s_idx = s_idx;
    a.blk_ptr = index->blk_ptr;
    a.col_ptr = index->col_ptr;
    a.kblk_ptr = index->kblk_ptr;
    a.vcol_ptr = index->vcol_ptr;
    a.blk_idx = index->blk_idx;
    a.blk_cap = index->blk_cap;
    a.col_idx = index->col_idx;
    a.col_cap = index->col_cap;
    a.kblk_idx = index->kblk_idx;
    a.vcol_idx = index->vcol_idx;
    a.vcol_cap = index->vcol_cap;
    a.diag_bits_out = index->diag_bits;
    a.q_blk_global = index->q_blk_global;
    a.k_blk_global = index->k_blk_global;
    a.overflow = index->overflow;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if ((st = check_hip(launch_index_prep(a, s), s, "index prep"))) return st;   // also clears the overflow flag
    if ((st = check_hip(launch_index_count(a, s), s, "index count"))) return st;
    a.scanned = int64_t(a.BH) * std::max(a.nchq, a.nchk) > kDirectChunks;
    if (a.scanned && (st = check_hip(launch_index_scan(a, s), s, "index scan"))) return st;
    return check_hip(launch_index_fill(a, s), s, "index fill");
}

msparse_status msparse_index_count_build(const msparse_dims* dims, const int32_t* v_idx, int32_t k_v,
                                         const int32_t* s_idx, int32_t k_s, const msparse_ring* ring,
                                         const msparse_index* index, int64_t* blk_nnz, int64_t* col_nnz,
                                         int64_t* vcol_nnz, void* ws, size_t ws_bytes, void* stream) {
    RingInfo ri;
    msparse_status st = check_index_inputs(dims, v_idx, k_v, s_idx, k_s, ring, &ri);
    if (st) return st;
    if ((st = check_index_struct(dims, index, true))) return st;
    if (!blk_nnz || !col_nnz || !vcol_nnz) return fail(MSPARSE_ERR_INVALID, "count outputs are NULL");
    if (!index->overflow) return fail(MSPARSE_ERR_INVALID, "msparse_index_count_build needs an overflow flag");
    if (index->world != ri.world)
        return fail(MSPARSE_ERR_INVALID, "index world %d differs from the ring world %d", index->world, ri.world);
    IndexPlan p = plan_index(dims, k_v, k_s, ri, ws, false);
    if (!ws || ws_bytes < p.bytes)
        return fail(MSPARSE_ERR_WORKSPACE, "index workspace %zu < %zu bytes", ws_bytes, p.bytes);
    IndexArgs& a = p.a;
    a.v_idx = v_idx;
    a.s_idx = s_idx;
    a.blk_ptr = index->blk_ptr;
    a.col_ptr = index->col_ptr;
    a.kblk_ptr = index->kblk_ptr;
    a.vcol_ptr = index->vcol_ptr;
    a.blk_idx = index->blk_idx;
    a.blk_cap = index->blk_cap;
    a.col_idx = index->col_idx;
    a.col_cap = index->col_cap;
    a.kblk_idx = index->kblk_idx;
    a.vcol_idx = index->vcol_idx;
    a.vcol_cap = index->vcol_cap;
    a.diag_bits_out = index->diag_bits;
    a.q_blk_global = index->q_blk_global;
    a.k_blk_global = index->k_blk_global;
    a.overflow = index->overflow;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if ((st = check_hip(launch_index_prep(a, s), s, "index prep"))) return st;   // also clears the overflow flag
    if ((st = check_hip(launch_index_count(a, s), s, "index count"))) return st;
    a.scanned = 1;
    if ((st = check_hip(launch_index_scan(a, s), s, "index scan"))) return st;
    int64_t tot[3];
    const int64_t nq = int64_t(a.BH) * a.nqb;
    hipError_t e = hipMemcpyAsync(&tot[0], a.blk_ptr + nq, 8, hipMemcpyDeviceToHost, s);
    if (e == hipSuccess) e = hipMemcpyAsync(&tot[1], a.col_ptr + nq, 8, hipMemcpyDeviceToHost, s);
    if (e == hipSuccess) e = hipMemcpyAsync(&tot[2], a.vcol_ptr + a.BH, 8, hipMemcpyDeviceToHost, s);
    if (e == hipSuccess) e = hipStreamSynchronize(s);
    if (e != hipSuccess) return fail(MSPARSE_ERR_HIP, "index count readback: %s", hipGetErrorString(e));
    *blk_nnz = tot[0];
    *col_nnz = tot[1];
    *vcol_nnz = tot[2];
    if (tot[0] > index->blk_cap || tot[1] > index->col_cap || tot[2] > index->vcol_cap) {
        // the lists stay unfilled: flag the index so that no attention call walks it
        if ((st = check_hip(launch_index_mark_overflow(a, s), s, "index overflow mark"))) return st;
        return fail(MSPARSE_ERR_CAPACITY, "index needs (%lld, %lld, %lld) entries; capacities (%lld, %lld, %lld)",
                    (long long)tot[0], (long long)tot[1], (long long)tot[2], (long long)index->blk_cap,
                    (long long)index->col_cap, (long long)index->vcol_cap);
    }
    return check_hip(launch_index_fill(a, s), s, "index fill");
}

msparse_status msparse_build_index_noalloc(const msparse_dims* dims, const int32_t* v_idx, int32_t k_v,
                                           const int32_t* s_idx, int32_t k_s, const msparse_ring* ring,
                                           const msparse_index* index, void* stream) {
    RingInfo ri;
    msparse_status st = check_index_inputs(dims, v_idx, k_v, s_idx, k_s, ring, &ri);
    if (st) return st;
    if ((st = check_index_struct(dims, index, true))) return st;
    const size_t need = plan_index(dims, k_v, k_s, ri, nullptr, false).bytes;
    if (need > kNoallocScratchBytes)
        return fail(MSPARSE_ERR_WORKSPACE, "index build needs %zu bytes of scratch; the fixed scratch holds %zu",
                    need, kNoallocScratchBytes);
    void* ws = nullptr;
    if ((st = scratch_on_current_device(&ws))) return st;
    return msparse_build_index(dims, v_idx, k_v, s_idx, k_s, ring, index, ws, need, stream);
}

// ------------------------------------------------------------------ attention
static msparse_status fill_attn(const msparse_dims* d, const msparse_index* x, AttnArgs* a) {
    a->B = d->batch;
    a->Hq = d->heads_q;
    a->Hkv = d->heads_kv;
    a->Nq = d->seq_q;
    a->Nk = d->seq_k;
    a->d = d->head_dim;
    a->nqb = d->seq_q / kBlock;
    a->nkb = d->seq_k / kBlock;
    a->scale = resolve_scale(d);
    a->blk_ptr = x->blk_ptr;
    a->blk_idx = x->blk_idx;
    a->col_ptr = x->col_ptr;
    a->col_idx = x->col_idx;
    a->kblk_ptr = x->kblk_ptr;
    a->kblk_idx = x->kblk_idx;
    a->vcol_ptr = x->vcol_ptr;
    a->vcol_idx = x->vcol_idx;
    a->diag_bits = x->diag_bits;
    a->dwords = (d->seq_q / kBlock * x->world + 31) / 32;
    a->q_blk_global = x->q_blk_global;
    a->k_blk_global = x->k_blk_global;
    a->overflow = x->overflow;
    return MSPARSE_OK;
}

// Forward workspace: the scaled fp16 copy of V and the max words.
static size_t carve_fwd(const msparse_dims* d, char* base, AttnArgs* a) {
    Carve c{base};
    uint16_t* v16 = c.take<uint16_t>(size_t(d->batch) * d->heads_kv * d->seq_k * d->head_dim);
    uint32_t* mx = c.take<uint32_t>(3);
    uint32_t* part = c.take<uint32_t>(kMaxParts);
    if (a) {
        a->v16 = v16;
        a->qkvmax = mx;
        a->maxpart = part;
    }
    return c.off;
}

size_t msparse_attn_fwd_workspace(const msparse_dims* dims) {
    if (check_dims(dims, false)) return 0;
    return carve_fwd(dims, nullptr, nullptr);
}

msparse_status msparse_attn_fwd(const msparse_dims* dims, const void* q, const void* k, const void* v,
                                const msparse_index* index, void* out, float* lse, float* out_f32, void* ws,
                                size_t ws_bytes, void* stream) {
    msparse_status st = check_dims(dims, false);
    if (st) return st;
    if (!q || !k || !v || (!out && !out_f32) || !lse) return fail(MSPARSE_ERR_INVALID, "tensor pointer is NULL");
    if (misaligned({q, k, v, out, out_f32, lse})) return fail(MSPARSE_ERR_INVALID, "tensor not 16-byte aligned");
    if ((st = check_index_struct(dims, index, false))) return st;
    const size_t need = msparse_attn_fwd_workspace(dims);
    if (need && (!ws || ws_bytes < need))
        return fail(MSPARSE_ERR_WORKSPACE, "fwd workspace %zu < %zu bytes", ws_bytes, need);
    if (dims->seq_q == 0) return MSPARSE_OK;
    AttnArgs a{};
    fill_attn(dims, index, &a);
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.out = static_cast<uint16_t*>(out);
    a.out_f32 = out_f32;
    a.lse = lse;
    carve_fwd(dims, static_cast<char*>(ws), &a);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return check_hip(launch_attn_fwd(a, s), s, "attn fwd");
}

msparse_status msparse_attn_fwd_merge(const msparse_dims* dims, const void* q, const void* k, const void* v,
                                      const msparse_index* index, float* o_acc, float* lse_acc, void* out_bf16,
                                      int32_t first, void* ws, size_t ws_bytes, void* stream) {
    msparse_status st = check_dims(dims, false);
    if (st) return st;
    if (!q || !k || !v || !o_acc || !lse_acc) return fail(MSPARSE_ERR_INVALID, "tensor pointer is NULL");
    if (misaligned({q, k, v, o_acc, lse_acc, out_bf16}))
        return fail(MSPARSE_ERR_INVALID, "tensor not 16-byte aligned");
    if ((st = check_index_struct(dims, index, false))) return st;
    const size_t need = msparse_attn_fwd_workspace(dims);
    if (need && (!ws || ws_bytes < need))
        return fail(MSPARSE_ERR_WORKSPACE, "fwd workspace %zu < %zu bytes", ws_bytes, need);
    if (dims->seq_q == 0) return MSPARSE_OK;
    AttnArgs a{};
    fill_attn(dims, index, &a);
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.out = static_cast<uint16_t*>(out_bf16);
    a.out_f32 = o_acc;
    a.lse = lse_acc;
    a.merge_acc = first ? 0 : 1;
    carve_fwd(dims, static_cast<char*>(ws), &a);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return check_hip(launch_attn_fwd(a, s), s, "attn fwd merge");
}

msparse_status msparse_merge_out_lse(const msparse_dims* dims, const float* o_part, const float* lse_part, float* o_acc,
                                     float* lse_acc, void* out_bf16, int32_t first, void* stream) {
    msparse_status st = check_dims(dims, false);
    if (st) return st;
    if (!o_part || !lse_part || !o_acc || !lse_acc) return fail(MSPARSE_ERR_INVALID, "tensor pointer is NULL");
    if (misaligned({o_part, lse_part, o_acc, lse_acc, out_bf16}))
        return fail(MSPARSE_ERR_INVALID, "tensor not 16-byte aligned");
    if (dims->seq_q == 0) return MSPARSE_OK;
    MergeArgs m{};
    m.o_part = o_part;
    m.lse_part = lse_part;
    m.o_acc = o_acc;
    m.lse_acc = lse_acc;
    m.out = static_cast<uint16_t*>(out_bf16);
    m.first = first;
    m.rows = int64_t(dims->batch) * dims->heads_q * dims->seq_q;
    m.d = dims->head_dim;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return check_hip(launch_merge(m, s), s, "merge out/lse");
}

// Backward workspace: scaled fp16 copies of K, V, Q and dO, Delta, s Delta, lse2, the
// max words, the column work list and the per-item column partials.
static size_t carve_bwd(const msparse_dims* d, int64_t vcol_cap, char* base, AttnArgs* a) {
    const int64_t bh = int64_t(d->batch) * d->heads_q;
    const ColPlanSizes z = col_plan_sizes(bh, vcol_cap, d->seq_q / kBlock);
    Carve c{base};
    uint16_t* k16 = c.take<uint16_t>(size_t(d->batch) * d->heads_kv * d->seq_k * d->head_dim);
    uint16_t* v16 = c.take<uint16_t>(size_t(d->batch) * d->heads_kv * d->seq_k * d->head_dim);
    uint16_t* q16 = c.take<uint16_t>(size_t(bh) * d->seq_q * d->head_dim);
    uint16_t* g16 = c.take<uint16_t>(size_t(bh) * d->seq_q * d->head_dim);
    float* draw = c.take<float>(size_t(bh) * d->seq_q);
    float* delta = c.take<float>(size_t(bh) * d->seq_q);
    float* lse2 = c.take<float>(size_t(bh) * d->seq_q);
    uint32_t* dmax = c.take<uint32_t>(4);   // max |dO|, |Q|, |K|, |V|
    int32_t* choff = c.take<int32_t>(size_t(bh) + 1);
    int64_t* e0 = c.take<int64_t>(size_t(z.chunk_cap));
    int32_t* head = c.take<int32_t>(size_t(z.chunk_cap));
    int32_t* qlo = c.take<int32_t>(size_t(z.chunk_cap));
    int32_t* item = c.take<int32_t>(size_t(z.chunk_cap) + 1);
    int32_t* span = c.take<int32_t>(1);
    uint32_t* part = c.take<uint32_t>(4 * kMaxParts);   // per-workgroup maxima, within one call
    float* dkc = c.take<float>(size_t(z.slots) * kBlock * d->head_dim);
    float* dvc = c.take<float>(size_t(z.slots) * kBlock * d->head_dim);
    if (a) {
        a->k16 = k16;
        a->v16 = v16;
        a->q16 = q16;
        a->g16 = g16;
        a->draw = draw;
        a->delta = delta;
        a->lse2 = lse2;
        a->dmax = dmax;
        a->qkvmax = dmax + 1;
        a->maxpart = part;
        a->col_choff = choff;
        a->col_e0 = e0;
        a->col_head = head;
        a->col_qlo = qlo;
        a->col_item = item;
        a->col_span = span;
        a->col_chunk_cap = z.chunk_cap;
        a->col_budget = z.budget;
        a->col_slots = z.slots;
        a->dk_col = dkc;
        a->dv_col = dvc;
    }
    return c.off;
}

size_t msparse_attn_bwd_workspace(const msparse_dims* dims, int64_t vcol_cap) {
    if (check_dims(dims, false) || vcol_cap < 0) return 0;
    return carve_bwd(dims, vcol_cap, nullptr, nullptr);
}

msparse_status msparse_attn_bwd(const msparse_dims* dims, const void* q, const void* k, const void* v,
                                const void* out, const float* out_f32, const void* dout, const float* lse,
                                const msparse_index* index, float* dq, float* dk, float* dv, int32_t flags,
                                void* ws, size_t ws_bytes, void* stream) {
    msparse_status st = check_dims(dims, false);
    if (st) return st;
    if (!q || !k || !v || !out || !dout || !lse || !dq || !dk || !dv)
        return fail(MSPARSE_ERR_INVALID, "tensor pointer is NULL");
    if (misaligned({q, k, v, out, out_f32, dout, lse, dq, dk, dv}))
        return fail(MSPARSE_ERR_INVALID, "tensor not 16-byte aligned");
    if ((st = check_index_struct(dims, index, true))) return st;
    if (flags & ~(MSPARSE_BWD_ACCUMULATE_DQ | MSPARSE_BWD_REUSE_QROWS))
        return fail(MSPARSE_ERR_INVALID, "backward flags 0x%x", unsigned(flags));
    const size_t need = msparse_attn_bwd_workspace(dims, index->vcol_cap);
    if (!ws || ws_bytes < need) return fail(MSPARSE_ERR_WORKSPACE, "bwd workspace %zu < %zu bytes", ws_bytes, need);
    if (dims->seq_q == 0 && dims->seq_k == 0) return MSPARSE_OK;
    AttnArgs a{};
    fill_attn(dims, index, &a);
    carve_bwd(dims, index->vcol_cap, static_cast<char*>(ws), &a);
    a.vcol_cap = index->vcol_cap;
    a.o_f32 = out_f32;
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.o = static_cast<const uint16_t*>(out);
    a.dout = static_cast<const uint16_t*>(dout);
    a.lse = const_cast<float*>(lse);
    a.dq = dq;
    a.dk = dk;
    a.dv = dv;
    a.dq_accumulate = (flags & MSPARSE_BWD_ACCUMULATE_DQ) != 0;
    a.reuse_qrows = (flags & MSPARSE_BWD_REUSE_QROWS) != 0;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return check_hip(launch_attn_bwd(a, s), s, "attn bwd");
}

// ------------------------------------------------------------------ ring workload
msparse_status msparse_ring_work(const msparse_dims* dims, const int32_t* v_idx, int32_t k_v, const int32_t* s_idx,
                                 int32_t k_s, int32_t world, int32_t layout, int64_t* tiles, int64_t* cols, void* ws,
                                 size_t ws_bytes, void* stream) {
    RingInfo ri;
    msparse_status st = check_index_inputs(dims, v_idx, k_v, s_idx, k_s, nullptr, &ri);
    if (st) return st;
    if (!tiles || !cols) return fail(MSPARSE_ERR_INVALID, "workload outputs are NULL");
    if (world < 1 || world > kMaxRingWorld) return fail(MSPARSE_ERR_INVALID, "world %d outside [1, %d]", world, kMaxRingWorld);
    if (layout != MSPARSE_LAYOUT_STRIPED && layout != MSPARSE_LAYOUT_ZIGZAG)
        return fail(MSPARSE_ERR_INVALID, "ring layout %d", layout);
    const int32_t nb = dims->seq_q / kBlock;
    const int32_t unit = layout == MSPARSE_LAYOUT_ZIGZAG ? 2 * world : world;
    if (nb % unit != 0)
        return fail(MSPARSE_ERR_UNSUPPORTED, "%d blocks do not split into %d equal %s shards", nb, world,
                    layout == MSPARSE_LAYOUT_ZIGZAG ? "zigzag" : "striped");
    IndexPlan p = plan_index(dims, k_v, k_s, ri, ws, true);
    if (!ws || ws_bytes < p.bytes)
        return fail(MSPARSE_ERR_WORKSPACE, "index workspace %zu < %zu bytes", ws_bytes, p.bytes);
    p.a.v_idx = v_idx;
    p.a.s_idx = s_idx;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if ((st = check_hip(launch_index_prep(p.a, s), s, "index prep"))) return st;
    return check_hip(launch_ring_work(p.a, world, layout, tiles, cols, s), s, "ring work");
}

// ------------------------------------------------------------------ estimation
size_t msparse_estimate_workspace(const msparse_dims* dims, int32_t last_q, int32_t k_v, int32_t k_s) {
    (void)k_v;
    (void)k_s;
    if (check_dims(dims, true) || last_q < 1) return 0;
    const size_t scores = align_up(size_t(dims->batch) * dims->heads_q * dims->seq_q * sizeof(float));
    return 2 * scores + est_workspace_bytes(dims->batch, dims->heads_q, dims->heads_kv, dims->seq_q,
                                            dims->head_dim);
}

static msparse_status estimate_impl(const msparse_dims* dims, const void* q, const void* k, int32_t last_q, int32_t k_v,
                                    int32_t k_s, double p_v, double p_s, int32_t* v_idx, int32_t* s_idx, int32_t* v_cnt,
                                    int32_t* s_cnt, float* v_score, float* s_score, void* ws, size_t ws_bytes,
                                    void* stream) {
    msparse_status st = check_dims(dims, true);
    if (st) return st;
    const int32_t N = dims->seq_q;
    if (!q || !k || !v_idx || !s_idx) return fail(MSPARSE_ERR_INVALID, "tensor pointer is NULL");
    if (misaligned({q, k})) return fail(MSPARSE_ERR_INVALID, "tensor not 16-byte aligned");
    if (N < 1) return fail(MSPARSE_ERR_INVALID, "empty sequence");
    if (last_q < 1 || last_q > N) return fail(MSPARSE_ERR_INVALID, "last_q %d outside [1, %d]", last_q, N);
    if (last_q > kBlock) return fail(MSPARSE_ERR_UNSUPPORTED, "last_q %d > 64", last_q);
    if (k_v < 1 || k_v > N || k_s < 1 || k_s > N)
        return fail(MSPARSE_ERR_INVALID, "budgets k_v=%d k_s=%d outside [1, %d]", k_v, k_s, N);
    const size_t need = msparse_estimate_workspace(dims, last_q, k_v, k_s);
    if (!ws || ws_bytes < need) return fail(MSPARSE_ERR_WORKSPACE, "estimate workspace %zu < %zu", ws_bytes, need);
    EstArgs a{};
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.B = dims->batch;
    a.Hq = dims->heads_q;
    a.Hkv = dims->heads_kv;
    a.N = N;
    a.d = dims->head_dim;
    a.L = last_q;
    a.k_v = k_v;
    a.k_s = k_s;
    a.p_v = p_v;
    a.p_s = p_s;
    a.v_cnt = v_cnt;
    a.s_cnt = s_cnt;
    a.scale = resolve_scale(dims);
    a.v_idx = v_idx;
    a.s_idx = s_idx;
    char* base = static_cast<char*>(ws);
    const size_t scores = align_up(size_t(dims->batch) * dims->heads_q * N * sizeof(float));
    a.v_score = v_score ? v_score : reinterpret_cast<float*>(base);
    a.s_score = s_score ? s_score : reinterpret_cast<float*>(base + scores);
    est_carve(a, base + 2 * scores);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return check_hip(launch_estimate(a, s), s, "estimate");
}

msparse_status msparse_estimate(const msparse_dims* dims, const void* q, const void* k, int32_t last_q, int32_t k_v,
                                int32_t k_s, int32_t* v_idx, int32_t* s_idx, float* v_score, float* s_score, void* ws,
                                size_t ws_bytes, void* stream) {
    return estimate_impl(dims, q, k, last_q, k_v, k_s, 0.0, 0.0, v_idx, s_idx, nullptr, nullptr, v_score, s_score, ws,
                         ws_bytes, stream);
}

size_t msparse_estimate_topp_workspace(const msparse_dims* dims, int32_t last_q, int32_t kmax_v, int32_t kmax_s) {
    return msparse_estimate_workspace(dims, last_q, kmax_v, kmax_s);
}

msparse_status msparse_estimate_topp(const msparse_dims* dims, const void* q, const void* k, int32_t last_q, double p_v,
                                     double p_s, int32_t kmax_v, int32_t kmax_s, int32_t* v_idx, int32_t* s_idx,
                                     int32_t* v_cnt, int32_t* s_cnt, float* v_score, float* s_score, void* ws,
                                     size_t ws_bytes, void* stream) {
    if (!(p_v > 0.0 && p_v < 1.0) || !(p_s > 0.0 && p_s < 1.0))
        return fail(MSPARSE_ERR_INVALID, "top-p fractions p_v=%g p_s=%g outside (0, 1)", p_v, p_s);
    if (!v_cnt || !s_cnt) return fail(MSPARSE_ERR_INVALID, "budget output pointer is NULL");
    return estimate_impl(dims, q, k, last_q, kmax_v, kmax_s, p_v, p_s, v_idx, s_idx, v_cnt, s_cnt, v_score, s_score,
                         ws, ws_bytes, stream);
}

// ------------------------------------------------------------------ window attention
// A tensor argument: strides multiples of 8 elements (rows 16-byte aligned), and
// for an output no two rows in the same place.
static msparse_status check_tensor(const msparse_tensor* t, const char* name, int64_t batch, int64_t heads, int64_t rows,
                                   int32_t head_dim, bool output) {
    if (!t || !t->data) return fail(MSPARSE_ERR_INVALID, "%s is NULL", name);
    if (misaligned({t->data})) return fail(MSPARSE_ERR_INVALID, "%s is not 16-byte aligned", name);
    const int64_t size[3] = {batch, heads, rows}, stride[3] = {t->batch, t->head, t->token};
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int x, int y) { return stride[x] < stride[y]; });
    int64_t span = head_dim;   // elements that the axes so far take
    for (int x : order) {
        if (size[x] <= 1) continue;
        if (stride[x] < 0 || stride[x] % 8)
            return fail(MSPARSE_ERR_INVALID, "%s has stride %lld (multiples of 8, >= 0)", name, (long long)stride[x]);
        if (stride[x] > (int64_t(1) << 60) / size[x])
            return fail(MSPARSE_ERR_INVALID, "%s has stride %lld", name, (long long)stride[x]);
        if (output && stride[x] < span) return fail(MSPARSE_ERR_INVALID, "%s overlaps itself", name);
        span += (size[x] - 1) * stride[x];
    }
    return MSPARSE_OK;
}

static RowView row_view(const msparse_tensor* t) {
    return RowView{static_cast<uint16_t*>(t->data), t->batch, t->head, t->token};
}

// The most tokens that a sequence can have.
static int32_t longest(const msparse_window* w) {
    return w->tokens > 0 ? int32_t(std::min<int64_t>(w->seq, w->tokens)) : w->seq;
}

static msparse_status check_window(const msparse_window* w, const int32_t* starts) {
    if (!w) return fail(MSPARSE_ERR_INVALID, "window is NULL");
    if (w->batch < 1 || w->heads_q < 1 || w->heads_kv < 1 || w->seq < 0 || w->tokens < 0)
        return fail(MSPARSE_ERR_INVALID, "batch, heads must be >= 1 and lengths >= 0");
    if (w->heads_q % w->heads_kv != 0)
        return fail(MSPARSE_ERR_INVALID, "heads_q (%d) is not a multiple of heads_kv (%d)", w->heads_q, w->heads_kv);
    if (w->head_dim != 64 && w->head_dim != 128)
        return fail(MSPARSE_ERR_UNSUPPORTED, "head_dim %d (supported: 64, 128)", w->head_dim);
    if (w->window < 0 || w->sinks < 0) return fail(MSPARSE_ERR_INVALID, "window %d, sinks %d", w->window, w->sinks);
    if (!std::isfinite(w->scale)) return fail(MSPARSE_ERR_INVALID, "scale is not finite");
    if (w->tokens > 0 && !starts) return fail(MSPARSE_ERR_INVALID, "packed sequences without starts");
    if (w->tokens == 0 && starts) return fail(MSPARSE_ERR_INVALID, "starts without packed tokens");
    if (odd_words({starts})) return fail(MSPARSE_ERR_INVALID, "starts not 4-byte aligned");
    const int64_t rows = w->tokens > 0 ? w->tokens : int64_t(w->batch) * w->seq;
    if (rows > ((int64_t(1) << 31) - 1) / w->heads_q || w->seq > (1 << 30))
        return fail(MSPARSE_ERR_UNSUPPORTED, "heads * tokens exceeds 2^31 rows");
    const int32_t seq = longest(w);
    const bool by_rows = grid_by_rows(w->batch, w->heads_q, seq, w->tokens);
    if (grid_blocks(by_rows, w->batch, seq, w->tokens, 64) > kMaxGroups / w->heads_q)
        return fail(MSPARSE_ERR_UNSUPPORTED, "%d sequences of up to %d tokens%s exceed 2^22 blocks of 64 rows", w->batch,
                    seq, by_rows ? " (packed: their rows and one block each)" : "");
    return MSPARSE_OK;
}

static WindowArgs window_args(const msparse_window* w, const int32_t* starts) {
    WindowArgs a{};
    a.starts = starts;
    a.tokens = w->tokens;
    a.B = w->batch;
    a.Hq = w->heads_q;
    a.Hkv = w->heads_kv;
    a.seq = longest(w);
    a.d = w->head_dim;
    // a window or sinks over the whole sequence leave the causal mask alone
    const bool all = w->window == 0 || w->window >= a.seq || w->sinks >= a.seq;
    a.W = all ? INT32_MAX : w->window;
    a.S = all ? 0 : w->sinks;
    a.scale = w->scale > 0.f ? w->scale : 1.0f / std::sqrt(float(w->head_dim));
    a.by_rows = grid_by_rows(w->batch, w->heads_q, a.seq, w->tokens);
    return a;
}

// lse log2(e) and Delta of every row, the keys' partial gradients.
static size_t carve_window_bwd(WindowArgs* a, char* base) {
    const int keys = window_key_group(a->d);
    const KeyPlan& p = a->plan = key_plan(a->B, a->Hkv, a->Hq / a->Hkv, a->seq, a->tokens, a->W, a->S, a->d, keys,
                                          window_key_resident(a->d), a->by_rows);
    const int64_t near = (a->by_rows ? p.far_docs : a->B) * int64_t(p.part_groups) * p.near_slots;
    const int64_t far = (a->by_rows ? 1 : a->B) * int64_t(p.sink_groups) * p.far_slots;
    a->rows_pad = a->tokens > 0 ? padded_rows(a->tokens) + 64 * (int64_t(a->B) + 1) : a->B * padded_rows(a->seq);
    Carve c{base};
    a->rows = c.take<float>(size_t(2) * a->Hq * a->rows_pad);
    a->part = c.take<float>(size_t(a->Hkv) * (near + far) * 2 * keys * a->d);
    return c.off;
}

// The key-major pass has the sink groups' chunks beside all groups: 512 threads each, below 2^32 together.
static msparse_status check_window_keys(const WindowArgs& a) {
    const KeyPlan& p = a.plan;
    const int keys = window_key_group(a.d);
    const int64_t each = (a.by_rows ? 1 : a.B) * int64_t(p.sink_groups) * p.far_slots +
                         grid_blocks(a.by_rows, a.B, a.seq, a.tokens, keys) * p.near_slots;
    if (each >= 2 * kMaxGroups / a.Hkv)
        return fail(MSPARSE_ERR_UNSUPPORTED, "%lld workgroups of keys exceed 2^23", (long long)(each * a.Hkv));
    return MSPARSE_OK;
}

msparse_status msparse_window_fwd(const msparse_window* win, const int32_t* starts, const msparse_tensor* q,
                                  const msparse_tensor* k, const msparse_tensor* v, const msparse_tensor* out,
                                  float* lse, void* stream) {
    msparse_status st = check_window(win, starts);
    if (st || win->seq == 0) return st;
    const int64_t B = win->tokens > 0 ? 1 : win->batch, N = win->tokens > 0 ? win->tokens : win->seq;
    const int32_t d = win->head_dim;
    if ((st = check_tensor(q, "q", B, win->heads_q, N, d, false))) return st;
    if ((st = check_tensor(k, "k", B, win->heads_kv, N, d, false))) return st;
    if ((st = check_tensor(v, "v", B, win->heads_kv, N, d, false))) return st;
    if ((st = check_tensor(out, "out", B, win->heads_q, N, d, true))) return st;
    if (!lse) return fail(MSPARSE_ERR_INVALID, "lse is NULL");
    if (misaligned({lse})) return fail(MSPARSE_ERR_INVALID, "lse is not 16-byte aligned");
    WindowArgs a = window_args(win, starts);
    a.q = row_view(q);
    a.k = row_view(k);
    a.v = row_view(v);
    a.out = row_view(out);
    a.lse = lse;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return check_hip(launch_window_fwd(a, s), s, "window fwd");
}

size_t msparse_window_bwd_workspace(const msparse_window* win) {
    static const int32_t present = 0;   // only whether starts are given counts
    if (check_window(win, win && win->tokens > 0 ? &present : nullptr)) return 0;
    WindowArgs a = window_args(win, nullptr);
    const size_t need = carve_window_bwd(&a, nullptr);
    return check_window_keys(a) ? 0 : need;
}

msparse_status msparse_window_bwd(const msparse_window* win, const int32_t* starts, const msparse_tensor* q,
                                  const msparse_tensor* k, const msparse_tensor* v, const msparse_tensor* out,
                                  const msparse_tensor* dout, const float* lse, const msparse_tensor* dq,
                                  const msparse_tensor* dk, const msparse_tensor* dv, void* ws, size_t ws_bytes,
                                  void* stream) {
    msparse_status st = check_window(win, starts);
    if (st || win->seq == 0) return st;
    const int64_t B = win->tokens > 0 ? 1 : win->batch, N = win->tokens > 0 ? win->tokens : win->seq;
    const int32_t d = win->head_dim;
    if ((st = check_tensor(q, "q", B, win->heads_q, N, d, false))) return st;
    if ((st = check_tensor(k, "k", B, win->heads_kv, N, d, false))) return st;
    if ((st = check_tensor(v, "v", B, win->heads_kv, N, d, false))) return st;
    if ((st = check_tensor(out, "out", B, win->heads_q, N, d, false))) return st;
    if ((st = check_tensor(dout, "dout", B, win->heads_q, N, d, false))) return st;
    if ((st = check_tensor(dq, "dq", B, win->heads_q, N, d, true))) return st;
    if ((st = check_tensor(dk, "dk", B, win->heads_kv, N, d, true))) return st;
    if ((st = check_tensor(dv, "dv", B, win->heads_kv, N, d, true))) return st;
    if (!lse) return fail(MSPARSE_ERR_INVALID, "lse is NULL");
    if (misaligned({lse, ws})) return fail(MSPARSE_ERR_INVALID, "lse or workspace is not 16-byte aligned");
    WindowArgs a = window_args(win, starts);
    const size_t need = carve_window_bwd(&a, static_cast<char*>(ws));
    if ((st = check_window_keys(a))) return st;
    if (need && (!ws || ws_bytes < need))
        return fail(MSPARSE_ERR_WORKSPACE, "window bwd workspace %zu < %zu bytes", ws_bytes, need);
    a.q = row_view(q);
    a.k = row_view(k);
    a.v = row_view(v);
    a.out = row_view(out);
    a.dout = row_view(dout);
    a.lse = const_cast<float*>(lse);
    a.dq = row_view(dq);
    a.dk = row_view(dk);
    a.dv = row_view(dv);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return check_hip(launch_window_bwd(a, s), s, "window bwd");
}

// ------------------------------------------------------------------ paged cache
static msparse_status check_cache(const msparse_cache* c, int32_t heads_q, int32_t tokens) {
    if (!c) return fail(MSPARSE_ERR_INVALID, "cache is NULL");
    if (c->batch < 1 || c->heads_kv < 1 || heads_q < 1 || tokens < 0)
        return fail(MSPARSE_ERR_INVALID, "batch, heads must be >= 1 and tokens >= 0");
    if (heads_q % c->heads_kv != 0)
        return fail(MSPARSE_ERR_INVALID, "heads_q (%d) is not a multiple of heads_kv (%d)", heads_q, c->heads_kv);
    if (c->head_dim != 64 && c->head_dim != 128)
        return fail(MSPARSE_ERR_UNSUPPORTED, "head_dim %d (supported: 64, 128)", c->head_dim);
    if (c->pages < 1 || c->width < 1) return fail(MSPARSE_ERR_INVALID, "pages %d, width %d", c->pages, c->width);
    if (c->width > kMaxWidth) return fail(MSPARSE_ERR_UNSUPPORTED, "width %d > 2^24", c->width);
    if (tokens > (1 << 30) || int64_t(c->batch) * tokens > ((int64_t(1) << 31) - 1) / heads_q)
        return fail(MSPARSE_ERR_UNSUPPORTED, "batch * heads * tokens exceeds 2^31 rows");
    return MSPARSE_OK;
}
static msparse_status check_cache_memory(const msparse_cache* c) {
    if (!c->k || !c->v || !c->k_scale || !c->v_scale || !c->page_table || !c->lens)
        return fail(MSPARSE_ERR_INVALID, "cache array is NULL");
    if (misaligned({c->k, c->v})) return fail(MSPARSE_ERR_INVALID, "cache codes not 16-byte aligned");
    if (odd_words({c->k_scale, c->v_scale, c->page_table, c->lens}))
        return fail(MSPARSE_ERR_INVALID, "cache array not 4-byte aligned");
    return MSPARSE_OK;
}
static CacheView cache_view(const msparse_cache* c) {
    return CacheView{static_cast<uint8_t*>(c->k), static_cast<uint8_t*>(c->v), c->k_scale, c->v_scale, c->page_table,
                     c->lens, c->pages, c->width, c->batch, c->heads_kv, c->head_dim};
}
static void set_strides(int64_t* s, const msparse_tensor* t) {
    s[0] = t->batch;
    s[1] = t->head;
    s[2] = t->token;
}

// A rotation's output in its input's place has its strides.
static msparse_status check_in_place(const msparse_tensor* x, const msparse_tensor* y, const char* name, int64_t batch,
                                     int64_t heads, int64_t tokens) {
    const bool same = (batch <= 1 || x->batch == y->batch) && (heads <= 1 || x->head == y->head) &&
                      (tokens <= 1 || x->token == y->token);
    if (x->data == y->data && !same) return fail(MSPARSE_ERR_INVALID, "%s rotated in place with other strides", name);
    return MSPARSE_OK;
}

static msparse_status check_positions(const msparse_positions* p) {
    if (!p || !p->at || !p->inv_freq) return fail(MSPARSE_ERR_INVALID, "positions or inv_freq NULL");
    if (p->axes < 1 || p->axes > kMaxAxes) return fail(MSPARSE_ERR_INVALID, "%d axes (1 to %d)", p->axes, kMaxAxes);
    if (odd_words({p->at, p->axis, p->inv_freq}))
        return fail(MSPARSE_ERR_INVALID, "positions, axis or inv_freq not 4-byte aligned");
    return MSPARSE_OK;
}
static Positions positions_of(const msparse_positions* p, int64_t batch, int64_t tokens) {
    return Positions{p->at, p->axis, p->inv_freq, p->axes, batch * tokens};
}

static msparse_status append_impl(const msparse_cache* cache, int32_t heads_q, int32_t tokens, const msparse_tensor* q,
                                  const msparse_tensor* k, const msparse_tensor* v, const msparse_tensor* q_out,
                                  const float* inv_freq, const msparse_positions* pos, const int32_t* counts,
                                  void* stream) {
    msparse_status st = check_cache(cache, heads_q, tokens);
    if (st) return st;
    if ((st = check_cache_memory(cache)) || tokens == 0) return st;
    const int64_t B = cache->batch;
    const int32_t d = cache->head_dim;
    if ((st = check_tensor(k, "k", B, cache->heads_kv, tokens, d, false))) return st;
    if ((st = check_tensor(v, "v", B, cache->heads_kv, tokens, d, false))) return st;
    if (odd_words({inv_freq, counts})) return fail(MSPARSE_ERR_INVALID, "inv_freq or counts not 4-byte aligned");
    if (!q != !q_out) return fail(MSPARSE_ERR_INVALID, "q and q_out go together");
    if (q) {
        if ((st = check_tensor(q, "q", B, heads_q, tokens, d, false))) return st;
        if ((st = check_tensor(q_out, "q_out", B, heads_q, tokens, d, true))) return st;
        if ((st = check_in_place(q, q_out, "q", B, heads_q, tokens))) return st;
    }
    if (pos && (st = check_positions(pos))) return st;
    AppendArgs a{};
    a.c = cache_view(cache);
    a.k = static_cast<const uint16_t*>(k->data);
    a.v = static_cast<const uint16_t*>(v->data);
    set_strides(a.ks, k);
    set_strides(a.vs, v);
    if (q) {
        a.q = static_cast<const uint16_t*>(q->data);
        a.qout = static_cast<uint16_t*>(q_out->data);
        set_strides(a.qs, q);
        set_strides(a.qos, q_out);
    }
    a.freq = inv_freq;
    if (pos) a.pos = positions_of(pos, B, tokens);
    a.counts = counts;
    a.Hq = heads_q;
    a.T = tokens;
    const int64_t P = (int64_t(tokens) + 2 * kPage - 2) / kPage;   // the most pages that tokens in a row touch
    if (B * P > kMaxGroups / 2) return fail(MSPARSE_ERR_UNSUPPORTED, "%lld pages in one call", (long long)(B * P));
    a.P = int32_t(P);
    share_heads(a, B * P);
    if (B * P > 2 * kMaxGroups / (a.kv_shares + a.q_shares))   // (of 256 threads)
        return fail(MSPARSE_ERR_UNSUPPORTED, "%lld pages of %d heads in one call", (long long)(B * P), heads_q);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return check_hip(launch_cache_append(a, s), s, "cache append");
}

msparse_status msparse_cache_append(const msparse_cache* cache, int32_t heads_q, int32_t tokens, const msparse_tensor* q,
                                    const msparse_tensor* k, const msparse_tensor* v, const msparse_tensor* q_out,
                                    const float* inv_freq, const int32_t* counts, void* stream) {
    return append_impl(cache, heads_q, tokens, q, k, v, q_out, inv_freq, nullptr, counts, stream);
}

msparse_status msparse_cache_append_at(const msparse_cache* cache, int32_t heads_q, int32_t tokens,
                                       const msparse_tensor* q, const msparse_tensor* k, const msparse_tensor* v,
                                       const msparse_tensor* q_out, const msparse_positions* positions,
                                       const int32_t* counts, void* stream) {
    if (!positions) return fail(MSPARSE_ERR_INVALID, "positions are NULL");
    return append_impl(cache, heads_q, tokens, q, k, v, q_out, nullptr, positions, counts, stream);
}

msparse_status msparse_rotate(int32_t batch, int32_t tokens, int32_t heads_q, int32_t heads_kv, int32_t head_dim,
                              int32_t type, const msparse_positions* positions, int32_t inverse,
                              const msparse_tensor* q, const msparse_tensor* k, const msparse_tensor* q_out,
                              const msparse_tensor* k_out, void* stream) {
    if (batch < 1 || heads_q < 1 || heads_kv < 0 || tokens < 0)
        return fail(MSPARSE_ERR_INVALID, "batch, heads_q must be >= 1, heads_kv and tokens >= 0");
    if (head_dim != 64 && head_dim != 128)
        return fail(MSPARSE_ERR_UNSUPPORTED, "head_dim %d (supported: 64, 128)", head_dim);
    if (type != MSPARSE_BF16 && type != MSPARSE_F32) return fail(MSPARSE_ERR_INVALID, "type %d", type);
    const int64_t heads = int64_t(heads_q) + heads_kv;
    if (tokens > (1 << 30) || int64_t(batch) * tokens > ((int64_t(1) << 31) - 1) / heads)
        return fail(MSPARSE_ERR_UNSUPPORTED, "batch * heads * tokens exceeds 2^31 rows");
    if (tokens == 0) return MSPARSE_OK;
    msparse_status st = check_positions(positions);
    if (st) return st;
    if (heads_kv == 0 ? k || k_out : !k || !k_out)
        return fail(MSPARSE_ERR_INVALID, "k and k_out go with heads_kv (%d)", heads_kv);
    RotateArgs a{};
    if ((st = check_tensor(q, "q", batch, heads_q, tokens, head_dim, false))) return st;
    if ((st = check_tensor(q_out, "q_out", batch, heads_q, tokens, head_dim, true))) return st;
    if ((st = check_in_place(q, q_out, "q", batch, heads_q, tokens))) return st;
    a.q = q->data;
    a.qout = q_out->data;
    set_strides(a.qs, q);
    set_strides(a.qos, q_out);
    if (k) {
        if ((st = check_tensor(k, "k", batch, heads_kv, tokens, head_dim, false))) return st;
        if ((st = check_tensor(k_out, "k_out", batch, heads_kv, tokens, head_dim, true))) return st;
        if ((st = check_in_place(k, k_out, "k", batch, heads_kv, tokens))) return st;
        a.k = k->data;
        a.kout = k_out->data;
        set_strides(a.ks, k);
        set_strides(a.kos, k_out);
    }
    a.pos = positions_of(positions, batch, tokens);
    a.B = batch;
    a.T = tokens;
    a.Hq = heads_q;
    a.Hkv = heads_kv;
    a.d = head_dim;
    a.inverse = inverse != 0;
    a.f32 = type == MSPARSE_F32;
    a.blocks = (tokens + kRotateTokens - 1) / kRotateTokens;
    share_heads(a);
    if (int64_t(batch) * a.blocks > 2 * kMaxGroups / a.shares)   // (of 256 threads)
        return fail(MSPARSE_ERR_UNSUPPORTED, "%lld blocks of tokens in one call", (long long)batch * a.blocks);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return check_hip(launch_rotate(a, s), s, "rotate");
}

static msparse_status check_nodes(int32_t tokens) {
    if (tokens > kMaxNodes) return fail(MSPARSE_ERR_UNSUPPORTED, "trees of %d nodes (up to %d)", tokens, kMaxNodes);
    return MSPARSE_OK;
}

static size_t carve_cache_attn(const msparse_cache* c, const CacheAttnPlan& p, char* base, CacheAttnArgs* a) {
    if (p.slots == 0) return 0;
    Carve w{base};
    a->info = w.take<int32_t>(size_t(2) * c->batch * p.tiles);
    a->pml = w.take<float>(size_t(p.slots) * c->heads_kv * p.rows * 2);
    a->po = w.take<float>(size_t(p.slots) * c->heads_kv * p.rows * c->head_dim);
    return w.off;
}

size_t msparse_cache_attn_workspace(const msparse_cache* cache, int32_t heads_q, int32_t tokens) {
    if (check_cache(cache, heads_q, tokens) || tokens == 0) return 0;
    CacheAttnArgs a{};
    const CacheAttnPlan p = cache_attn_plan(cache->batch, heads_q, cache->heads_kv, tokens, cache->width,
                                            cache->head_dim, INT32_MAX, 0);
    return carve_cache_attn(cache, p, nullptr, &a);
}

size_t msparse_cache_tree_attn_workspace(const msparse_cache* cache, int32_t heads_q, int32_t tokens) {
    if (check_cache(cache, heads_q, tokens) || check_nodes(tokens) || tokens == 0) return 0;
    CacheAttnArgs a{};
    const CacheAttnPlan p = cache_attn_plan(cache->batch, heads_q, cache->heads_kv, tokens, cache->width,
                                            cache->head_dim, INT32_MAX, 0, true);
    return carve_cache_attn(cache, p, nullptr, &a);
}

// tree: NULL, or the tree's part of the arguments (seen, at, counts)
static msparse_status attn_impl(const msparse_cache* cache, int32_t heads_q, int32_t tokens, int32_t window,
                                int32_t sinks, float scale, const msparse_tensor* q, const msparse_tensor* out,
                                float* lse, const CacheAttnArgs* tree, void* ws, size_t ws_bytes, void* stream) {
    msparse_status st = check_cache(cache, heads_q, tokens);
    if (st || (tree && (st = check_nodes(tokens)))) return st;
    if ((st = check_cache_memory(cache)) || tokens == 0) return st;
    if (window < 0 || sinks < 0) return fail(MSPARSE_ERR_INVALID, "window %d, sinks %d", window, sinks);
    if (!std::isfinite(scale)) return fail(MSPARSE_ERR_INVALID, "scale is not finite");
    const int64_t B = cache->batch;
    const int32_t d = cache->head_dim;
    if ((st = check_tensor(q, "q", B, heads_q, tokens, d, false))) return st;
    if ((st = check_tensor(out, "out", B, heads_q, tokens, d, true))) return st;
    if (misaligned({lse, ws})) return fail(MSPARSE_ERR_INVALID, "lse or workspace is not 16-byte aligned");
    const CacheAttnPlan p = cache_attn_plan(B, heads_q, cache->heads_kv, tokens, cache->width, d,
                                            window == 0 ? INT32_MAX : window, window == 0 ? 0 : sinks, tree != nullptr);
    if (cache_attn_groups(p, B) > kMaxGroups / cache->heads_kv)
        return fail(MSPARSE_ERR_UNSUPPORTED, "%lld row tiles of %d heads", (long long)(B * p.tiles), cache->heads_kv);
    if (tree) {
        if (!tree->seen) return fail(MSPARSE_ERR_INVALID, "seen is NULL");
        if (window > 0 && !tree->at) return fail(MSPARSE_ERR_INVALID, "a window without positions");
        if (odd_words({tree->seen, tree->at, tree->counts}))
            return fail(MSPARSE_ERR_INVALID, "seen, positions or counts not 4-byte aligned");
    }
    CacheAttnArgs a = tree ? *tree : CacheAttnArgs{};
    const size_t need = carve_cache_attn(cache, p, static_cast<char*>(ws), &a);
    if (need && (!ws || ws_bytes < need))
        return fail(MSPARSE_ERR_WORKSPACE, "cache attn workspace %zu < %zu bytes", ws_bytes, need);
    a.c = cache_view(cache);
    a.q = static_cast<const uint16_t*>(q->data);
    a.out = static_cast<uint16_t*>(out->data);
    set_strides(a.qs, q);
    set_strides(a.os, out);
    a.lse = lse;
    a.Hq = heads_q;
    a.T = tokens;
    a.W = window == 0 ? INT32_MAX : window;
    a.S = window == 0 ? 0 : sinks;
    a.scale = scale > 0.f ? scale : 1.0f / std::sqrt(float(d));
    a.tiles = p.tiles;
    a.items = p.items;
    a.chunk = p.chunk;
    a.per_tile = p.per_tile;
    a.unit = p.unit;
    a.slots = p.slots;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return check_hip(launch_cache_attn(a, p, s), s, "cache attn");
}

msparse_status msparse_cache_attn(const msparse_cache* cache, int32_t heads_q, int32_t tokens, int32_t window,
                                  int32_t sinks, float scale, const msparse_tensor* q, const msparse_tensor* out,
                                  float* lse, void* ws, size_t ws_bytes, void* stream) {
    return attn_impl(cache, heads_q, tokens, window, sinks, scale, q, out, lse, nullptr, ws, ws_bytes, stream);
}

msparse_status msparse_cache_tree_attn(const msparse_cache* cache, int32_t heads_q, int32_t tokens, int32_t window,
                                       int32_t sinks, float scale, const msparse_tensor* q, const int32_t* seen,
                                       const int32_t* positions, const int32_t* counts, const msparse_tensor* out,
                                       float* lse, void* ws, size_t ws_bytes, void* stream) {
    CacheAttnArgs tree{};
    tree.seen = seen;
    tree.at = window > 0 ? positions : nullptr;
    tree.counts = counts;
    tree.words = (tokens + 31) / 32;
    return attn_impl(cache, heads_q, tokens, window, sinks, scale, q, out, lse, &tree, ws, ws_bytes, stream);
}

// ------------------------------------------------------------------ drafted trees, pages
msparse_status msparse_tree_mask(int32_t batch, int32_t tokens, const int32_t* parents, const int32_t* lens,
                                 const int32_t* counts, int32_t window, int32_t sinks, int32_t* positions, int32_t* seen,
                                 void* stream) {
    if (batch < 1 || tokens < 0) return fail(MSPARSE_ERR_INVALID, "batch must be >= 1 and tokens >= 0");
    msparse_status st = check_nodes(tokens);
    if (st) return st;
    if (batch > kMaxGroups) return fail(MSPARSE_ERR_UNSUPPORTED, "%d trees exceed 2^22", batch);
    if (window < 0 || sinks < 0) return fail(MSPARSE_ERR_INVALID, "window %d, sinks %d", window, sinks);
    if (tokens == 0) return MSPARSE_OK;
    if (!parents || !lens || !positions || !seen) return fail(MSPARSE_ERR_INVALID, "tree array is NULL");
    if (odd_words({parents, lens, counts, positions, seen}))
        return fail(MSPARSE_ERR_INVALID, "tree array not 4-byte aligned");
    const TreeMaskArgs a{parents, lens,   counts, positions, seen, batch, tokens, (tokens + 31) / 32,
                         window == 0 ? INT32_MAX : window, window == 0 ? 0 : sinks};
    hipStream_t s = static_cast<hipStream_t>(stream);
    return check_hip(launch_tree_mask(a, s), s, "tree mask");
}

msparse_status msparse_cache_keep(const msparse_cache* cache, int32_t tokens, const int32_t* path, const int32_t* kept,
                                  const int32_t* counts, void* stream) {
    msparse_status st = check_cache(cache, cache ? cache->heads_kv : 1, tokens);
    if (st) return st;
    if ((st = check_cache_memory(cache)) || tokens == 0) return st;
    if (!path || !kept) return fail(MSPARSE_ERR_INVALID, "path or kept is NULL");
    if (odd_words({path, kept, counts})) return fail(MSPARSE_ERR_INVALID, "path, kept or counts not 4-byte aligned");
    if (cache->batch > kMaxGroups / cache->heads_kv)
        return fail(MSPARSE_ERR_UNSUPPORTED, "%d sequences of %d heads", cache->batch, cache->heads_kv);
    KeepArgs a{};
    a.c = cache_view(cache);
    a.counts = counts;
    a.path = path;
    a.kept = kept;
    a.T = tokens;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return check_hip(launch_cache_keep(a, s), s, "cache keep");
}

static msparse_status check_fork(const msparse_cache* c, int32_t sequences) {
    msparse_status st = check_cache(c, c ? c->heads_kv : 1, 1);
    if (st) return st;
    if (sequences < 1) return fail(MSPARSE_ERR_INVALID, "%d sequences", sequences);
    if (sequences > kMaxForks || c->batch > kMaxForks)
        return fail(MSPARSE_ERR_UNSUPPORTED, "more than %d sequences", kMaxForks);
    return MSPARSE_OK;
}
static size_t carve_cache_fork(const msparse_cache* c, int32_t sequences, char* base, ForkArgs* a) {
    Carve w{base};
    a->cap = int32_t(std::min(int64_t(sequences) * c->width, int64_t(c->pages)));
    a->need = w.take<int32_t>(size_t(sequences));
    a->list = w.take<int32_t>(std::max(size_t(1) + a->cap, size_t(c->pages)));   // (or a copy of the counts)
    return w.off;
}

// What a fork writes shares no memory with what it reads (some workgroups read while others write), nor with each other;
// the counts alone may be updated in their place.
static msparse_status check_fork_memory(const msparse_cache* c, int32_t sequences, const int32_t* src,
                                        const int32_t* room, const int32_t* refs, const int32_t* refs_out,
                                        const int32_t* table_out, const int32_t* lens_out, const int32_t* missing,
                                        const void* ws, size_t ws_bytes) {
    struct Range {
        const char* name;
        const void* at;
        uint64_t bytes;
    };
    const uint64_t old = uint64_t(c->batch), n = uint64_t(sequences), width = uint64_t(c->width);
    const Range written[] = {{"refs_out", refs_out, 4 * uint64_t(c->pages)}, {"page_table_out", table_out, 4 * n * width},
                             {"lens_out", lens_out, 4 * n}, {"missing", missing, 4 * n}, {"workspace", ws, ws_bytes}};
    const Range read[] = {{"refs", refs, 4 * uint64_t(c->pages)}, {"page_table", c->page_table, 4 * old * width},
                          {"lens", c->lens, 4 * old}, {"src", src, 4 * n}, {"room", room, room ? 4 * n : 0}};
    auto share = [](const Range& x, const Range& y) {
        const uint64_t a = reinterpret_cast<uintptr_t>(x.at), b = reinterpret_cast<uintptr_t>(y.at);
        return a < b + y.bytes && b < a + x.bytes;
    };
    for (const Range& w : written) {
        for (const Range& r : read)
            if (share(w, r) && !(&w == written && &r == read && refs == refs_out))   // (the counts in their place)
                return fail(MSPARSE_ERR_INVALID, "%s and %s share memory", w.name, r.name);
        for (const Range* x = written; x < &w; ++x)
            if (share(w, *x)) return fail(MSPARSE_ERR_INVALID, "%s and %s share memory", w.name, x->name);
    }
    return MSPARSE_OK;
}

size_t msparse_cache_fork_workspace(const msparse_cache* cache, int32_t sequences) {
    if (check_fork(cache, sequences)) return 0;
    ForkArgs a{};
    return carve_cache_fork(cache, sequences, nullptr, &a);
}

msparse_status msparse_cache_fork(const msparse_cache* cache, int32_t sequences, const int32_t* src, const int32_t* room,
                                  const int32_t* refs, int32_t* refs_out, int32_t* table_out, int32_t* lens_out,
                                  int32_t* missing, void* ws, size_t ws_bytes, void* stream) {
    msparse_status st = check_fork(cache, sequences);
    if (st) return st;
    if ((st = check_cache_memory(cache))) return st;
    if (!src || !refs || !refs_out || !table_out || !lens_out || !missing)
        return fail(MSPARSE_ERR_INVALID, "fork array is NULL");
    if (odd_words({src, room, refs, refs_out, table_out, lens_out, missing}))
        return fail(MSPARSE_ERR_INVALID, "fork array not 4-byte aligned");
    if (misaligned({ws})) return fail(MSPARSE_ERR_INVALID, "workspace is not 16-byte aligned");
    ForkArgs a{};
    const size_t need = carve_cache_fork(cache, sequences, static_cast<char*>(ws), &a);
    if (!ws || ws_bytes < need) return fail(MSPARSE_ERR_WORKSPACE, "cache fork workspace %zu < %zu bytes", ws_bytes, need);
    if ((st = check_fork_memory(cache, sequences, src, room, refs, refs_out, table_out, lens_out, missing, ws, need)))
        return st;
    a.c = cache_view(cache);
    a.refs = refs;
    a.src = src;
    a.room = room;
    a.refs_out = refs_out;
    a.table_out = table_out;
    a.lens_out = lens_out;
    a.missing = missing;
    a.N = sequences;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return check_hip(launch_cache_fork(a, s), s, "cache fork");
}

}  // extern "C"
