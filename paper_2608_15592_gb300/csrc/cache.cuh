// The paged KV cache as the kernels see it, and the cut of an attention call into units.
//
// A call's units are (sequence b, KV head g, block of RB rows, tile of 128 keys), a tile of a block of
// more than 128 rows counted twice (it costs twice).  The rows of
// (b, g) are its n_b drafts times the rep query heads that read KV head g, row r = i rep + h';
// the tiles are the cached slots in order and, last, one tile of the drafts themselves.  Units
// are numbered with the tile fastest, then the row block, the KV head and the sequence; the
// CTAs of a persistent grid take equal ranges of them, so that every CTA reads as many bytes
// whatever the lengths.  Consecutive units of one (b, g, row block), a group, share a running
// softmax; a group that several CTAs hold leaves one partial a CTA, in slot CTA + group (both
// only grow along the unit axis, so every (CTA, group) pair that meets has a slot of its own).
#pragma once

#include "estp_internal.cuh"

namespace estp {

constexpr int kCacheTile = 128;     // keys of a tile
constexpr int kCacheMaxRows = 128;  // drafts of a sequence (one tile holds them)
constexpr int kCacheMaxGroupRows = 1024;  // drafts times query heads of a KV head

struct CacheView {
    char* k;
    char* v;
    float* weight;      // [n_pages, Hkv, page]
    int32_t* position;  // [n_pages, Hkv, page]
    const int32_t* table;
    int64_t page_stride, slot_stride, head_stride;  // bytes
    int64_t n_pages;
    int ld_table;
    int shift;          // log2 of the page size
    int Hkv, d;

    __host__ __device__ __forceinline__ int64_t capacity() const { return (int64_t)ld_table << shift; }
    // byte offset of a slot's row of KV head g, element offset of its weight and position
    __device__ __forceinline__ int64_t row(int64_t page, int slot, int g) const {
        return page * page_stride + (slot & ((1 << shift) - 1)) * slot_stride + g * head_stride;
    }
    __device__ __forceinline__ int64_t meta(int64_t page, int slot, int g) const {
        return ((page * Hkv + g) << shift) + (slot & ((1 << shift) - 1));
    }
    // bounds of the checked build: a slot's place in the pool
    __device__ __forceinline__ bool inside(int64_t page, int slot, int g, int* status) const {
        return in_bounds(page >= 0 && page < n_pages && slot >= 0 && slot < capacity() && g >= 0 && g < Hkv, status);
    }
    // page of a slot of sequence b; -1 (reported) when the table holds no page of the pool there
    __device__ __forceinline__ int64_t page_of(int b, int slot, int* status) const {
        const int p = table[(int64_t)b * ld_table + (slot >> shift)];
        if (p >= 0 && p < n_pages) return p;
        report(status, ESTP_ERR_INVALID_ARG);
        return -1;
    }
};

struct CacheAttnArgs {
    CacheView c;
    const int32_t* length;
    const int32_t* cu;
    int B;
    int64_t n_rows, n_slots;
    int max_rows, Hq, rep;
    const char* Q;
    const char* kn;              // NULL: rows see cached slots only
    const char* vn;
    int64_t ldq, ldn;            // bytes
    const uint64_t* tree;        // NULL: draft i sees drafts j <= i
    int words;
    const float* row_weight;
    float scale, scale_log2;
    int RB, G;
    int whole;                   // the forward finishes the groups that one CTA holds by itself
    int row_blocks;              // blocks of the finish kernel that merge rows, warps of one of them
    int row_warps;
    int store;                   // scores are kept for the weights
    int64_t n_parts, n_units;    // bounds of the slots of partials, of the units
    float* part_o;               // [n_parts][RB][d]
    float2* part_ml;             // [n_parts][RB]: running max (log2 units) and sum
    float* score;                // [n_units][RB][128], unscaled
    float2* factor;              // [n_rows, Hq]: (-M, c / L), where the weights are wanted
    char* out;
    float* lse;
    float* w_new;
    int accumulate;
    int* status;
    volatile int* timed_out;     // a kernel of the attention gave up: the weights stay as they are
    long long wait_cycles;
    // bounds of the checked build: the slots of n partials from one on, a unit, rows of the call
    __device__ __forceinline__ bool part_inside(int64_t slot, int n = 1) const {
        return in_bounds(slot >= 0 && n >= 1 && slot + n <= n_parts, status);
    }
    __device__ __forceinline__ bool unit_inside(int64_t u) const { return in_bounds(u >= 0 && u < n_units, status); }
    __device__ __forceinline__ bool row_inside(int64_t row, int n = 1) const {
        return in_bounds(row >= 0 && n >= 1 && row + n <= n_rows, status);
    }
};

// What sequence b brings to the call.
struct SeqShape {
    int len, n, nrb, nt;
    int cost, last;  // units of a tile: of a KV head's blocks together, and of its last block
    // the host has made sure that the call's units fit 31 bits
    __device__ __forceinline__ int groups(int Hkv) const { return Hkv * nrb; }
    __device__ __forceinline__ int units(int Hkv) const { return Hkv * cost * nt; }
    __device__ __forceinline__ int items(int Hkv) const { return n > 0 ? Hkv * nt : 0; }
};
__device__ __forceinline__ bool seq_ok(const CacheAttnArgs& a, int b) {
    const int len = a.length[b], lo = a.cu[b], hi = a.cu[b + 1];
    return len >= 0 && len <= a.c.capacity() && lo >= 0 && hi >= lo && hi - lo <= a.max_rows && hi <= a.n_rows &&
           (b > 0 || lo == 0) && (b + 1 < a.B || hi == a.n_rows);
}
// kRB: the rows of a block where the kernel knows them (0: a.RB), which leaves little of the divisions
template <int kRB = 0>
__device__ __forceinline__ SeqShape seq_shape(const CacheAttnArgs& a, int b) {
    const int RB = kRB != 0 ? kRB : a.RB;
    SeqShape s;
    s.len = a.length[b];
    s.n = a.cu[b + 1] - a.cu[b];
    s.nrb = (s.n * a.rep + RB - 1) / RB;
    s.nt = (s.len + kCacheTile - 1) / kCacheTile + 1;
    s.last = s.n * a.rep - (s.nrb - 1) * RB > 128 ? 2 : 1;
    s.cost = RB <= 128 ? s.nrb : s.nrb > 0 ? (s.nrb - 1) * 2 + s.last : 0;
    return s;
}

// Sums over the sequences before sequence b.
struct Place {
    int b;
    int unit0, group0, item0;  // units, groups, items (KV head, tile) before it
    __device__ __forceinline__ void pass(const SeqShape& s, int Hkv) {
        ++b;
        unit0 += s.units(Hkv);
        group0 += s.groups(Hkv);
        item0 += s.items(Hkv);
    }
};
struct PlanTotals {
    int units, groups, items;
    bool ok;                   // lengths, cu and their sums are what the host was told
};
struct PlanScratch {
    int sum[3][33];            // units, groups, items
    int64_t slots[32];
    Place place;
    int bad;
};

__device__ __forceinline__ int scan_lanes(int x, int lane) {  // inclusive
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    return x;
}

// Launches.  Every kernel of the cache may begin before the one ahead of it in the stream has ended
// (launch_dependent).  The first kernel of a call waits for that one (await_stream) before it touches
// anything, and only after its wait lets the next begin (admit_next).  So when a later kernel of the call
// begins, everything ahead of the call is over: it may read the call's inputs, such as the lengths, and
// admit its own successor before its wait, but nothing that the call's kernels write, and it waits before
// it ends.
__device__ __forceinline__ void await_stream() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void admit_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// The call's totals, and the place of the one sequence that want(place, shape, totals) picks (b = B
// where it picks none).  Every thread of the block calls it.  Up to 32 sequences every warp scans
// them by itself, a lane each, and no thread waits for another; more are shared out over the block
// (a multiple of 32 threads), a run of consecutive ones a thread.
template <class Want>
__device__ __forceinline__ PlanTotals plan(const CacheAttnArgs& a, PlanScratch* sc, Place* out, Want want) {
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5, n_warps = blockDim.x >> 5, Hkv = a.c.Hkv;
    if (a.B <= 32) {
        const bool mine = lane < a.B, ok = !mine || seq_ok(a, lane);
        SeqShape s{0, 0, 0, 0};
        if (mine && ok) s = seq_shape(a, lane);
        int64_t slots = s.len;
        for (int o = 16; o > 0; o >>= 1) slots += __shfl_xor_sync(0xffffffffu, slots, o);
        const int u = mine ? s.units(Hkv) : 0, g = s.groups(Hkv), i = mine ? s.items(Hkv) : 0;
        const int iu = scan_lanes(u, lane), ig = scan_lanes(g, lane), ii = scan_lanes(i, lane);
        const PlanTotals tot{__shfl_sync(0xffffffffu, iu, 31), __shfl_sync(0xffffffffu, ig, 31),
                             __shfl_sync(0xffffffffu, ii, 31), __all_sync(0xffffffffu, ok) && slots <= a.n_slots};
        if (!tot.ok) {
            if (t == 0) report(a.status, ESTP_ERR_INVALID_ARG);
            return tot;
        }
        Place p{lane, iu - u, ig - g, ii - i};
        const unsigned hit = __ballot_sync(0xffffffffu, mine && want(p, s, tot));
        const int from = hit ? __ffs(hit) - 1 : 0;
        out->b = hit ? from : a.B;
        out->unit0 = __shfl_sync(0xffffffffu, p.unit0, from);
        out->group0 = __shfl_sync(0xffffffffu, p.group0, from);
        out->item0 = __shfl_sync(0xffffffffu, p.item0, from);
        return tot;
    }
    const int run = (a.B + blockDim.x - 1) / blockDim.x;
    const int b0 = min(a.B, t * run), b1 = min(a.B, b0 + run);
    if (t == 0) {
        sc->bad = 0;
        sc->place = Place{a.B, 0, 0, 0};
    }
    __syncthreads();
    int s[3] = {0, 0, 0};
    int64_t slots = 0;
    for (int b = b0; b < b1; ++b) {
        if (!seq_ok(a, b)) {
            sc->bad = 1;
            break;
        }
        const SeqShape q = seq_shape(a, b);
        s[0] += q.units(Hkv);
        s[1] += q.groups(Hkv);
        s[2] += q.items(Hkv);
        slots += q.len;
    }
    int inc[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        inc[k] = scan_lanes(s[k], lane);
        if (lane == 31) sc->sum[k][warp] = inc[k];
    }
    for (int o = 16; o > 0; o >>= 1) slots += __shfl_xor_sync(0xffffffffu, slots, o);
    if (lane == 0) sc->slots[warp] = slots;
    __syncthreads();
    // every warp adds up the warps before it
    int before[3], all[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const int x = scan_lanes(lane < n_warps ? sc->sum[k][lane] : 0, lane);
        all[k] = __shfl_sync(0xffffffffu, x, 31);
        const int y = __shfl_sync(0xffffffffu, x, warp > 0 ? warp - 1 : 0);
        before[k] = warp > 0 ? y : 0;
    }
    slots = lane < n_warps ? sc->slots[lane] : 0;
    for (int o = 16; o > 0; o >>= 1) slots += __shfl_xor_sync(0xffffffffu, slots, o);
    const PlanTotals tot{all[0], all[1], all[2], sc->bad == 0 && slots <= a.n_slots};
    if (!tot.ok) {
        if (t == 0) report(a.status, ESTP_ERR_INVALID_ARG);
        return tot;
    }
    Place p{b0, before[0] + inc[0] - s[0], before[1] + inc[1] - s[1], before[2] + inc[2] - s[2]};
    while (p.b < b1) {
        const SeqShape q = seq_shape(a, p.b);
        if (want(p, q, tot)) sc->place = p;
        p.pass(q, Hkv);
    }
    __syncthreads();
    *out = sc->place;
    return tot;
}

// `total` cut into G shares that differ by one at most: the first of share c, and the share of x.
__device__ __forceinline__ int share_begin(int c, int total, int G) { return c * (total / G) + min(c, total % G); }
__device__ __forceinline__ int share_of(int x, int total, int G) {
    const int each = total / G, more = total % G, wide = more * (each + 1);
    return x < wide ? x / (each + 1) : more + (x - wide) / each;
}
// CTAs of the forward that get units, each at least one, or two where tiles may cost two: then every CTA
// whose share lies within a group holds the first unit of a tile, which is whose the tile is.
__device__ __forceinline__ int ctas_of(const CacheAttnArgs& a, int total) {
    return min(a.RB > 128 ? max(total / 2, 1) : total, a.G);
}
// The part of a sequence's units from loc on, count of them, that lies in one group: block k of KV head g,
// tiles [tile0, tile1) (none, where the tile of the first unit is another CTA's); `units` is how many.
struct Span {
    int g, k, tile0, tile1, units;
};
template <int kRB = 0>
__device__ __forceinline__ Span span_of(const CacheAttnArgs& a, const SeqShape& s, int loc, int count) {
    Span x;
    if ((kRB != 0 ? kRB : a.RB) <= 128) {  // a unit a tile
        const int grp = loc / s.nt;
        x.tile0 = loc - grp * s.nt;
        x.tile1 = min(s.nt, x.tile0 + count);
        x.units = x.tile1 - x.tile0;
        x.g = s.nrb == 1 ? grp : grp / s.nrb;
        x.k = grp - x.g * s.nrb;
        return x;
    }
    const int per = 2, head = s.cost * s.nt, block = per * s.nt;
    x.g = loc / head;
    const int in = loc % head;
    x.k = min(in / block, s.nrb - 1);
    const int c = x.k < s.nrb - 1 ? per : s.last, off = in - x.k * block;
    x.units = min(count, c * s.nt - off);
    x.tile0 = (off + c - 1) / c;
    x.tile1 = (off + x.units + c - 1) / c;
    return x;
}

// (-M, c / L) of a row: a row without keys, or of factor 0, has a factor of 0 and is left out.
__device__ __forceinline__ float2 weight_factor(const CacheAttnArgs& a, float2 x, int64_t row) {
    const float cw = a.row_weight != nullptr ? a.row_weight[row] : 1.f;
    const bool none = cw == 0.f || (x.x == -INFINITY && x.y == 0.f);
    return none ? make_float2(0.f, 0.f) : make_float2(x.x == -INFINITY ? 0.f : -x.x, cw / x.y);
}

// Which of the rows first .. first + nr - 1 (nr <= 64) of a (b, KV head) see draft j of the sequence's
// n drafts (from row0): bit r for row first + r, which is draft (first + r) / rep.
__device__ __forceinline__ uint64_t rows_that_see(const CacheAttnArgs& a, int64_t row0, int n, int j, int first, int nr) {
    if (j >= n || nr <= 0) return 0;
    if (a.tree == nullptr) {  // those from draft j's own on
        const int lo = max(j * a.rep - first, 0);
        return lo < nr ? ~0ull >> (64 - nr) & ~0ull << lo : 0;
    }
    const int i0 = first / a.rep, i1 = (first + nr - 1) / a.rep;
    const uint64_t* p = a.tree + row0 * a.words + (j >> 6);
    uint64_t rows = 0;
    for (int i = i0; i <= i1; i += 4) {
        bool sees[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)  // loads in flight together
            sees[k] = i + k <= i1 && (p[(int64_t)(i + k) * a.words] >> (j & 63) & 1);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int lo = max((i + k) * a.rep - first, 0), hi = min((i + k + 1) * a.rep - first, nr);
            if (sees[k]) rows |= ~0ull >> (64 - (hi - lo)) << lo;
        }
    }
    return rows;
}

// A launch that may begin before the one ahead of it has ended.
template <class Kernel, class... Args>
cudaError_t launch_dependent(Kernel kernel, int64_t grid, int threads, size_t smem, cudaStream_t st, const Args&... args) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
    return e == cudaSuccess ? cudaGetLastError() : e;
}

// The tensor-core forwards of bf16 caches: keys on the lanes (up to 32 rows a (b, KV head)), rows on the
// lanes (more).
estp_status launch_cache_fwd_tc(estp_ctx* ctx, const CacheAttnArgs& a, cudaStream_t st);
estp_status launch_cache_rows_tc(estp_ctx* ctx, const CacheAttnArgs& a, cudaStream_t st);
estp_status launch_cache_weight_tc(estp_ctx* ctx, const CacheAttnArgs& a, cudaStream_t st);
estp_status launch_cache_attention(estp_ctx* ctx, CacheAttnArgs& a, estp_dtype dtype, cudaStream_t st);
estp_status launch_cache_append(estp_ctx* ctx, const CacheView& c, int row_bytes, int B, const int32_t* length,
                                const int32_t* seen, int32_t* length_out, int32_t* seen_out, const void* kn,
                                const void* vn, int64_t ldn_bytes, int64_t n_src, const float* weight,
                                const int32_t* rows, const int32_t* cu, int64_t n_rows, cudaStream_t st);
estp_status launch_cache_evict(estp_ctx* ctx, const CacheView& c, int row_bytes, int B, const int32_t* length,
                               const int32_t* seen, int32_t* length_out, int budget, int recent, int sinks,
                               cudaStream_t st);

}  // namespace estp
