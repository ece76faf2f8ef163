// The paged KV cache as the kernels see it, and the cut of an attention call into units.
//
// A call's units are (sequence b, KV head g, block of RB rows, tile of 128 keys).  The rows of
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
    int KS;                      // partials of a segment
    int row_blocks;              // blocks of the finish kernel that merge rows
    int store;                   // scores are kept for the weights
    float* part_o;               // [G + groups][KS][RB][d]
    float2* part_ml;             // [G + groups][KS][RB]: running max (log2 units) and sum
    float* score;                // [units][RB][128], unscaled
    float2* factor;              // [n_rows, Hq]: (-M, c / L), where scores are formed again
    char* out;
    float* lse;
    float* w_new;
    int accumulate;
    int* status;
    long long wait_cycles;
};

// What sequence b brings to the call.
struct SeqShape {
    int len, n, nrb, nt;
    __device__ __forceinline__ int64_t units(int Hkv) const { return (int64_t)Hkv * nrb * nt; }
    __device__ __forceinline__ int64_t items(int Hkv) const { return n > 0 ? (int64_t)Hkv * nt : 0; }
};
__device__ __forceinline__ bool seq_ok(const CacheAttnArgs& a, int b) {
    const int len = a.length[b], lo = a.cu[b], hi = a.cu[b + 1];
    return len >= 0 && len <= a.c.capacity() && lo >= 0 && hi >= lo && hi - lo <= a.max_rows && hi <= a.n_rows &&
           (b > 0 || lo == 0) && (b + 1 < a.B || hi == a.n_rows);
}
__device__ __forceinline__ SeqShape seq_shape(const CacheAttnArgs& a, int b) {
    SeqShape s;
    s.len = a.length[b];
    s.n = a.cu[b + 1] - a.cu[b];
    s.nrb = (s.n * a.rep + a.RB - 1) / a.RB;
    s.nt = (s.len + kCacheTile - 1) / kCacheTile + 1;
    return s;
}

// Sums over the sequences before sequence b.
struct Place {
    int b;
    int64_t unit0, group0, item0;  // units, groups, items (KV head, tile) before it
};
struct PlanTotals {
    int64_t units, groups, items;
    bool ok;                       // lengths, cu and their sums are what the host was told
};
struct PlanScratch {
    int64_t sum[4][33];  // units, groups, items, slots
    int bad;
};

// Block-wide (a multiple of 32 threads): the call's totals, and visit(place, shape, totals) for every
// sequence, by one thread each.  A thread sums a run of consecutive sequences; an exclusive scan over
// the block gives each run's start.  Ends in a barrier.
template <class Visit>
__device__ __forceinline__ PlanTotals plan_block(const CacheAttnArgs& a, PlanScratch* sc, Visit visit) {
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5, n_warps = blockDim.x >> 5;
    const int run = (a.B + blockDim.x - 1) / blockDim.x;
    const int b0 = min(a.B, t * run), b1 = min(a.B, b0 + run);
    if (t == 0) sc->bad = 0;
    __syncthreads();
    int64_t s[4] = {0, 0, 0, 0};
    for (int b = b0; b < b1; ++b) {
        if (!seq_ok(a, b)) {
            sc->bad = 1;
            break;
        }
        const SeqShape q = seq_shape(a, b);
        s[0] += q.units(a.c.Hkv);
        s[1] += (int64_t)a.c.Hkv * q.nrb;
        s[2] += q.items(a.c.Hkv);
        s[3] += q.len;
    }
    int64_t inc[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        inc[k] = s[k];
        if (warp * 32 * run < a.B) {  // warps without sequences have nothing to add
            for (int o = 1; o < 32; o <<= 1) {
                const int64_t x = __shfl_up_sync(0xffffffffu, inc[k], o);
                if (lane >= o) inc[k] += x;
            }
        }
        if (lane == 31) sc->sum[k][warp] = inc[k];
    }
    __syncthreads();
    if (t < 4) {
        int64_t sum = 0;
        for (int w = 0; w < n_warps; ++w) {
            const int64_t x = sc->sum[t][w];
            sc->sum[t][w] = sum;
            sum += x;
        }
        sc->sum[t][32] = sum;
    }
    __syncthreads();
    const PlanTotals tot{sc->sum[0][32], sc->sum[1][32], sc->sum[2][32],
                         sc->bad == 0 && sc->sum[3][32] <= a.n_slots};
    if (!tot.ok && t == 0) report(a.status, ESTP_ERR_INVALID_ARG);
    if (tot.ok) {
        Place p{0, sc->sum[0][warp] + inc[0] - s[0], sc->sum[1][warp] + inc[1] - s[1],
                sc->sum[2][warp] + inc[2] - s[2]};
        for (int b = b0; b < b1; ++b) {
            const SeqShape q = seq_shape(a, b);
            p.b = b;
            visit(p, q, tot);
            p.unit0 += q.units(a.c.Hkv);
            p.group0 += (int64_t)a.c.Hkv * q.nrb;
            p.item0 += q.items(a.c.Hkv);
        }
    }
    __syncthreads();
    return tot;
}

// The CTAs that get units (each at least one), and the CTA that holds unit u when G CTAs share
// `total` units: CTA c holds [c total / G, (c + 1) total / G).
__device__ __forceinline__ int64_t ctas_of(const CacheAttnArgs& a, int64_t total) {
    return total < a.G ? total : a.G;
}
__device__ __forceinline__ int64_t unit_begin(int64_t c, int64_t total, int64_t G) { return c * total / G; }
__device__ __forceinline__ int64_t cta_of(int64_t u, int64_t total, int64_t G) { return ((u + 1) * G - 1) / total; }

// Which of the rows first .. first + nr - 1 (nr <= 64) of a (b, KV head) see draft j of the sequence's
// n drafts (from row0): bit r for row first + r, which is draft (first + r) / rep.
__device__ __forceinline__ uint64_t rows_that_see(const CacheAttnArgs& a, int64_t row0, int n, int j, int first, int nr) {
    if (j >= n || nr <= 0) return 0;
    const int i0 = first / a.rep, i1 = (first + nr - 1) / a.rep;
    const uint64_t* p = a.tree + row0 * a.words + (j >> 6);
    uint64_t rows = 0;
    for (int i = i0; i <= i1; i += 8) {
        bool sees[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)  // loads in flight together
            sees[k] = i + k <= i1 && (a.tree == nullptr ? j <= i + k : p[(int64_t)(i + k) * a.words] >> (j & 63) & 1);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int lo = max((i + k) * a.rep - first, 0), hi = min((i + k + 1) * a.rep - first, nr);
            if (sees[k]) rows |= ~0ull >> (64 - (hi - lo)) << lo;
        }
    }
    return rows;
}

// The tensor-core forward of bf16 caches: rows of a block and partials of a segment for a call's
// rows of a (b, KV head), and the launch.
void cache_tc_shape(int rows, int* RB, int* KS);
estp_status launch_cache_fwd_tc(const CacheAttnArgs& a, cudaStream_t st);
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
