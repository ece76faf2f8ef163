// Rows into a paged KV cache, and slots out of it.
//
// append_kernel: entry e of sequence b takes slot length_b + e (K and V rows, weight, position
// seen_b + e).  A warp an entry; bound by the rows' bytes, read and written once.
//
// evict_kernel: every (sequence, KV head) keeps its `budget` slots of the greatest rank: the sinks
// and the recent tokens first, then by weight, the lower slot first among equals.  The kept slots
// at or past `budget`, in order, fill the slots below it that lost their row, in order: only rows
// that have to move are read and written, at most min(budget, length - budget) a head, and a
// source is never a destination, so the moves need no order among themselves.  A cluster of C CTAs
// takes one (sequence, head), each CTA an equal run of its slots:
//   1. ranks of its slots as 32-bit keys in shared memory (formed again from the cache where they
//      do not fit);
//   2. the key T of rank `budget` by three rounds of 2048 bins, the CTAs' histograms added through
//      distributed shared memory;
//   3. one tally of the slots against T, exchanged once, gives every slot its place in the two lists;
//   4. the moves, dealt to all warps of the cluster.
// Integer work throughout: results do not depend on the launch.
#include <cooperative_groups.h>

#include "cache.cuh"

namespace cg = cooperative_groups;

namespace estp {
namespace {

// The last of the grid's blocks to arrive, each after it has read the lengths it needs (the new
// lengths may replace the old ones in place); the counter is zero again afterwards.
__device__ __forceinline__ bool last_arrival(uint32_t* done, uint32_t n) {
    __threadfence();
    if (atomicAdd(done, 1u) != n - 1) return false;
    *done = 0;
    __threadfence();
    return true;
}

constexpr int kAppendWarps = 8;

struct AppendArgs {
    CacheView c;
    int row_bytes, B;
    const int32_t* length;  // NULL: every sequence is empty
    const int32_t* seen;
    int32_t* length_out;
    int32_t* seen_out;
    const char* kn;
    const char* vn;
    int64_t ldn, n_src;
    const float* weight;
    const int32_t* rows;
    const int32_t* cu;
    int64_t n_rows;
    uint32_t* done;
    int* status;
};

// Whether sequence b's entries are an orderly part of the list and fit its slots.
__device__ __forceinline__ bool append_ok(const AppendArgs& a, int lo, int hi, int len) {
    return lo >= 0 && hi >= lo && hi <= a.n_rows && len >= 0 && (int64_t)len + (hi - lo) <= a.c.capacity();
}

__global__ void __launch_bounds__(32 * kAppendWarps, 4) append_kernel(const AppendArgs a) {
    await_stream();
    admit_next();
    const int lane = threadIdx.x & 31;
    const int per = a.row_bytes / 16, n = a.c.Hkv * per;
    const int64_t total = min((int64_t)max(a.cu[a.B], 0), a.n_rows), e0 = max(a.cu[0], 0);
    const int64_t step_e = (int64_t)gridDim.x * kAppendWarps;
    // a row's first 16-byte units, on their way while the row before it and its slot are dealt with
    constexpr int kAhead = 2;
    uint4 x[kAhead], y[kAhead];
    auto fetch = [&](int64_t e) {
        const int64_t src = e >= total ? -1 : a.rows != nullptr ? a.rows[e] : e;
        if (src < 0 || src >= a.n_src) return (int64_t)-1;
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (lane + 32 * i < n) {
                x[i] = ld_stream(a.kn + src * a.ldn + (lane + 32 * i) * 16);
                y[i] = ld_stream(a.vn + src * a.ldn + (lane + 32 * i) * 16);
            }
        return src;
    };
    int64_t e = e0 + (int64_t)blockIdx.x * kAppendWarps + (threadIdx.x >> 5), ahead = fetch(e);
    for (; e < total; e += step_e) {
        const int64_t src = ahead;
        uint4 u[kAhead], v[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) u[i] = x[i], v[i] = y[i];
        ahead = fetch(e + step_e);
        if (src < 0) {
            if (lane == 0) report(a.status, ESTP_ERR_INVALID_ARG);
            continue;
        }
        const char* kr = a.kn + src * a.ldn;
        const char* vr = a.vn + src * a.ldn;
        // the last b with cu[b] <= e: 32 probes a step
        int lo = 0, hi = a.B;  // cu[lo] <= e < cu[hi]
        while (hi - lo > 1) {
            const int step = (hi - lo + 31) / 32, at = lo + (lane + 1) * step;
            const unsigned below = __ballot_sync(0xffffffffu, at < hi && a.cu[at] <= e);
            const int k = __ffs(~below) - 1;  // leading probes at or below e; the last one is never below hi
            hi = min(hi, lo + (k + 1) * step);
            lo += k * step;
        }
        const int b = lo, first = a.cu[b], next = a.cu[b + 1], len = a.length != nullptr ? a.length[b] : 0;
        if (!append_ok(a, first, next, len) || e < first || e >= next) continue;  // reported below
        const int slot = len + (int)(e - first), pos = (a.length != nullptr ? a.seen[b] : 0) + (int)(e - first);
        const int64_t page = a.c.page_of(b, slot, a.status);
        if (page < 0 || !a.c.inside(page, slot, 0, a.status) || !in_bounds(src < a.n_src, a.status)) continue;
        auto put = [&](int i, const uint4& p, const uint4& q) {
            const int g = i / per, o = (i - g * per) * 16;
            const int64_t to = a.c.row(page, slot, g) + o;
            *reinterpret_cast<uint4*>(a.c.k + to) = p;
            *reinterpret_cast<uint4*>(a.c.v + to) = q;
        };
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (lane + 32 * i < n) put(lane + 32 * i, u[i], v[i]);
        for (int i = lane + 32 * kAhead; i < n; i += 32)
            put(i, ld_stream(kr + (int64_t)i * 16), ld_stream(vr + (int64_t)i * 16));
        for (int g = lane; g < a.c.Hkv; g += 32) {
            const int64_t m = a.c.meta(page, slot, g);
            if (a.c.weight != nullptr) a.c.weight[m] = a.weight != nullptr ? a.weight[src * a.c.Hkv + g] : 0.f;
            if (a.c.position != nullptr) a.c.position[m] = pos;
        }
    }
    __shared__ bool last;
    __syncthreads();
    if (threadIdx.x == 0) last = last_arrival(a.done, gridDim.x);
    __syncthreads();
    if (!last) return;
    for (int i = threadIdx.x; i < a.B; i += blockDim.x) {
        const int first = a.cu[i], next = a.cu[i + 1], len = a.length != nullptr ? a.length[i] : 0;
        const int seen = a.length != nullptr ? a.seen[i] : 0;
        const bool fits = append_ok(a, first, next, len) && (i > 0 || first == 0);
        if (!fits) report(a.status, ESTP_ERR_INVALID_ARG);
        a.length_out[i] = len + (fits ? next - first : 0);
        a.seen_out[i] = seen + (fits ? next - first : 0);
    }
}

constexpr int kEvictThreads = 512, kEvictWarps = kEvictThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kRounds = 3, kBins = 2048;  // digits of 11, 11 and 10 bits, from the top
constexpr int kBinsOf = kBins / kEvictThreads;
static_assert(kBinsOf == 4, "a thread sums one 16-byte group of bins");

struct EvictArgs {
    CacheView c;
    int row_bytes, B;
    const int32_t* length;
    const int32_t* seen;
    int32_t* length_out;
    int budget, recent, sinks;
    int key_cap;            // keys a CTA holds in shared memory
    int max_moves;
    int2* list;             // [groups][2][max_moves] (page, slot of it): freed slots, kept slots past the budget
    uint32_t* done;
    int* status;
};

// Order of the weights as unsigned integers: NaN below everything, -0 as 0.
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Slots of a run by their key against T: those that say how many are freed and kept past the budget
// once the number of kept equals is known.  Kept equals are the first in slot order, so those below
// the budget come before those past it.
struct Tally {
    int below_lt, below_eq, past_gt, past_eq;
    __device__ __forceinline__ int kept_equal(int left, int equal_before) const {
        return max(0, min(left - equal_before, below_eq + past_eq));
    }
    __device__ __forceinline__ int freed(int kept) const { return below_lt + below_eq - min(kept, below_eq); }
    __device__ __forceinline__ int kept_past(int kept) const { return past_gt + max(0, kept - below_eq); }
};

// Two CTAs an SM: 64 registers
__global__ void __launch_bounds__(kEvictThreads, 2) evict_kernel(const EvictArgs a) {
    extern __shared__ uint32_t dyn[];
    uint32_t* hist = dyn;                     // [kRounds][kBins]
    uint32_t* keys = dyn + kRounds * kBins;   // [key_cap]
    __shared__ Tally tally[kEvictWarps], cta_tally;
    __shared__ uint32_t warp_sum[kEvictWarps], pick[2];
    cg::cluster_group cl = cg::this_cluster();
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const int C = (int)cl.num_blocks(), rank = (int)cl.block_rank();
    for (int i = t; i < kRounds * kBins / 4; i += kEvictThreads) reinterpret_cast<uint4*>(hist)[i] = make_uint4(0, 0, 0, 0);
    await_stream();
    admit_next();
    const int group = blockIdx.x / C, b = group / a.c.Hkv, g = group % a.c.Hkv;
    const int len = a.length[b], seen = a.seen[b];
    const bool bad = len < 0 || len > a.c.capacity();
    const int n = bad ? 0 : len;
    __syncthreads();
    __shared__ bool last;
    if (t == 0) last = last_arrival(a.done, gridDim.x);
    __syncthreads();
    if (last)
        for (int i = t; i < a.B; i += kEvictThreads) {
            const int l = a.length[i];
            const bool fits = l >= 0 && l <= a.c.capacity();  // else nothing was ranked or moved: the length stays
            if (!fits) report(a.status, ESTP_ERR_INVALID_ARG);
            a.length_out[i] = fits ? min(l, a.budget) : l;
        }
    if (n <= a.budget) return;  // the whole cluster

    const int run = ((n + C - 1) / C + 127) / 128 * 128;  // a warp takes 128 slots at a time, a lane 4
    const int lo = min(n, rank * run), hi = min(n, lo + run);
    const int32_t* table = a.c.table + (int64_t)b * a.c.ld_table;
    // keys of 4 slots of one page, from a multiple of 4; 0 past the sequence's slots
    auto form_keys = [&](int slot) -> uint4 {
        const int page = table[slot >> a.c.shift];
        if (page < 0 || page >= a.c.n_pages) {
            report(a.status, ESTP_ERR_INVALID_ARG);
            return make_uint4(0, 0, 0, 0);
        }
        const int64_t m = a.c.meta(page, slot, g);
        const int4 pos = *reinterpret_cast<const int4*>(a.c.position + m);
        const float4 w = *reinterpret_cast<const float4*>(a.c.weight + m);
        auto one = [&](int p, float x, int s) {
            return s >= n ? 0u : p < a.sinks || p >= seen - a.recent ? 0xffffffffu : weight_key(x);
        };
        return make_uint4(one(pos.x, w.x, slot), one(pos.y, w.y, slot + 1), one(pos.z, w.z, slot + 2), one(pos.w, w.w, slot + 3));
    };
    {
        constexpr int kBatch = 2;  // 8 slots a thread has in flight
        const int top = min(hi, lo + a.key_cap);
        for (int s0 = lo + 4 * t; s0 < top; s0 += kBatch * 4 * kEvictThreads) {
            uint4 k[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (s0 + i * 4 * kEvictThreads < top) k[i] = form_keys(s0 + i * 4 * kEvictThreads);
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (s0 + i * 4 * kEvictThreads < top) *reinterpret_cast<uint4*>(keys + (s0 + i * 4 * kEvictThreads - lo)) = k[i];
        }
    }
    __syncthreads();
    auto keys_of = [&](int slot) {
        return slot - lo < a.key_cap ? *reinterpret_cast<const uint4*>(keys + (slot - lo)) : form_keys(slot);
    };

    // the key T of rank `budget`, digit by digit; `left` keys equal to what is known of it are still wanted
    uint32_t T = 0;
    int left = a.budget;
#pragma unroll
    for (int d = 0; d < kRounds; ++d) {
        const int bits = d == kRounds - 1 ? 10 : 11, shift = d == 0 ? 21 : d == 1 ? 10 : 0;
        uint32_t* h = hist + d * kBins;
        for (int s = lo + 4 * t; s < hi; s += 4 * kEvictThreads) {
            const uint4 k4 = keys_of(s);
            const uint32_t k[4] = {k4.x, k4.y, k4.z, k4.w};
            int safe = 0;  // alike and many: counted apart
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (s + i >= hi || (d > 0 && (k[i] ^ T) >> (shift + bits) != 0)) continue;
                if (k[i] == 0xffffffffu) ++safe;
                else atomicAdd(&h[k[i] >> shift & ((1u << bits) - 1)], 1u);
            }
            if (safe) atomicAdd(&h[(1u << bits) - 1], (uint32_t)safe);
        }
        if (C > 1) cl.sync();
        else __syncthreads();
        // thread t: bins top - 4 t .. top - 4 t - 3 of the whole cluster
        const int bin = kBins - 4 - 4 * t;
        uint4 sum = *reinterpret_cast<const uint4*>(h + bin);
        if (C > 1) {
            uint4 other[kMaxCluster - 1];
#pragma unroll
            for (int r = 1; r < kMaxCluster; ++r)
                if (r < C) other[r - 1] = *reinterpret_cast<const uint4*>(cl.map_shared_rank(h, (rank + r) % C) + bin);
#pragma unroll
            for (int r = 1; r < kMaxCluster; ++r)
                if (r < C) {
                    sum.x += other[r - 1].x;
                    sum.y += other[r - 1].y;
                    sum.z += other[r - 1].z;
                    sum.w += other[r - 1].w;
                }
        }
        const uint32_t mine = sum.x + sum.y + sum.z + sum.w;
        uint32_t inc = mine;
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += x;
        }
        if (lane == 31) warp_sum[warp] = inc;
        __syncthreads();
        uint32_t above = lane < warp ? warp_sum[lane] : 0u;
        for (int o = 16; o > 0; o >>= 1) above += __shfl_xor_sync(0xffffffffu, above, o);
        above += inc - mine;
        if (above < (uint32_t)left && (uint32_t)left <= above + mine) {  // one thread
            const uint32_t c4[4] = {sum.w, sum.z, sum.y, sum.x};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (above < (uint32_t)left && (uint32_t)left <= above + c4[i]) {
                    pick[0] = bin + 3 - i;
                    pick[1] = left - above;
                }
                above += c4[i];
            }
        }
        __syncthreads();
        T |= pick[0] << shift;
        left = (int)pick[1];
    }

    // every warp's run of slots, tallied against T
    const int per_warp = (run / 128 + kEvictWarps - 1) / kEvictWarps * 128;
    const int w0 = min(hi, lo + warp * per_warp), w1 = min(hi, w0 + per_warp);
    Tally mine{0, 0, 0, 0};
    for (int s = w0 + 4 * lane; s < w1; s += 128) {
        const uint4 k4 = keys_of(s);
        const uint32_t k[4] = {k4.x, k4.y, k4.z, k4.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (s + i >= w1) continue;
            const bool below = s + i < a.budget;
            mine.below_lt += below && k[i] < T;
            mine.below_eq += below && k[i] == T;
            mine.past_gt += !below && k[i] > T;
            mine.past_eq += !below && k[i] == T;
        }
    }
    auto warp_add = [&](Tally x) {  // over the warp's lanes
        for (int o = 16; o > 0; o >>= 1) {
            x.below_lt += __shfl_xor_sync(0xffffffffu, x.below_lt, o);
            x.below_eq += __shfl_xor_sync(0xffffffffu, x.below_eq, o);
            x.past_gt += __shfl_xor_sync(0xffffffffu, x.past_gt, o);
            x.past_eq += __shfl_xor_sync(0xffffffffu, x.past_eq, o);
        }
        return x;
    };
    mine = warp_add(mine);
    if (lane == 0) tally[warp] = mine;
    __syncthreads();
    const Tally none{0, 0, 0, 0};
    const Tally cta_all = warp_add(lane < kEvictWarps ? tally[lane] : none);
    if (t == 0) cta_tally = cta_all;
    if (C > 1) cl.sync();
    else __syncthreads();
    // what lies before this CTA's run and before this warp's: equals first, then the lists' places
    const Tally of_rank = lane < C ? *cl.map_shared_rank(&cta_tally, lane) : none;
    const Tally of_warp = lane < kEvictWarps ? tally[lane] : none;
    auto before = [&](int x, int upto) {  // sum of x over the lanes below `upto`
        x = lane < upto ? x : 0;
        for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        return x;
    };
    auto lane_before = [&](int x) {  // exclusive scan over the lanes
        int inc = x;
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += y;
        }
        return inc - x;
    };
    const int rank_eq = of_rank.below_eq + of_rank.past_eq, warp_eq = of_warp.below_eq + of_warp.past_eq;
    const int rank_kept = of_rank.kept_equal(left, lane_before(rank_eq));
    const int eq_cta = before(rank_eq, rank);
    const int warp_kept = of_warp.kept_equal(left, eq_cta + lane_before(warp_eq));
    const int moves = before(of_rank.freed(rank_kept), 32);
    int f0 = before(of_rank.freed(rank_kept), rank) + before(of_warp.freed(warp_kept), warp);
    int p0 = before(of_rank.kept_past(rank_kept), rank) + before(of_warp.kept_past(warp_kept), warp);
    int eq0 = eq_cta + before(warp_eq, warp);

    int2* list_f = a.list + (int64_t)group * 2 * a.max_moves;
    int2* list_p = list_f + a.max_moves;
    for (int s0 = w0; s0 < w1; s0 += 128) {
        const int s = s0 + 4 * lane;
        const uint4 k4 = s < w1 ? keys_of(s) : make_uint4(0, 0, 0, 0);
        const uint32_t k[4] = {k4.x, k4.y, k4.z, k4.w};
        int eq = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) eq += s + i < w1 && k[i] == T;
        const int eq_scan = lane_before(eq);
        unsigned freed = 0, past = 0;
        int e = eq0 + eq_scan;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool in = s + i < w1, keep = in && (k[i] > T || (k[i] == T && e < left));
            e += in && k[i] == T;
            if (in && s + i < a.budget && !keep) freed |= 1u << i;
            if (keep && s + i >= a.budget) past |= 1u << i;
        }
        // both counts in one scan: each is at most 128
        const int both = __popc(freed) | __popc(past) << 16, scan = lane_before(both);
        int f = f0 + (scan & 0xffff), p = p0 + (scan >> 16);
        if (freed | past) {
            const int page = table[s >> a.c.shift];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (freed >> i & 1 && in_bounds(f >= 0 && f < a.max_moves, a.status)) list_f[f++] = make_int2(page, s + i);
                if (past >> i & 1 && in_bounds(p >= 0 && p < a.max_moves, a.status)) list_p[p++] = make_int2(page, s + i);
            }
        }
        const int all = __shfl_sync(0xffffffffu, scan + both, 31);
        f0 += all & 0xffff;
        p0 += all >> 16;
        eq0 += __shfl_sync(0xffffffffu, eq_scan + eq, 31);
    }
    if (C > 1) cl.sync();  // the lists are complete, and no CTA reads another's shared memory any more
    else __syncthreads();
    const int per = a.row_bytes / 16;  // 8, 16 or 32 lanes a row: as many rows a warp at once as fit
    const int sub = lane / per, at = lane % per, together = 32 / per;
    constexpr int kBatch = 4;  // rows a lane has in flight
    const int stride = C * kEvictWarps * together;
    for (int j0 = (rank * kEvictWarps + warp) * together + sub; j0 < moves; j0 += kBatch * stride) {
        int2 dst[kBatch], src[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int j = j0 + i * stride;
            const bool there = j < moves && in_bounds(j < a.max_moves, a.status);
            dst[i] = there ? list_f[j] : make_int2(-1, 0);
            src[i] = there ? list_p[j] : make_int2(-1, 0);
        }
        uint4 x[kBatch], y[kBatch];
        float w[kBatch];
        int pos[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            // a page that is none was reported with its key
            if (src[i].x < 0 || src[i].x >= a.c.n_pages || dst[i].x >= a.c.n_pages) dst[i].x = -1;
            if (dst[i].x >= 0 && !(a.c.inside(src[i].x, src[i].y, g, a.status) && a.c.inside(dst[i].x, dst[i].y, g, a.status))) dst[i].x = -1;
            if (dst[i].x < 0) continue;
            const int64_t from = a.c.row(src[i].x, src[i].y, g) + at * 16, ms = a.c.meta(src[i].x, src[i].y, g);
            x[i] = *reinterpret_cast<const uint4*>(a.c.k + from);
            y[i] = *reinterpret_cast<const uint4*>(a.c.v + from);
            if (at == 0) {
                w[i] = a.c.weight[ms];
                pos[i] = a.c.position[ms];
            }
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            if (dst[i].x < 0) continue;
            const int64_t to = a.c.row(dst[i].x, dst[i].y, g) + at * 16, md = a.c.meta(dst[i].x, dst[i].y, g);
            *reinterpret_cast<uint4*>(a.c.k + to) = x[i];
            *reinterpret_cast<uint4*>(a.c.v + to) = y[i];
            if (at == 0) {
                a.c.weight[md] = w[i];
                a.c.position[md] = pos[i];
            }
        }
    }
}

}  // namespace

estp_status launch_cache_append(estp_ctx* ctx, const CacheView& c, int row_bytes, int B, const int32_t* length,
                                const int32_t* seen, int32_t* length_out, int32_t* seen_out, const void* kn,
                                const void* vn, int64_t ldn_bytes, int64_t n_src, const float* weight,
                                const int32_t* rows, const int32_t* cu, int64_t n_rows, cudaStream_t st) {
    AppendArgs a{c, row_bytes, B, length, seen, length_out, seen_out, static_cast<const char*>(kn),
                 static_cast<const char*>(vn), ldn_bytes, n_src, weight, rows, cu, n_rows, ctx->done, ctx->status};
    // a warp an entry, up to 4 blocks an SM, all resident (32 warps with two rows each in flight), then
    // several.  Four prompts of 32k, 4 KV heads of 128: 94 us for 540 MB; without the row ahead 114, with 5
    // blocks resident 175, and 105 where a warp's entries follow one another
    const int64_t blocks = n_rows > 0 ? (n_rows + kAppendWarps - 1) / kAppendWarps : 1, most = 4 * ctx->num_sms;
    const int64_t grid = blocks < most ? blocks : most;
    const cudaError_t e = launch_dependent(append_kernel, grid, 32 * kAppendWarps, 0, st, a);
    return e == cudaSuccess ? ESTP_OK : cuda_fail(e, "cache append launch");
}

estp_status launch_cache_evict(estp_ctx* ctx, const CacheView& c, int row_bytes, int B, const int32_t* length,
                               const int32_t* seen, int32_t* length_out, int budget, int recent, int sinks,
                               cudaStream_t st) {
    const int64_t groups = (int64_t)B * c.Hkv, cap = c.capacity();
    // CTAs of a cluster: up to two an SM over all groups, while each keeps a run of 512 slots
    int C = 1;
    while (C < kMaxCluster && groups * C * 2 <= 2 * ctx->num_sms && cap >= (int64_t)C * 2 * 512) C *= 2;
    const int64_t run = ((cap + C - 1) / C + 127) / 128 * 128;
    const int64_t max_keys = 48 * 1024;  // 192 KB
    EvictArgs a{c, row_bytes, B, length, seen, length_out, budget, recent, sinks};
    a.key_cap = (int)(run < max_keys ? run : max_keys);
    const int64_t moves = cap > budget ? (cap - budget < budget ? cap - budget : budget) : 0;
    a.max_moves = (int)moves;
    estp_status s = ws_reserve(ctx, sizeof(int2) * 2 * (size_t)groups * (size_t)moves + 16);
    if (s != ESTP_OK) return s;
    a.list = static_cast<int2*>(ctx->ws);
    a.done = ctx->done;
    a.status = ctx->status;
    const size_t smem = sizeof(uint32_t) * ((size_t)a.key_cap + kRounds * kBins);
    cudaError_t e = set_smem(ctx, 0, evict_kernel, (size_t)(max_keys + kRounds * kBins) * 4);
    if (e != cudaSuccess) return cuda_fail(e, "cache evict smem attribute");
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)C;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(groups * C));
    cfg.blockDim = dim3(kEvictThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, evict_kernel, a);
    if (e == cudaSuccess) e = cudaGetLastError();
    return e == cudaSuccess ? ESTP_OK : cuda_fail(e, "cache evict launch");
}

}  // namespace estp
