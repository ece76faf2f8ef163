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
//   2. the key T of rank `budget` by four rounds of 256 bins, the CTAs' histograms added through
//      distributed shared memory;
//   3. counts of keys equal to T, of freed slots and of kept ones past the budget, scanned over
//      warps and CTAs, give every slot its place in the two lists;
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

__global__ void __launch_bounds__(32 * kAppendWarps) append_kernel(const AppendArgs a) {
    const int lane = threadIdx.x & 31;
    const int64_t e = (int64_t)blockIdx.x * kAppendWarps + (threadIdx.x >> 5);
    bool ok = false;
    int b = 0, slot = 0, pos = 0;
    if (e < a.n_rows && e < a.cu[a.B] && a.cu[0] <= e) {
        // the last b with cu[b] <= e: 32 probes a step
        int lo = 0, hi = a.B;  // cu[lo] <= e < cu[hi]
        while (hi - lo > 1) {
            const int step = (hi - lo + 31) / 32, at = lo + (lane + 1) * step;
            const unsigned below = __ballot_sync(0xffffffffu, at < hi && a.cu[at] <= e);
            const int k = __ffs(~below) - 1;  // leading probes at or below e; the last one is never below hi
            hi = min(hi, lo + (k + 1) * step);
            lo += k * step;
        }
        b = lo;
        const int first = a.cu[b], next = a.cu[b + 1], len = a.length != nullptr ? a.length[b] : 0;
        slot = len + (int)(e - first);
        pos = (a.length != nullptr ? a.seen[b] : 0) + (int)(e - first);
        ok = append_ok(a, first, next, len) && e >= first && e < next;
    }
    __syncthreads();
    __shared__ bool last;
    if (threadIdx.x == 0) last = last_arrival(a.done, gridDim.x);
    __syncthreads();
    if (last) {
        for (int i = threadIdx.x; i < a.B; i += blockDim.x) {
            const int first = a.cu[i], next = a.cu[i + 1], len = a.length != nullptr ? a.length[i] : 0;
            const int seen = a.length != nullptr ? a.seen[i] : 0;
            const bool fits = append_ok(a, first, next, len) && (i > 0 || first == 0);
            if (!fits) report(a.status, ESTP_ERR_INVALID_ARG);
            a.length_out[i] = len + (fits ? next - first : 0);
            a.seen_out[i] = seen + (fits ? next - first : 0);
        }
    }
    if (!ok) return;
    const int64_t src = a.rows != nullptr ? a.rows[e] : e;
    if (src < 0 || src >= a.n_src) {
        if (lane == 0) report(a.status, ESTP_ERR_INVALID_ARG);
        return;
    }
    const int64_t page = a.c.page_of(b, slot, a.status);
    if (page < 0) return;
    const int per = a.row_bytes / 16, n = a.c.Hkv * per;
    const char* kr = a.kn + src * a.ldn;
    const char* vr = a.vn + src * a.ldn;
    for (int i = lane; i < n; i += 32) {
        const int g = i / per, o = (i - g * per) * 16;
        const int64_t to = a.c.row(page, slot, g) + o;
        const uint4 x = ld_stream(kr + (int64_t)i * 16), y = ld_stream(vr + (int64_t)i * 16);
        *reinterpret_cast<uint4*>(a.c.k + to) = x;
        *reinterpret_cast<uint4*>(a.c.v + to) = y;
    }
    for (int g = lane; g < a.c.Hkv; g += 32) {
        const int64_t m = a.c.meta(page, slot, g);
        if (a.c.weight != nullptr) a.c.weight[m] = a.weight != nullptr ? a.weight[src * a.c.Hkv + g] : 0.f;
        if (a.c.position != nullptr) a.c.position[m] = pos;
    }
}

constexpr int kEvictThreads = 512, kEvictWarps = kEvictThreads / 32;
constexpr int kMaxCluster = 8;

struct EvictArgs {
    CacheView c;
    int row_bytes, B;
    const int32_t* length;
    const int32_t* seen;
    int32_t* length_out;
    int budget, recent, sinks;
    int key_cap;            // keys a CTA holds in shared memory
    int max_moves;
    int32_t* list;          // [groups][2][max_moves]: freed slots, kept slots past the budget
    uint32_t* done;
    int* status;
};

// Order of the weights as unsigned integers: NaN below everything, -0 as 0.
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// What a CTA tells the others of its cluster.
struct EvictShare {
    uint32_t hist[4][256];
    int equal, freed, kept_past;
};

__global__ void __launch_bounds__(kEvictThreads) evict_kernel(const EvictArgs a) {
    extern __shared__ uint32_t keys[];
    __shared__ EvictShare sh;
    __shared__ int warp_sum[2][kEvictWarps];
    __shared__ uint32_t pick[2];
    cg::cluster_group cl = cg::this_cluster();
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const int C = (int)cl.num_blocks(), rank = (int)cl.block_rank();
    const int group = blockIdx.x / C, b = group / a.c.Hkv, g = group % a.c.Hkv;
    const int len = a.length[b], seen = a.seen[b];
    const bool bad = len < 0 || len > a.c.capacity();
    const int n = bad ? 0 : len;
    for (int i = t; i < 4 * 256; i += kEvictThreads) (&sh.hist[0][0])[i] = 0;
    __syncthreads();
    __shared__ bool last;
    if (t == 0) last = last_arrival(a.done, gridDim.x);
    __syncthreads();
    if (last)
        for (int i = t; i < a.B; i += kEvictThreads) {
            const int l = a.length[i];
            if (l < 0 || l > a.c.capacity()) report(a.status, ESTP_ERR_INVALID_ARG);
            a.length_out[i] = min(l, a.budget);
        }
    if (n <= a.budget) return;  // the whole cluster

    const int run = ((n + C - 1) / C + 31) / 32 * 32;
    const int lo = min(n, rank * run), hi = min(n, lo + run);
    auto form_key = [&](int slot) -> uint32_t {
        const int page = a.c.table[(int64_t)b * a.c.ld_table + (slot >> a.c.shift)];
        const bool there = page >= 0 && page < a.c.n_pages;
        if (!there) report(a.status, ESTP_ERR_INVALID_ARG);
        const int64_t m = a.c.meta(there ? page : 0, slot, g);
        const int pos = there ? a.c.position[m] : 0;
        const float w = there ? a.c.weight[m] : 0.f;
        return !there ? 0u : pos < a.sinks || pos >= seen - a.recent ? 0xffffffffu : weight_key(w);
    };
    {
        constexpr int kBatch = 4;  // slots a thread has in flight
        const int top = min(hi, lo + a.key_cap);
        for (int s0 = lo + t; s0 < top; s0 += kBatch * kEvictThreads) {
            uint32_t k[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) k[i] = s0 + i * kEvictThreads < top ? form_key(s0 + i * kEvictThreads) : 0u;
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (s0 + i * kEvictThreads < top) keys[s0 + i * kEvictThreads - lo] = k[i];
        }
    }
    __syncthreads();
    auto key = [&](int slot) { return slot - lo < a.key_cap ? keys[slot - lo] : form_key(slot); };

    // the key of rank `budget`, digit by digit from the top; `left` keys of it are still to be found
    uint32_t T = 0;
    int left = a.budget;
    for (int d = 0; d < 4; ++d) {
        const int shift = 24 - 8 * d;
        for (int s0 = lo + warp * 32; s0 < hi; s0 += kEvictThreads) {
            const int s = s0 + lane;
            const uint32_t k = s < hi ? key(s) : 0u;
            const bool in = s < hi && (d == 0 || (k ^ T) >> (shift + 8) == 0);
            const uint32_t bin = in ? k >> shift & 255u : 256u;
            const unsigned same = __match_any_sync(0xffffffffu, bin);
            if (in && lane == __ffs(same) - 1) atomicAdd(&sh.hist[d][bin], (uint32_t)__popc(same));
        }
        cl.sync();
        if (warp == 0) {  // bins of 8 a lane, the highest digit in lane 0
            uint32_t h[8], sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int bin = 255 - (lane * 8 + i);
                h[i] = 0;
                for (int r = 0; r < C; ++r) h[i] += cl.map_shared_rank(&sh, r)->hist[d][bin];
                sum += h[i];
            }
            uint32_t inc = sum;
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t x = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= o) inc += x;
            }
            uint32_t above = inc - sum;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (above < (uint32_t)left && (uint32_t)left <= above + h[i]) {
                    pick[0] = 255 - (lane * 8 + i);
                    pick[1] = left - above;
                }
                above += h[i];
            }
        }
        __syncthreads();
        T |= pick[0] << shift;
        left = (int)pick[1];
        __syncthreads();
    }

    // slots equal to T before each warp's run of this CTA
    const int per_warp = (run / 32 + kEvictWarps - 1) / kEvictWarps * 32;
    const int w0 = min(hi, lo + warp * per_warp), w1 = min(hi, w0 + per_warp);
    auto scan_warps = [&](int* sums, int mine, int* total) {  // exclusive over the block's warps
        if (lane == 0) sums[warp] = mine;
        __syncthreads();
        int before = 0, all = 0;
        for (int w = 0; w < kEvictWarps; ++w) {
            before += w < warp ? sums[w] : 0;
            all += sums[w];
        }
        *total = all;
        return before;
    };
    int n_eq = 0;
    for (int s0 = w0; s0 < w1; s0 += 32) {
        const int s = s0 + lane;
        n_eq += __popc(__ballot_sync(0xffffffffu, s < w1 && key(s) == T));
    }
    int total;
    int eq = scan_warps(warp_sum[0], n_eq, &total);
    if (t == 0) sh.equal = total;
    cl.sync();
    for (int r = 0; r < rank; ++r) eq += cl.map_shared_rank(&sh, r)->equal;
    const int eq0 = eq;

    // freed slots below the budget and kept ones at or past it
    auto classify = [&](int s, int& eq_run, bool& freed, bool& past) {
        const uint32_t k = s < w1 ? key(s) : 0u;
        const unsigned is_eq = __ballot_sync(0xffffffffu, s < w1 && k == T);
        const int my_eq = eq_run + __popc(is_eq & ((1u << lane) - 1));
        const bool keep = s < w1 && (k > T || (k == T && my_eq < left));
        eq_run += __popc(is_eq);
        freed = s < w1 && s < a.budget && !keep;
        past = keep && s >= a.budget;
    };
    int nf = 0, np = 0;
    bool freed, past;
    for (int s0 = w0; s0 < w1; s0 += 32) {
        classify(s0 + lane, eq, freed, past);
        nf += __popc(__ballot_sync(0xffffffffu, freed));
        np += __popc(__ballot_sync(0xffffffffu, past));
    }
    __syncthreads();
    int tf, tp;
    int f0 = scan_warps(warp_sum[0], nf, &tf), p0 = scan_warps(warp_sum[1], np, &tp);
    if (t == 0) {
        sh.freed = tf;
        sh.kept_past = tp;
    }
    cl.sync();
    int moves = 0;
    for (int r = 0; r < C; ++r) {
        const EvictShare* o = cl.map_shared_rank(&sh, r);
        if (r < rank) {
            f0 += o->freed;
            p0 += o->kept_past;
        }
        moves += o->freed;
    }
    int32_t* list_f = a.list + (int64_t)group * 2 * a.max_moves;
    int32_t* list_p = list_f + a.max_moves;
    eq = eq0;
    for (int s0 = w0; s0 < w1; s0 += 32) {
        const int s = s0 + lane;
        classify(s, eq, freed, past);
        const unsigned bf = __ballot_sync(0xffffffffu, freed), bp = __ballot_sync(0xffffffffu, past);
        const unsigned below = (1u << lane) - 1;
        if (freed) list_f[f0 + __popc(bf & below)] = s;
        if (past) list_p[p0 + __popc(bp & below)] = s;
        f0 += __popc(bf);
        p0 += __popc(bp);
    }
    cl.sync();  // the lists are complete, and no CTA reads another's shared memory any more
    const int per = a.row_bytes / 16;  // 8, 16 or 32 lanes a row: as many rows a warp at once as fit
    const int sub = lane / per, at = lane % per, together = 32 / per;
    constexpr int kBatch = 4;  // rows a lane has in flight
    const int stride = C * kEvictWarps * together;
    for (int j0 = (rank * kEvictWarps + warp) * together + sub; j0 < moves; j0 += kBatch * stride) {
        int dst[kBatch], src[kBatch], pd[kBatch], ps[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int j = j0 + i * stride;
            dst[i] = j < moves ? list_f[j] : -1;
            src[i] = j < moves ? list_p[j] : 0;
        }
        const int32_t* table = a.c.table + (int64_t)b * a.c.ld_table;
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            pd[i] = dst[i] >= 0 ? table[dst[i] >> a.c.shift] : -1;
            ps[i] = dst[i] >= 0 ? table[src[i] >> a.c.shift] : -1;
        }
        uint4 x[kBatch], y[kBatch];
        float w[kBatch];
        int pos[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            if (pd[i] < 0 || ps[i] < 0 || pd[i] >= a.c.n_pages || ps[i] >= a.c.n_pages) dst[i] = -1;  // reported with its key
            if (dst[i] < 0) continue;
            const int64_t from = a.c.row(ps[i], src[i], g) + at * 16, ms = a.c.meta(ps[i], src[i], g);
            x[i] = *reinterpret_cast<const uint4*>(a.c.k + from);
            y[i] = *reinterpret_cast<const uint4*>(a.c.v + from);
            w[i] = a.c.weight[ms];
            pos[i] = a.c.position[ms];
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            if (dst[i] < 0) continue;
            const int64_t to = a.c.row(pd[i], dst[i], g) + at * 16, md = a.c.meta(pd[i], dst[i], g);
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
    const int64_t grid = n_rows > 0 ? (n_rows + kAppendWarps - 1) / kAppendWarps : 1;
    append_kernel<<<(unsigned)grid, 32 * kAppendWarps, 0, st>>>(a);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? ESTP_OK : cuda_fail(e, "cache append launch");
}

estp_status launch_cache_evict(estp_ctx* ctx, const CacheView& c, int row_bytes, int B, const int32_t* length,
                               const int32_t* seen, int32_t* length_out, int budget, int recent, int sinks,
                               cudaStream_t st) {
    const int64_t groups = (int64_t)B * c.Hkv, cap = c.capacity();
    // CTAs of a cluster: enough clusters' CTAs for the SMs, while each keeps a run of 1024 slots
    int C = 1;
    while (C < kMaxCluster && groups * C * 2 <= ctx->num_sms && cap >= (int64_t)C * 2 * 1024) C *= 2;
    const int64_t run = ((cap + C - 1) / C + 31) / 32 * 32;
    const int64_t max_keys = 48 * 1024;  // 192 KB
    EvictArgs a{c, row_bytes, B, length, seen, length_out, budget, recent, sinks};
    a.key_cap = (int)(run < max_keys ? run : max_keys);
    const int64_t moves = cap > budget ? (cap - budget < budget ? cap - budget : budget) : 0;
    a.max_moves = (int)moves;
    estp_status s = ws_reserve(ctx, sizeof(int32_t) * 2 * (size_t)groups * (size_t)moves + 16);
    if (s != ESTP_OK) return s;
    a.list = static_cast<int32_t*>(ctx->ws);
    a.done = ctx->done;
    a.status = ctx->status;
    const size_t smem = sizeof(uint32_t) * (size_t)a.key_cap;
    cudaError_t e = cudaFuncSetAttribute(evict_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(max_keys * 4));
    if (e != cudaSuccess) return cuda_fail(e, "cache evict smem attribute");
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)C;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(groups * C));
    cfg.blockDim = dim3(kEvictThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, evict_kernel, a);
    if (e == cudaSuccess) e = cudaGetLastError();
    return e == cudaSuccess ? ESTP_OK : cuda_fail(e, "cache evict launch");
}

}  // namespace estp
